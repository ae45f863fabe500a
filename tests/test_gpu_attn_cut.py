"""Arrays on the device that say more than there is: a sequence is what of its rows lies inside the given ones, and no longer than len_q and len_k; beside those nothing is written.  The
given rows lie between others, which hold NaN or, where results go, a fill that has to stay."""
import pytest
import torch

from attn_ref import Case
from operators_ref import DEV

pytestmark = pytest.mark.gpu
LOW, HIGH = -2**31, 2**31 - 1
# lengths of what is left; q_starts; k_starts; k_lens or None.  60 rows are given, len_q and len_k are the longest of the lengths.
CUTS = {
    "in front and behind": ([(20, 20), (30, 30), (10, 10)], [-5, 20, 50, HIGH], [-9, 20, 50, HIGH], None),
    "longer than len_q and len_k": ([(20, 20), (30, 30), (0, 0)], [0, 20, 60, 60], [0, 20, 60, 60], None),
    "far outside": ([(0, 0), (0, 0), (60, 60)], [LOW, LOW, -1, HIGH], [LOW, LOW, LOW, HIGH], None),
    "backwards": ([(0, 0), (60, 60), (0, 0)], [HIGH, 0, 60, LOW], [HIGH, 0, 60, LOW], None),
    "lengths": ([(20, 20), (30, 0), (10, 5)], [-5, 20, 50, 61], [-7, 30, 55, LOW], [27, -3, HIGH]),
    "few queries": ([(2, 20), (16, 22), (1, 10)], [-5, 2, 18, 19], [-9, 20, 50, HIGH], [29, 22, 1000]),
    "few queries, longer": ([(16, 20), (4, 40), (0, 0)], [0, 56, 70, 90], [0, 20, HIGH, 5], [20, 100, 7]),
}


@pytest.mark.parametrize("hd,dtype,pad", [(64, "bf16", 0), (128, "f16", 0), (72, "f16", 3)])
@pytest.mark.parametrize("which", list(CUTS))
def test_what_reaches_past_the_rows_is_cut_off(paro, which, hd, dtype, pad):
    lengths, q_starts, k_starts, k_lens = CUTS[which]
    c = Case(paro, lengths, heads=4, kv=2, hd=hd, dtype=dtype, pad=pad, window=18, sinks=2, buckets=6)
    given = 60
    # Case packs from row 3 on, one sequence behind the other; here they lie where the arrays say
    into = lambda x: min(max(x, 0), given)                                                    # noqa: E731
    c.q_at, c.k_at = [into(x) for x in q_starts[:-1]], [into(x) for x in k_starts[:3]]
    generator = torch.Generator().manual_seed(4)
    for x, at, of in ((c.q, c.q_at, 0), (c.dout, c.q_at, 0), (c.out, c.q_at, 0), (c.dq, c.q_at, 0), (c.k, c.k_at, 1), (c.v, c.k_at, 1), (c.dk, c.k_at, 1), (c.dv, c.k_at, 1)):
        heads, written = x.view.shape[1], x in (c.out, c.dq, c.dk, c.dv)
        grown = type(x)(given + 6, heads, hd, pad, dtype, fill=5.0 if written else float("nan"))
        x.__dict__.update(grown.__dict__)
        x.view, held = x.view[3:], x.held[3:]
        for b, n in enumerate(lengths):
            rows = slice(at[b], at[b] + n[of])
            held[rows] = True
            if not written:
                x.put(rows, torch.randn(n[of], heads, hd, generator=generator))
    every = torch.full((given + 6, c.heads, 2), 5.0, device=DEV)
    c.stats, c.rows_q, c.rows_k = every[3:], given, given
    to = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)                             # noqa: E731
    c.q_starts, c.k_starts, c.k_lens = to(q_starts), to(k_starts), None if k_lens is None else to(k_lens)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
    rest = torch.ones(given + 6, dtype=torch.bool, device=DEV)
    for at, n in zip(c.q_at, lengths):
        rest[3 + at:3 + at + n[0]] = False
    assert bool((every[rest] == 5).all()), "wrote beside the rows of stats"
