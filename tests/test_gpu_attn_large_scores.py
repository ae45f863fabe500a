"""Scores of millions and scales from 2^-59 to 2^59.  Heads hold whole numbers whose sums of products are below 2^24 and scales are powers of two, so that a score is exact in fp32 whatever the order
of its sum: what a kernel may be off is a difference's exponential, however large the scores."""
import pytest
import torch

import attn_ref
from attn_ref import Case
from operators_ref import check as check_within

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def infinities(monkeypatch):
    """fp16 rounds to an infinity exactly what lies 65520 = 65504 + half a step and more from zero, on its side.  A result may lie anywhere within `bound` of ref, so an infinity of sign s is a
    rounding of what it may be where s * ref + bound >= 65520.  (Where a scale of 2^20 and more multiplies the roundings of dS, ref is zero or of either sign there.)"""
    def check_rounded(got, ref, bound, dtype, what):
        got = got.detach().cpu().double()
        if dtype == "f16":
            got = torch.where(got.isinf() & (got.sign() * ref + bound >= 65520), ref, got)
        check_within(got, ref, bound, what)
    monkeypatch.setattr(attn_ref, "check_rounded", check_rounded)


class Exact(Case):
    """high: the scores' common part, in 2^22, before the scale."""

    def __init__(self, paro, lengths, scale, high, bias=True, **kw):
        super().__init__(paro, lengths, **kw)
        g = torch.Generator().manual_seed(7)
        self.scale = scale
        for b, (nq, nk) in enumerate(self.lengths):
            q, k = torch.zeros(nq, self.heads, self.hd), torch.zeros(nk, self.kv, self.hd)
            q[..., 1:8] = torch.randint(-1, 2, (nq, self.heads, 7), generator=g)
            k[..., 1:8] = torch.randint(-2, 3, (nk, self.kv, 7), generator=g)
            q[..., 0] = 2048.0 + 16 * torch.randint(0, 32, (nq, self.heads), generator=g)         # rows differ in how their largest score rounds
            k[..., 0] = 2048.0 * high
            self.q.put(slice(self.q_at[b], self.q_at[b] + nq), q)
            self.k.put(slice(self.k_at[b], self.k_at[b] + nk), k)
        if self.buckets:
            self.table.copy_(torch.randint(-3, 4, self.table.shape, generator=g))

    def scores(self, b, h):
        s, off, far, seen = super().scores(b, h)
        return s, torch.zeros_like(off), far, seen

    def check(self, which):
        """The bounds of Case for a bias hold no share of the largest score's size: one bucket of zeros stands for none."""
        plain = self.buckets == 0
        if plain:
            self.buckets, self.first_list, self.table = 1, [0], torch.zeros(1, self.heads)
        which(*([False] if plain and which == self.check_backward else []))
        if plain:
            self.buckets, self.table = 0, None


def both(paro, lengths, scale, high, backward=True, **kw):
    c = Exact(paro, lengths, scale, high, **kw)
    c.forward()
    c.check(c.check_forward)
    if backward:
        c.backward()
        c.check(c.check_backward)
    return c


SCALES = [(1.0, 1), (1.0, -1), (1.0, 0), (2.0 ** -4, 1), (2.0 ** 6, 1), (2.0 ** 20, -1), (2.0 ** 59, 1), (2.0 ** 59, 0), (2.0 ** -59, 1)]


@pytest.mark.parametrize("scale,high", SCALES)
@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (72, "f16"), (128, "f16")])
def test_many_queries(paro, hd, dtype, scale, high):
    both(paro, [(200, 200), (40, 70), (20, 5)], scale, high, hd=hd, dtype=dtype, heads=4, kv=2)
    both(paro, [(300, 300)], scale, high, hd=hd, dtype=dtype, window=90, sinks=3)


@pytest.mark.parametrize("scale,high", SCALES)
@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "f16")])
def test_few_queries(paro, hd, dtype, scale, high):
    for n in (1, 5, 16):
        both(paro, [(n, 300), (n, 17)], scale, high, hd=hd, dtype=dtype, heads=4, kv=2)
    both(paro, [(2, 4000), (2, 100)], scale, high, hd=hd, dtype=dtype, backward=False)


@pytest.mark.parametrize("scale,high", SCALES)
@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "f16")])
def test_keys_shared_among_blocks(paro, hd, dtype, scale, high):
    both(paro, [(64, 5000)], scale, high, hd=hd, dtype=dtype, backward=False)
    both(paro, [(1100, 1100)], scale, high, hd=hd, dtype=dtype, heads=1, window=200, sinks=4)


# with a bias a score is exact up to 2^24
@pytest.mark.parametrize("scale,high", [(1.0, 1), (1.0, -1), (2.0 ** -4, 1), (1.0, 0)])
@pytest.mark.parametrize("hd,dtype", [(64, "bf16"), (128, "bf16"), (72, "f16")])
@pytest.mark.parametrize("far", [40, 1500])
def test_with_a_bias(paro, hd, dtype, far, scale, high):
    """Tiles all of whose distances have the last bucket, and others."""
    kw = dict(hd=hd, dtype=dtype, buckets=12, far=far, table="f32")
    both(paro, [(300, 300), (20, 5)], scale, high, heads=4, kv=2, **kw)
    both(paro, [(3, 300)], scale, high, **kw)
    both(paro, [(64, 5000)], scale, high, backward=True, **kw)


@pytest.mark.parametrize("lengths", [[(200, 200)], [(1, 300), (16, 300), (9, 9)], [(64, 5000)]])
@pytest.mark.parametrize("hd,buckets", [(64, 0), (128, 0), (128, 12)])
def test_shares_are_at_most_one(paro, hd, buckets, lengths):
    """Scores of 10^8 to 10^9 whose sums round: the forward pass gives means of values all the same, and the gradient, which has to form the same scores to the bit (few queries take other products forward
    than backward), a P of at most exp(-log_sum), which is at most one.  So |out| is at most the largest |v| and |dv_j| the sum of |dout_i| over queries and heads, each but for its roundings: of out by half a step, its
    shares by another; of P and dv by half a step each; of sums by 2^-24 a term."""
    for dtype, size in (("bf16", 3e4), ("f16", 1e4)):
        c = Case(paro, lengths, heads=4, kv=2, hd=hd, dtype=dtype, buckets=buckets, size=size)
        c.k.view.mul_(size).clamp_(-6e4, 6e4)
        c.q.view.clamp_(-6e4, 6e4)
        c.forward()
        c.backward()
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
        for (nq, nk), q_at, k_at in zip(lengths, c.q_at, c.k_at):
            out, dout = (x.view[q_at:q_at + nq].double() for x in (c.out, c.dout))
            v, dv = (x.view[k_at:k_at + nk].double() for x in (c.v, c.dv))
            assert bool((out.abs() <= v.abs().amax(0).repeat_interleave(2, 0) * (1 + half) * (1 + half) * (1 + 2 * nk * 2.0 ** -24) + 2.0 ** -25).all())
            most = dout.abs().sum(0).unflatten(0, (2, 2)).sum(1)
            assert bool((dv.abs() <= most * (1 + half) ** 2 * (1 + 4 * nq * 2.0 ** -24) + 2.0 ** -25).all()), float((dv.abs() / most).max())
            if dtype == "bf16":
                assert all(bool(x.view[at:at + n].isfinite().all()) for x, at, n in ((c.dq, q_at, nq), (c.dk, k_at, nk)))
