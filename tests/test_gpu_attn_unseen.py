"""What the attention does not look at is of no account, fp16 with its common power of two included: keys between the sinks and the first window, queries that see no key."""
import pytest
import torch

from attn_ref import Case

pytestmark = pytest.mark.gpu


def gradients(c):
    c.set_forward()
    c.backward()
    return [x.whole.clone() for x in (c.dq, c.dk, c.dv)] + ([c.dtable.clone()] if c.buckets else [])


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("hd,pad", [(64, 0), (128, 0), (72, 0), (77, 3)])
@pytest.mark.parametrize("sinks", [0, 3, 20])
def test_large_values_that_no_query_sees(paro, sinks, hd, pad):
    """Large numbers in keys and values that have left the window: every gradient to the bit as with zeros there."""
    c = Case(paro, [(200, 500), (40, 60), (0, 70), (33, 33)], window=60, sinks=sinks, hd=hd, pad=pad, heads=4, kv=2, dtype="f16", buckets=6, spread=8.0)
    gone = []
    for (nq, nk), at in zip(c.lengths, c.k_at):
        first = nk - nq - 60 + 1 if nq else nk               # the first query's window begins here
        gone.append(slice(at + min(sinks if nq else 0, nk), at + max(first, 0)))
    assert gone[0].stop - gone[0].start > 200 and gone[2].stop - gone[2].start == 70
    gone = [s for s in gone if s.stop > s.start]
    got = []
    for value in (0.0, 60000.0, -60000.0):
        for s in gone:
            c.k.view[s] = value
            c.v.view[s] = value
        got.append(gradients(c))
        if value == 0.0:
            c.check_backward()
    assert same(got[0], got[1]) and same(got[0], got[2])


@pytest.mark.parametrize("hd", [64, 128])
def test_large_gradients_of_queries_that_see_no_key(paro, hd):
    """More queries than keys: those in front of the first key."""
    c = Case(paro, [(200, 50), (40, 40)], hd=hd, heads=2, dtype="f16", buckets=6, spread=1e-3)
    got = []
    for value in (0.0, 60000.0):
        c.dout.view[c.q_at[0]:c.q_at[0] + 150] = value
        got.append(gradients(c))
    assert same(*got)
    c.dout.view[c.q_at[0]:c.q_at[0] + 150] = 0.0
    gradients(c)
    c.check_backward()


def test_large_gradients_of_queries_whose_keys_are_hidden(paro):
    """A table of -inf hides every key from a head."""
    c = Case(paro, [(200, 200), (40, 40)], heads=4, kv=2, dtype="f16", buckets=6, spread=1e-3)
    c.table[:, 2] = -torch.inf
    got = []
    for value in (0.0, 60000.0):
        c.dout.view[c.q_at[0]:, 2] = value
        got.append(gradients(c))
    assert same(*got)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("hd,pad", [(64, 0), (128, 0), (77, 3)])
def test_queries_that_see_no_key_hold_anything(paro, hd, pad, dtype):
    """More queries than keys: NaN and infinities in those in front of the first key stay out of every other row, and their own results are zeros."""
    for nq, nk in ((200, 50), (161, 1), (40, 39), (300, 0)):
        c = Case(paro, [(nq, nk), (40, 40)], hd=hd, pad=pad, heads=4, kv=2, dtype=dtype, buckets=6, window=30, sinks=2)
        rows = slice(c.q_at[0], c.q_at[0] + nq - nk)
        got = []
        for value in (0.0, torch.nan, torch.inf):
            c.q.view[rows] = value
            c.dout.view[rows] = value
            c.forward()
            c.backward()
            got.append([x.clone() for x in (c.out.whole, c.stats, c.dq.whole, c.dk.whole, c.dv.whole, c.dtable)])
            if value == 0.0:
                c.check_forward()
                c.check_backward()
        assert same(got[0], got[1]) and same(got[0], got[2])
        assert bool((c.out.view[rows] == 0).all()) and bool((c.dq.view[rows] == 0).all())
