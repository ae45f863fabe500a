"""Gradient of the attention with a window, sinks and a bias by buckets, against its definition in 64 bits and against differences."""
import pytest
import torch

from attn_ref import Case

pytestmark = pytest.mark.gpu
LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257]


def backward(paro, lengths, want_table=True, **kw):
    c = Case(paro, lengths, **kw)
    c.set_forward()
    c.backward(want_table)
    c.check_backward(want_table)
    held = [c.dq.whole, c.dk.whole, c.dv.whole] + ([c.dtable] if c.buckets else [])
    bits = [t.clone() for t in held]
    c.backward(want_table)
    assert all(torch.equal(a, b) for a, b in zip(bits, held)), "the same call gave other bits"
    return c


@pytest.mark.parametrize("n", LENGTHS)
def test_any_length(paro, n):
    backward(paro, [(n, n)], hd=64)
    backward(paro, [(n, n)], hd=128, dtype="f16", window=20, sinks=3, buckets=9, layout="dense")


@pytest.mark.parametrize("hd", [8, 9, 11, 16, 31, 32, 33, 56, 63, 64, 65, 72, 77, 80, 96, 120, 127, 128])
def test_any_head_width(paro, hd):
    backward(paro, [(70, 70)], hd=hd, heads=3, pad=hd % 3)
    backward(paro, [(5, 150)], hd=hd, dtype="f16", pad=5, heads=4, kv=2)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (31, 0), (32, 1), (33, 64), (63, 63), (64, 0), (65, 65), (100, 4), (128, 130), (129, 200), (400, 7), (2**40, 2**40)])
def test_any_window_and_sinks(paro, window, sinks):
    backward(paro, [(300, 300)], hd=64, window=window, sinks=sinks)
    backward(paro, [(131, 300)], hd=128, window=window, sinks=sinks, dtype="f16", buckets=8, far=20)


@pytest.mark.parametrize("buckets,far", [(1, 1), (2, 5), (3, 2), (8, 10), (32, 128), (33, 100), (128, 3000), (255, 200), (256, 128)])
@pytest.mark.parametrize("dtype,table", [("bf16", "f32"), ("f16", "f16"), ("bf16", "bf16")])
def test_any_buckets(paro, buckets, far, dtype, table):
    backward(paro, [(260, 260), (33, 40)], heads=3, buckets=buckets, far=far, dtype=dtype, table=table)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (4, 2), (8, 1), (17, 1), (12, 12)])
def test_head_groups(paro, heads, kv):
    backward(paro, [(50, 50), (37, 37)], heads=heads, kv=kv, hd=32, dtype="f16", window=20, sinks=2, buckets=6)
    backward(paro, [(150, 150)], heads=heads, kv=kv, hd=128)


@pytest.mark.parametrize("layout", ["packed", "dense", "planes"])
@pytest.mark.parametrize("use_lens", [False, True])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_layouts(paro, layout, use_lens, pad):
    backward(paro, [(40, 40)] * 3 if layout == "dense" else [(40, 40), (1, 1), (129, 200)], layout=layout, use_lens=use_lens, pad=pad, heads=4, kv=2, hd=72)


@pytest.mark.parametrize("hd", [64, 128])
def test_sequences_of_nothing(paro, hd):
    for buckets in (0, 5):
        backward(paro, [(20, 20), (0, 30), (50, 0), (0, 0), (150, 20), (33, 33)], hd=hd, buckets=buckets, dtype="f16")
        backward(paro, [(20, 0)], hd=hd, buckets=buckets)
        backward(paro, [(0, 20)], hd=hd, buckets=buckets)


def test_long_sequences(paro):
    """Keys and sinks that are shared out among blocks."""
    backward(paro, [(1100, 1100)], heads=1, hd=128, window=100, sinks=4)
    backward(paro, [(1500, 1500)], heads=2, kv=1, hd=64, window=200, sinks=140, buckets=32, far=128, dtype="f16")
    backward(paro, [(700, 1500)], heads=1, hd=64, buckets=32, far=128)
    backward(paro, [(700, 700)], heads=6, window=40, sinks=4)
    backward(paro, [(700, 700)], heads=6, window=40, sinks=140, dtype="f16", buckets=8)


@pytest.mark.parametrize("spread", [1e-6, 3e4])
def test_small_and_large_gradients(paro, spread):
    """fp16: the products' scores of gradients would leave its range on either side."""
    backward(paro, [(140, 140)], spread=spread, hd=64, dtype="f16", buckets=8)
    backward(paro, [(140, 140)], spread=spread, hd=128, dtype="bf16")


@pytest.mark.parametrize("hd", [64, 72])
def test_keys_that_no_query_sees(paro, hd):
    """Between the sinks and the first window: whatever they hold, their gradients are zeros and the others as they were."""
    c = Case(paro, [(200, 500)], window=60, sinks=3, hd=hd, heads=2)
    gone = slice(c.k_at[0] + 3, c.k_at[0] + 500 - 200 - 60 + 1)
    c.set_forward()
    c.backward()
    c.check_backward()
    want = [x.view.clone() for x in (c.dq, c.dk, c.dv)]
    assert bool((want[1][gone] == 0).all()) and bool((want[2][gone] == 0).all())
    c.k.view[gone] = torch.inf
    c.v.view[gone] = torch.nan
    c.backward()
    assert all(torch.equal(x.view, y) for x, y in zip((c.dq, c.dk, c.dv), want))


def test_without_the_tables_gradient(paro):
    c = backward(paro, [(150, 150)], want_table=False, buckets=8)
    assert bool((c.dtable == 7).all())


def test_a_table_that_hides(paro):
    for value in (-torch.inf, torch.finfo(torch.float32).min):
        c = Case(paro, [(150, 150)], buckets=6, far=30)
        c.table[1] = value
        c.table[5] = value
        c.set_forward()
        c.backward()
        c.check_backward()
        c.table[:] = value                        # every row: nothing seen, or all alike
        c.set_forward()
        c.backward()
        c.check_backward()


def test_against_differences(paro):
    """d/dx of sum(dout * out) along a random direction, from the forward pass in 64 bits."""
    c = Case(paro, [(60, 60)], heads=2, hd=16, dtype="f16", window=25, sinks=2, buckets=6, far=20)
    c.set_forward()
    c.backward()
    g = torch.Generator().manual_seed(3)
    inputs = [c.rows_of(x, c.q_at[0], 60) for x in (c.q, c.k, c.v)] + [c.table.double().cpu()]
    dout = c.rows_of(c.dout, c.q_at[0], 60)
    of = (torch.tensor(c.first_list)[None] <= torch.arange(61)[:, None]).sum(1) - 1
    far, seen = c.pairs(60, 60)

    def value(q, k, v, table):
        s = torch.einsum("ihd,jhd->hij", q, k) * c.scale + table[of][far.clamp(min=0)].permute(2, 0, 1)
        return (torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(~seen, -torch.inf), 2), v) * dout).sum()

    got = [c.rows_of(x, c.q_at[0], 60) for x in (c.dq, c.dk, c.dv)] + [c.dtable.double().cpu()]
    # What a gradient may be off: its bound against the formula; and the formula takes out as it was rounded, by which D_i is off half a unit of each product.
    q, k, v, table = inputs
    P = torch.softmax((torch.einsum("ihd,jhd->hij", q, k) * c.scale + table[of][far.clamp(min=0)].permute(2, 0, 1)).masked_fill(~seen, -torch.inf), 2)
    off = P * (dout * torch.einsum("hij,jhd->ihd", P, v)).abs().sum(2).t()[:, :, None] * 2.0 ** -11
    more = [c.scale * torch.einsum("hij,jhd->ihd", off, k.abs()), c.scale * torch.einsum("hij,ihd->jhd", off, q.abs()), 0 * v,
            torch.zeros_like(table).index_add_(0, of[far.clamp(min=0)].flatten(), off.flatten(1).t())]
    c.check_backward()
    for which in range(4):
        way = torch.randn(inputs[which].shape, generator=g, dtype=torch.float64)
        up, down = ([x + h * way if i == which else x for i, x in enumerate(inputs)] for h in (1e-5, -1e-5))
        slope = (value(*up) - value(*down)) / 2e-5
        # 1.01: the statistics, rounded to fp32, move a share by less than a hundredth of an fp16 unit; 1e-7: the third difference
        assert ((got[which] * way).sum() - slope).abs() < ((1.01 * c.bounds[which] + 1.01 * more[which]) * way.abs()).sum() + 1e-7 * slope.abs()


def test_forward_and_backward_together(paro):
    """As a training step has them: the gradient from what the forward pass left."""
    for dtype, buckets in (("bf16", 0), ("f16", 7)):
        c = Case(paro, [(200, 200), (77, 77)], heads=4, kv=2, hd=64, dtype=dtype, window=60, sinks=3, buckets=buckets)
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_row_that_is_not_finite_stays_in_its_place(paro, dtype):
    """A row of infinite gradient: its own dq, and keys up to its tile of 32 queries; nothing of other heads, earlier keys' other rows or another sequence."""
    c = Case(paro, [(200, 200), (90, 90)], heads=2, hd=64, dtype=dtype, spread=1e4)
    c.set_forward()
    c.backward()
    want = [x.view.clone() for x in (c.dq, c.dk, c.dv)]
    row = c.q_at[0] + 100
    c.dout.view[row, 0] = torch.inf
    c.backward()
    got = [x.view for x in (c.dq, c.dk, c.dv)]
    assert torch.equal(got[0][row + 1:, 0], want[0][row + 1:, 0]) and torch.equal(got[0][c.q_at[0]:row, 0], want[0][c.q_at[0]:row, 0])
    assert not got[0][row, 0].isfinite().any() and not got[1][c.k_at[0]:c.k_at[0] + 101, 0].isfinite().any()
    for x, y in zip(got, want):
        assert torch.equal(x[c.q_at[0]:, 1].nan_to_num(7), y[c.q_at[0]:, 1].nan_to_num(7)) and torch.equal(x[c.q_at[1]:].nan_to_num(7), y[c.q_at[1]:].nan_to_num(7))
        assert torch.equal(x[c.q_at[0] + 128:c.q_at[0] + 200], y[c.q_at[0] + 128:c.q_at[0] + 200])


@pytest.mark.parametrize("sequences,heads,kv,hd", [(43, 32, 1, 16), (70, 12, 12, 8)])
def test_many_sequences(paro, sequences, heads, kv, hd):
    """More than an XCD takes at a time, and some left over: few key heads of many blocks, many of two."""
    n = [(7 * b % 160, 7 * b % 160) for b in range(sequences)]
    backward(paro, n, heads=heads, kv=kv, hd=hd, window=90, sinks=3, buckets=6)
