"""Attention with a window, sinks and a bias by buckets, forward, against its definition in 64 bits: lengths that begin and end tiles, every head width,
windows and sinks that cut tiles, layouts, sequences of no query or key, queries in front of the first key, what lies between and behind the rows."""
import pytest

from attn_ref import Case

pytestmark = pytest.mark.gpu
LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257]


def forward(paro, lengths, stats=True, **kw):
    c = Case(paro, lengths, **kw)
    c.forward(stats)
    c.check_forward(stats)
    bits = c.out.whole.clone()
    c.forward(stats)
    assert bool((c.out.whole.view(-1) == bits).all()), "the same call gave other bits"
    return c


@pytest.mark.parametrize("n", LENGTHS)
def test_any_length(paro, n):
    forward(paro, [(n, n)], hd=64)
    forward(paro, [(n, n)], hd=128, dtype="f16", window=20, sinks=3, buckets=9, layout="dense", stats=False)


@pytest.mark.parametrize("hd", [8, 9, 11, 16, 31, 32, 33, 56, 63, 64, 65, 72, 77, 80, 96, 120, 127, 128])
def test_any_head_width(paro, hd):
    forward(paro, [(70, 70)], hd=hd, heads=3, pad=hd % 3)
    forward(paro, [(5, 150)], hd=hd, dtype="f16", pad=5, heads=4, kv=2)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 5), (31, 0), (32, 1), (33, 64), (63, 63), (64, 0), (65, 65), (100, 4), (128, 130), (129, 200), (400, 7), (2**40, 2**40)])
def test_any_window_and_sinks(paro, window, sinks):
    forward(paro, [(300, 300)], hd=64, window=window, sinks=sinks)
    forward(paro, [(131, 300)], hd=128, window=window, sinks=sinks, dtype="f16", buckets=8, far=20)
    forward(paro, [(3, 300)], hd=64, window=window, sinks=sinks, heads=2, kv=1)


@pytest.mark.parametrize("buckets,far", [(1, 1), (2, 5), (3, 2), (8, 10), (32, 128), (33, 100), (128, 3000), (255, 200), (256, 128)])
@pytest.mark.parametrize("dtype,table", [("bf16", "f32"), ("f16", "f16"), ("bf16", "bf16")])
def test_any_buckets(paro, buckets, far, dtype, table):
    forward(paro, [(260, 260)], heads=3, buckets=buckets, far=far, dtype=dtype, table=table)
    forward(paro, [(4, 260), (2, 1)], heads=4, kv=2, buckets=buckets, far=far, dtype=dtype, table=table, window=77, sinks=2)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (4, 2), (8, 1), (17, 1), (12, 12), (40, 4)])
@pytest.mark.parametrize("new", [1, 2, 5, 16, 17])
def test_head_groups(paro, heads, kv, new):
    forward(paro, [(new, 100), (new, 37)], heads=heads, kv=kv, hd=32, dtype="f16", window=50, sinks=2, buckets=6)
    forward(paro, [(new, 70)], heads=heads, kv=kv, hd=128)


@pytest.mark.parametrize("layout", ["packed", "dense", "planes"])
@pytest.mark.parametrize("use_lens", [False, True])
@pytest.mark.parametrize("pad", [0, 3, 8])
def test_layouts(paro, layout, use_lens, pad):
    forward(paro, [(40, 40)] * 3 if layout == "dense" else [(40, 40), (1, 1), (129, 200)], layout=layout, use_lens=use_lens, pad=pad, heads=4, kv=2, hd=72)
    forward(paro, [(2, 40), (2, 300), (2, 5)], layout=layout, use_lens=use_lens, pad=pad, heads=4, kv=2, hd=40, window=33, sinks=1)


@pytest.mark.parametrize("hd", [64, 128])
def test_sequences_of_nothing(paro, hd):
    """No query, no key, neither; more queries than keys, of which the first stand in front of every key."""
    for buckets in (0, 5):
        forward(paro, [(20, 20), (0, 30), (50, 0), (0, 0), (150, 20), (33, 33)], hd=hd, buckets=buckets)
        forward(paro, [(3, 20), (0, 30), (5, 0), (0, 0), (16, 2), (7, 33)], hd=hd, buckets=buckets, window=9, sinks=1, dtype="f16")
        forward(paro, [(5, 0), (3, 0)], hd=hd, buckets=buckets)
        forward(paro, [(50, 0)], hd=hd, buckets=buckets, use_lens=True)


@pytest.mark.parametrize("new", [1, 3, 16])
def test_long_caches(paro, new):
    """Shared out among many blocks, with and without a window; ends inside every kind of tile."""
    forward(paro, [(new, 4001), (new, 3000), (new, 129)], heads=2, hd=64)
    forward(paro, [(new, 5000), (new, 31)], heads=4, kv=2, hd=128, window=3001, sinks=70, buckets=32, far=128, dtype="f16")


def test_long_sequences(paro):
    forward(paro, [(1100, 1100)], heads=1, hd=128, window=500, sinks=4)
    forward(paro, [(700, 1500)], heads=1, hd=64, buckets=32, far=128)


@pytest.mark.parametrize("size", [1e-3, 30.0])
def test_small_and_large_scores(paro, size):
    forward(paro, [(140, 140), (2, 300)], size=size, hd=64)
    forward(paro, [(140, 140), (2, 300)], size=size, hd=128, buckets=8, dtype="f16")


def test_a_table_that_hides(paro):
    """-inf in the table: a bucket of distances is not seen; with every bucket, nothing is.  A type's lowest number for all: as zeros for all."""
    import torch
    for lengths in ([(150, 150)], [(3, 150)]):
        c = Case(paro, lengths, buckets=6, far=30)
        c.table[1] = -torch.inf
        c.table[5] = -torch.inf
        c.forward()
        c.check_forward()
        c.table[:] = -torch.inf
        c.forward()
        c.check_forward()
        assert bool((c.out.view[c.q_at[0]:c.q_at[0] + lengths[0][0]] == 0).all())
        c.table[:] = torch.finfo(torch.float32).min
        c.forward()
        low = c.out.view.clone()
        c.table[:] = 0
        c.q.view[:] = 0
        c.forward()
        assert torch.equal(low[c.q_at[0]:c.q_at[0] + lengths[0][0]], c.out.view[c.q_at[0]:c.q_at[0] + lengths[0][0]])


def test_keys_that_no_query_sees_are_not_read(paro):
    """What left the window of a cache may hold anything."""
    import torch
    for new in (1, 5, 16, 40):
        c = Case(paro, [(new, 500)], window=100, sinks=5, hd=128)
        gone = slice(c.k_at[0] + 5, c.k_at[0] + 500 - new - 100 + 1)
        c.forward()
        want = c.out.view[c.q_at[0]:c.q_at[0] + new].clone()
        c.k.view[gone] = torch.inf
        c.v.view[gone] = torch.nan
        c.forward()
        assert torch.equal(want, c.out.view[c.q_at[0]:c.q_at[0] + new])


def test_arrays_on_the_device_that_reach_too_far_are_cut_off(paro):
    """Whatever the arrays hold, no row outside the given ones is touched (rows past the end would be other memory: here they are the same buffer's)."""
    import torch
    c = Case(paro, [(40, 40), (30, 30)], layout="packed")
    c.q_starts[:] = torch.tensor([-5, 1 << 30, -(1 << 31)], dtype=torch.int32)
    c.k_starts[:] = torch.tensor([1 << 30, -7, 2**31 - 1], dtype=torch.int32)
    c.forward()
    torch.cuda.synchronize()


@pytest.mark.parametrize("sequences,heads,kv,hd", [(43, 32, 1, 16), (70, 12, 12, 8)])
def test_many_sequences(paro, sequences, heads, kv, hd):
    """More than an XCD takes at a time, and some left over: few key heads of many blocks, many of two."""
    n = [(7 * b % 160, 7 * b % 160) for b in range(sequences)]
    forward(paro, n, heads=heads, kv=kv, hd=hd, window=90, sinks=3, buckets=6)


@pytest.mark.parametrize("hd,dtype,buckets", [(64, "bf16", 0), (128, "f16", 0), (40, "f16", 9), (128, "bf16", 32), (77, "bf16", 0)])
def test_keys_shared_among_blocks(paro, hd, dtype, buckets):
    """More than 16 queries over many keys, in fewer blocks than the chip has room for: a few shares, by eights, shares of nothing, sequences of few keys or none."""
    forward(paro, [(64, 5000)], hd=hd, dtype=dtype, buckets=buckets, far=128)
    forward(paro, [(17, 20500), (150, 3000), (40, 10), (30, 0), (0, 50)], heads=3, kv=1, hd=hd, dtype=dtype, buckets=buckets, pad=3, stats=False)
    forward(paro, [(33, 9000), (20, 70)], heads=4, kv=2, hd=hd, dtype=dtype, buckets=buckets, window=5001, sinks=40, use_lens=True)
    forward(paro, [(2200, 2200)], heads=1, hd=hd, dtype=dtype, buckets=buckets)
