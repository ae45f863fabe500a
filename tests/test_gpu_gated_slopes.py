"""The backward pass of the gated projections in fp16 where the slopes dg and du leave the type's range: many tokens, for which they are rounded
on their way to the matrix cores."""
import math

import pytest
import torch

from operators_ref import DEV, EPS32, FLOOR, HALF_ULP, check, put, rng, rounding, rows, stream, workspace

pytestmark = pytest.mark.gpu


def act64(g, act):
    if act == "silu":
        y = torch.sigmoid(g)
        return g * y, y * (1 + g * (1 - y))
    y = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
    return g * y, y + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def backward(paro, n, dim, hidden, act, of_dh, of_up, of_x, of_w, spread=None, pad=0, buffers=None):
    """of_*: sizes of the inputs' values.  spread: factors of dh's columns."""
    g = rng(n + dim)
    x, x64 = put(torch.randn(n, dim, generator=g) * of_x, pad, "f16")
    (wg, wg64), (wu, wu64) = (put(torch.randn(hidden, dim, generator=g) * of_w, 0, "f16") for _ in range(2))
    gate, g64 = put(torch.randn(n, hidden, generator=g) * 1.3, pad, "f16")
    up, u64 = put(torch.randn(n, hidden, generator=g) * of_up, pad, "f16")
    dh, dh64 = put(torch.randn(n, hidden, generator=g) * of_dh * (1.0 if spread is None else spread), pad, "f16")
    whole, dx = rows(n, dim, pad, "f16", fill=5.0)
    dwg, dwu = (torch.full((hidden, dim), 7.0, dtype=torch.float16, device=DEV) for _ in range(2))
    d = paro.make_gated(n=n, dim=dim, hidden=hidden, dtype=paro.PARO_F16, act=paro.PARO_SILU if act == "silu" else paro.PARO_GELU, ld_x=dim + pad,
                        ld_h=hidden + pad)
    ws = workspace(paro.paro_gated_workspace(d, True))
    call = [d, dh.data_ptr(), gate.data_ptr(), up.data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), dx.data_ptr(), dwg.data_ptr(), dwu.data_ptr(),
            ws.data_ptr(), ws.numel(), stream()]
    paro.paro_gated_grad(*call)
    a64, slope = act64(g64, act)
    dg64, du64 = dh64 * u64 * slope, dh64 * a64
    # half an ulp of each, or of the smallest number beside the largest: 25 binary places below it at least
    floor = 2.0 ** -25 * float(torch.maximum(dg64.abs().max(), du64.abs().max()))

    def off(v, size):
        e = 16 * EPS32 * size
        return e + HALF_ULP["f16"] * (v.abs() + e) + floor
    edg, edu = off(dg64, (dh64 * u64).abs() * (1 + g64.abs())), off(du64, (dh64 * g64).abs())
    size = dg64.abs() @ wg64.abs() + du64.abs() @ wu64.abs()
    dx64, edx = dg64 @ wg64 + du64 @ wu64, edg @ wg64.abs() + edu @ wu64.abs()
    assert float(dx64.abs().max()) < 6e4 and float((dg64.t() @ x64).abs().max()) < 6e4, "the case's own results leave the range"
    check(dx, dx64, rounding(dx64, "f16", edx + 2 * (2 * hidden + 4) * EPS32 * (size + edx)), "dx")
    for got, v, e, what in ((dwg, dg64, edg, "dwg"), (dwu, du64, edu, "dwu")):
        ref, err = v.t() @ x64, e.t() @ x64.abs()
        check(got, ref, rounding(ref, "f16", err + 2 * (n + 4) * EPS32 * (v.abs().t() @ x64.abs() + err)), what)
    bits = [t.clone() for t in (dx, dwg, dwu)]
    ws.fill_(0x3C)
    paro.paro_gated_grad(*call)
    assert all(torch.equal(a, b) for a, b in zip(bits, (dx, dwg, dwu))), "the same call gave other bits"
    dx.fill_(5.0)
    assert bool((whole == 5.0).all()), "wrote between the rows"


# together in one launch, dx and dW each on its own, odd rows
SIZES = [(40, 72, 136, 0), (333, 130, 257, 3), (1500, 2048, 4096, 0)]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,dim,hidden,pad", SIZES)
def test_slopes_beyond_the_largest_number(paro, n, dim, hidden, pad, act):
    """dh * u passes 65504, what it is multiplied by is small: dx, dWg and dWu are ordinary numbers."""
    backward(paro, n, dim, hidden, act, 400.0, 400.0, 2.0 ** -10, 2.0 ** -11, pad=pad)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("n,dim,hidden,pad", SIZES)
def test_slopes_among_the_subnormals(paro, n, dim, hidden, pad, act):
    """Slopes around 1e-7, of which fp16 keeps a binary place or two, beside inputs that lift their sums to where it keeps all."""
    backward(paro, n, dim, hidden, act, 2.0 ** -13, 2.0 ** -10, 64.0, 64.0, pad=pad)


@pytest.mark.parametrize("n,dim,hidden,pad", SIZES)
def test_slopes_of_many_sizes(paro, n, dim, hidden, pad):
    spread = 2.0 ** (torch.arange(hidden) % 16 - 8.0)
    backward(paro, n, dim, hidden, "silu", 4.0, 100.0, 2.0 ** -9, 2.0 ** -11, spread=spread, pad=pad)
    backward(paro, n, dim, hidden, "gelu", 2.0 ** -12, 0.25, 1.0, 1.0, spread=spread, pad=pad)


@pytest.mark.parametrize("size", [1.0, 3000.0, 2.0 ** -12])
def test_infinities_stay_in_their_rows(paro, size):
    """What no power of two brings into range spoils its own token and its own hidden element, and scales nothing else."""
    n, dim, hidden, g, small = 60, 64, 136, rng(3), 2.0 ** -14 if size > 1 else 2.0 ** -6
    x, gate, up, dh = (torch.randn(n, w, generator=g) for w in (dim, hidden, hidden, hidden))
    wg, wu = (torch.randn(hidden, dim, generator=g) * small for _ in range(2))
    d = paro.make_gated(n=n, dim=dim, hidden=hidden, dtype=paro.PARO_F16, act=paro.PARO_SILU)
    ws = workspace(paro.paro_gated_workspace(d, True))

    def run(dh):
        t = [v.to(DEV, torch.float16) for v in (dh, gate, up * size, x * small, wg, wu)]
        out = [torch.empty(s, dtype=torch.float16, device=DEV) for s in ((n, dim), (hidden, dim), (hidden, dim))]
        paro.paro_gated_grad(d, *[v.data_ptr() for v in t + out], ws.data_ptr(), ws.numel(), stream())
        return out
    clean = run(dh * size)
    dh[17, 5], dh[31, 9] = math.inf, math.nan
    spoilt = run(dh * size)
    for a, b, spoils in zip(clean, spoilt, ((17, 31), (5, 9), (5, 9))):
        keep = torch.ones(a.shape[0], dtype=torch.bool)
        keep[list(spoils)] = False
        assert bool(a.isfinite().all()) and not bool(b[~keep.to(DEV)].isfinite().any())
        assert bool(b[keep.to(DEV)].isfinite().all())


def test_zero_gradient(paro):
    d = paro.make_gated(n=50, dim=64, hidden=72, dtype=paro.PARO_F16)
    g, ws = rng(1), workspace(paro.paro_gated_workspace(d, True))
    t = [torch.zeros(50, 72)] + [torch.randn(*s, generator=g) for s in ((50, 72), (50, 72), (50, 64), (72, 64), (72, 64))]
    t = [v.to(DEV, torch.float16) for v in t]
    out = [torch.full(s, 3.0, dtype=torch.float16, device=DEV) for s in ((50, 64), (72, 64), (72, 64))]
    paro.paro_gated_grad(d, *[v.data_ptr() for v in t + out], ws.data_ptr(), ws.numel(), stream())
    assert all(bool((o == 0).all()) for o in out)


def test_in_a_graph_whose_slopes_change_size(paro):
    n, dim, hidden, g = 150, 104, 200, rng(2)
    d = paro.make_gated(n=n, dim=dim, hidden=hidden, dtype=paro.PARO_F16)
    shapes = ((n, hidden), (n, hidden), (n, hidden), (n, dim), (hidden, dim), (hidden, dim))
    t = [(torch.randn(*s, generator=g) * f).to(DEV, torch.float16) for s, f in zip(shapes, (1.0, 1.0, 1.0, 2.0 ** -9, 2.0 ** -9, 2.0 ** -9))]
    ref, got = ([torch.zeros(s, dtype=torch.float16, device=DEV) for s in shapes[3:]] for _ in range(2))
    ws = workspace(paro.paro_gated_workspace(d, True))

    def run(out):
        paro.paro_gated_grad(d, *[v.data_ptr() for v in t + out], ws.data_ptr(), ws.numel(), stream())
    run(ref)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(got)
    for size in (1.0, 3000.0, 2.0 ** -9, 1.0, 2000.0):
        t[0].copy_(torch.randn(n, hidden, generator=g) * size)
        t[2].copy_(torch.randn(n, hidden, generator=g) * min(size, 30.0))
        for o in got:
            o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        run(ref)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, got)) and all(bool(a.isfinite().all()) for a in ref)
