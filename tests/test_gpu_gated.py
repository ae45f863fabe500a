"""The gated projections and their gradient against their definitions in 64 bits: every size from one up that begins, ends or splits a
tile, a stage or a piece, both tile shapes, split inner dimensions, rows apart and off alignment, both activations, both dtypes."""
import math

import pytest
import torch

from operators_ref import DEV, EPS32, HALF_ULP, TORCH, check, code, put, rng, rounding, rows, stream, workspace

pytestmark = pytest.mark.gpu


def act64(g, act):
    """Activation, slope, in 64 bits."""
    if act == "silu":
        y = torch.sigmoid(g)
        return g * y, y * (1 + g * (1 - y))
    y = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
    return g * y, y + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def plan(paro, n, dim, hidden, dtype, act, pad):
    return paro.make_gated(n=n, dim=dim, hidden=hidden, dtype=code(paro, dtype), act=paro.PARO_SILU if act == "silu" else paro.PARO_GELU,
                           ld_x=dim + pad, ld_h=hidden + pad)


def weights(g, hidden, dim, dtype):
    return put(torch.randn(hidden, dim, generator=g) * (1.3 / math.sqrt(dim)), 0, dtype)


def untouched(whole, views):
    for v in views:
        v.fill_(5.0)
    assert bool((whole == 5.0).all()), "wrote between the rows"


def forward(paro, n, dim, hidden, dtype="bf16", act="silu", pad=0, seed=1, save=True):
    g = rng(seed)
    x, x64 = put(torch.randn(n, dim, generator=g), pad, dtype)
    (wg, wg64), (wu, wu64) = weights(g, hidden, dim, dtype), weights(g, hidden, dim, dtype)
    outs = [rows(n, hidden, pad, dtype, fill=5.0) for _ in range(3)]
    h, gate, up = (v for _, v in outs)
    d = plan(paro, n, dim, hidden, dtype, act, pad)
    ws = workspace(paro.paro_gated_workspace(d, False))
    paro.paro_gated(d, x.data_ptr(), wg.data_ptr(), wu.data_ptr(), h.data_ptr(), gate.data_ptr() if save else 0, up.data_ptr() if save else 0,
                    ws.data_ptr(), ws.numel(), stream())
    g64, u64 = x64 @ wg64.t(), x64 @ wu64.t()
    # an fp32 sum of dim exact products, in any order, and what each addition of the matrix cores may drop
    eg, eu = (2 * (dim + 4) * EPS32 * (x64.abs() @ w.abs().t()) for w in (wg64, wu64))
    a64, slope = act64(g64, act)
    # slopes are below 1.2 in size; the activation in fp32: a few roundings of its result and of its argument
    ea = 1.2 * eg + 8 * EPS32 * (a64.abs() + g64.abs())
    eh = ea * (u64.abs() + eu) + a64.abs() * eu + EPS32 * (a64 * u64).abs()
    check(h, a64 * u64, rounding(a64 * u64, dtype, eh), "h")
    if save:
        check(gate, g64, rounding(g64, dtype, eg), "gate")
        check(up, u64, rounding(u64, dtype, eu), "up")
    for whole, view in outs:
        untouched(whole, [view])


def backward(paro, n, dim, hidden, dtype="bf16", act="silu", pad=0, seed=1):
    g = rng(seed)
    x, x64 = put(torch.randn(n, dim, generator=g), pad, dtype)
    (wg, wg64), (wu, wu64) = weights(g, hidden, dim, dtype), weights(g, hidden, dim, dtype)
    (gate, g64), (up, u64) = (put(torch.randn(n, hidden, generator=g) * 1.3, pad, dtype) for _ in range(2))
    dh, dh64 = put(torch.randn(n, hidden, generator=g) * 0.3, pad, dtype)
    whole, dx = rows(n, dim, pad, dtype, fill=5.0)
    dwg, dwu = (torch.full((hidden, dim), 7.0, dtype=TORCH[dtype], device=DEV) for _ in range(2))
    d = plan(paro, n, dim, hidden, dtype, act, pad)
    ws = workspace(paro.paro_gated_workspace(d, True))
    call = [d, dh.data_ptr(), gate.data_ptr(), up.data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), dx.data_ptr(), dwg.data_ptr(), dwu.data_ptr(),
            ws.data_ptr(), ws.numel(), stream()]
    paro.paro_gated_grad(*call)
    a64, slope = act64(g64, act)
    dg64, du64 = dh64 * u64 * slope, dh64 * a64
    # dg and du in fp32 (a few roundings), then rounded to the dtype
    edg, edu = (rounding(v, dtype, 16 * EPS32 * size) for v, size in ((dg64, (dh64 * u64).abs() * (1 + g64.abs())), (du64, (dh64 * g64).abs())))
    size = dg64.abs() @ wg64.abs() + du64.abs() @ wu64.abs()
    dx64, edx = dg64 @ wg64 + du64 @ wu64, edg @ wg64.abs() + edu @ wu64.abs()
    check(dx, dx64, rounding(dx64, dtype, edx + 2 * (2 * hidden + 4) * EPS32 * (size + edx)), "dx")
    for got, v, e, what in ((dwg, dg64, edg, "dwg"), (dwu, du64, edu, "dwu")):
        ref, err = v.t() @ x64, e.t() @ x64.abs()
        check(got, ref, rounding(ref, dtype, err + 2 * (n + 4) * EPS32 * (v.abs().t() @ x64.abs() + err)), what)
    bits = [t.clone() for t in (dx, dwg, dwu)]
    ws.fill_(0x3C)
    paro.paro_gated_grad(*call)
    assert all(torch.equal(a, b) for a, b in zip(bits, (dx, dwg, dwu))), "the same call gave other bits"
    untouched(whole, [dx])


SIZES = [1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 200]


@pytest.mark.parametrize("n", SIZES)
def test_forward_of_any_count(paro, n):
    forward(paro, n, 72, 40, pad=0)
    forward(paro, n, 136, 264, dtype="f16", act="gelu", pad=8)


@pytest.mark.parametrize("dim", SIZES + [320, 1601])
def test_forward_of_any_width(paro, dim):
    forward(paro, 37, dim, 72, pad=dim % 4)
    forward(paro, 5, dim, 33, dtype="f16", pad=8, act="gelu")


@pytest.mark.parametrize("hidden", SIZES + [257, 520])
def test_forward_of_any_hidden_width(paro, hidden):
    forward(paro, 70, 64, hidden, act="gelu")
    forward(paro, 3, 96, hidden, dtype="f16", pad=1, save=False)


@pytest.mark.parametrize("n", SIZES)
def test_backward_of_any_count(paro, n):
    backward(paro, n, 72, 40)
    backward(paro, n, 24, 136, dtype="f16", act="gelu", pad=8)


@pytest.mark.parametrize("dim", SIZES + [320])
def test_backward_of_any_width(paro, dim):
    backward(paro, 37, dim, 72, pad=dim % 4, act="gelu")


@pytest.mark.parametrize("hidden", SIZES + [257, 520])
def test_backward_of_any_hidden_width(paro, hidden):
    backward(paro, 70, 64, hidden, dtype="f16")
    backward(paro, 33, 40, hidden, pad=3)


# tiles of 256 x 256 of each product, with and without a remainder; splits of the inner dimension
@pytest.mark.parametrize("n,dim,hidden,dtype,act,pad", [(2304, 264, 2056, "bf16", "silu", 0), (4104, 2060, 600, "f16", "gelu", 8), (333, 2049, 2313, "bf16", "gelu", 5),
                                                       (40, 2048, 5000, "bf16", "silu", 0), (300, 5128, 136, "f16", "silu", 0), (2048, 2048, 2048, "bf16", "silu", 0)])
def test_large(paro, n, dim, hidden, dtype, act, pad):
    forward(paro, n, dim, hidden, dtype, act, pad)
    backward(paro, n, dim, hidden, dtype, act, pad)


@pytest.mark.parametrize("n,dim,hidden", [(1, 4096, 11008), (3, 4096, 1000), (16, 2048, 4096), (17, 1111, 3333), (32, 768, 2048)])
def test_few_tokens(paro, n, dim, hidden):
    forward(paro, n, dim, hidden, save=n > 1)
    forward(paro, n, dim + 3, hidden + 1, dtype="f16", act="gelu", pad=1)


def test_no_tokens(paro):
    d = plan(paro, 0, 24, 40, "bf16", "silu", 0)
    dw = torch.full((2, 40, 24), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = workspace(paro.paro_gated_workspace(d, True))
    w = torch.zeros(40, 24, dtype=torch.bfloat16, device=DEV)
    paro.paro_gated(d, 0, w.data_ptr(), w.data_ptr(), 0, 0, 0, ws.data_ptr(), ws.numel(), stream())
    paro.paro_gated_grad(d, 0, 0, 0, 0, w.data_ptr(), w.data_ptr(), 0, dw[0].data_ptr(), dw[1].data_ptr(), ws.data_ptr(), ws.numel(), stream())
    assert bool((dw == 0).all())


@pytest.mark.parametrize("n,dim,hidden", [(2, 64, 64), (40, 72, 136), (300, 264, 520)])
def test_nan_stays_in_its_row(paro, n, dim, hidden):
    """A token with NaN spoils its own rows of h and dx; a weight's, its own column of h: no tile's edge reads a neighbour into a result."""
    g = rng(4)
    x = torch.randn(n, dim, generator=g).to(DEV, torch.bfloat16)
    wg, wu = (torch.randn(hidden, dim, generator=g).to(DEV, torch.bfloat16) for _ in range(2))
    x[n // 2, dim // 3] = float("nan")
    wu[hidden // 2, dim // 2] = float("inf")
    h = torch.empty(n, hidden, dtype=torch.bfloat16, device=DEV)
    d = plan(paro, n, dim, hidden, "bf16", "silu", 0)
    ws = workspace(paro.paro_gated_workspace(d, True))
    paro.paro_gated(d, x.data_ptr(), wg.data_ptr(), wu.data_ptr(), h.data_ptr(), 0, 0, ws.data_ptr(), ws.numel(), stream())
    spoilt = ~h.isfinite()
    expect = torch.zeros_like(spoilt)
    expect[n // 2], expect[:, hidden // 2] = True, True
    assert torch.equal(spoilt, expect)
    gate, up, dh = (torch.randn(n, hidden, generator=g).to(DEV, torch.bfloat16) for _ in range(3))
    dh[n // 2, 3] = float("nan")
    wu[hidden // 2, dim // 2] = 0.5
    x[n // 2, dim // 3] = 0.5
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    paro.paro_gated_grad(d, dh.data_ptr(), gate.data_ptr(), up.data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), dx.data_ptr(), dwg.data_ptr(),
                         dwu.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    for t, row in ((dx, n // 2), (dwg, 3), (dwu, 3)):
        assert bool(t[row].isnan().all()) and int(t.isnan().any(dim=1).sum()) == 1


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_against_differences_of_the_forward_pass(paro, act):
    """Central differences of sum(h * dh), with h from the library, along random directions of x, Wg and Wu: in fp16, the step such that the
    moved inputs are exact and the difference of h is far above its rounding."""
    n, dim, hidden, g = 6, 32, 48, rng(9)
    grid = lambda *s: torch.randint(-8, 9, s, generator=g).float() / 16       # noqa: E731 - multiples of 1/16
    x, wg, wu = grid(n, dim), grid(hidden, dim), grid(hidden, dim)
    dh = torch.randint(-2, 3, (n, hidden), generator=g).float()
    d = plan(paro, n, dim, hidden, "f16", act, 0)
    ws = workspace(paro.paro_gated_workspace(d, True))

    def run(x, wg, wu):
        t = [v.to(DEV, torch.float16) for v in (x, wg, wu)]
        out = [torch.empty(n, hidden, dtype=torch.float16, device=DEV) for _ in range(3)]
        paro.paro_gated(d, *[v.data_ptr() for v in t + out], ws.data_ptr(), ws.numel(), stream())
        return out
    _, gate, up = run(x, wg, wu)
    dev = [v.to(DEV, torch.float16) for v in (dh, x, wg, wu)]
    grads = [torch.empty_like(v) for v in dev[1:]]
    paro.paro_gated_grad(d, dev[0].data_ptr(), gate.data_ptr(), up.data_ptr(), *[v.data_ptr() for v in dev[1:] + grads], ws.data_ptr(), ws.numel(), stream())
    step = 1 / 16
    for k in range(3):
        way = torch.randint(-1, 2, (x, wg, wu)[k].shape, generator=g).float()
        there = [v + step * way if i == k else v for i, v in enumerate((x, wg, wu))]
        back = [v - step * way if i == k else v for i, v in enumerate((x, wg, wu))]
        hi, lo = (run(*v)[0].cpu().double() for v in (there, back))
        slope = float(((hi - lo) * dh.double()).sum()) / (2 * step)
        got = float((grads[k].cpu().double() * way.double()).sum())
        # the same difference in 64 bits says what the finite step itself is off by
        h64 = [act64(a.double() @ b.double().t(), act)[0] * (a.double() @ c.double().t()) for a, b, c in (there, back)]
        exact_slope = float(((h64[0] - h64[1]) * dh.double()).sum()) / (2 * step)
        g64, u64 = x.double() @ wg.double().t(), x.double() @ wu.double().t()
        a64, da64 = act64(g64, act)
        dg, du = dh.double() * u64 * da64, dh.double() * a64
        true = ((dg @ wg.double() + du @ wu.double()), dg.t() @ x.double(), du.t() @ x.double())[k]
        off = abs(exact_slope - float((true * way.double()).sum()))
        u = HALF_ULP["f16"]
        err = float((u * (h64[0].abs() + h64[1].abs()) * 1.01 * dh.double().abs()).sum()) / (2 * step)
        terms = (dg.abs() @ wg.double().abs() + du.abs() @ wu.double().abs(), dg.abs().t() @ x.double().abs(), du.abs().t() @ x.double().abs())[k]
        # the stored projections, dg and du, and the gradient are rounded once each; slopes change by at most 1.2 of the gate's rounding
        moved = (dh.double().abs() * u64.abs() * 1.2 * u * g64.abs(), dh.double().abs() * 1.2 * u * g64.abs())
        extra = (moved[0] @ wg.double().abs() + moved[1] @ wu.double().abs(), moved[0].t() @ x.double().abs(), moved[1].t() @ x.double().abs())[k]
        err += float(((3.1 * u * terms + extra + u * true.abs()) * way.double().abs()).sum())
        assert abs(got - slope) <= off + err, (k, got, slope, off, err)


def test_in_a_graph_and_on_another_stream(paro):
    n, dim, hidden, g = 150, 104, 200, rng(2)
    d = plan(paro, n, dim, hidden, "bf16", "silu", 0)
    x, wg, wu, dh = (torch.randn(*s, generator=g).to(DEV, torch.bfloat16) for s in ((n, dim), (hidden, dim), (hidden, dim), (n, hidden)))
    sizes = [(n, hidden)] * 3 + [(n, dim), (hidden, dim), (hidden, dim)]
    ref, got = ([torch.zeros(*s, dtype=torch.bfloat16, device=DEV) for s in sizes] for _ in range(2))
    ws = workspace(max(paro.paro_gated_workspace(d, k) for k in (False, True)))

    def both(o):
        paro.paro_gated(d, x.data_ptr(), wg.data_ptr(), wu.data_ptr(), *[t.data_ptr() for t in o[:3]], ws.data_ptr(), ws.numel(), stream())
        paro.paro_gated_grad(d, dh.data_ptr(), o[1].data_ptr(), o[2].data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(),
                             *[t.data_ptr() for t in o[3:]], ws.data_ptr(), ws.numel(), stream())
    both(ref)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        both(got)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    with torch.cuda.graph(graph):
        both(got)
    for i in range(3):
        x.copy_(torch.randn(n, dim, generator=g))
        for t in got:
            t.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        both(ref)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


@pytest.mark.parametrize("n,dim,hidden,dtype,act,pad", [(474, 384, 896, "bf16", "silu", 8), (1000, 768, 2999, "bf16", "gelu", 0), (4544, 640, 640, "bf16", "silu", 0),
                                                        (321, 81, 865, "f16", "gelu", 3), (1861, 2176, 128, "bf16", "silu", 0), (293, 121, 5000, "f16", "silu", 0),
                                                        (4000, 512, 1024, "f16", "gelu", 0), (129, 130, 131, "bf16", "silu", 0)])
def test_backward_of_middling_sizes(paro, n, dim, hidden, dtype, act, pad):
    backward(paro, n, dim, hidden, dtype, act, pad=pad)
