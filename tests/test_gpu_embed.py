"""Embedding lookup and its gradient against their definitions in 64 bits: widths below, at and off the vector width, token counts from
none to long runs that are summed in parts, tokens that the table does not hold, rows apart, every dtype."""
import pytest
import torch

from operators_ref import DEV, EPS32, TORCH, check, code, put, rng, rounding, rows, stream, workspace

pytestmark = pytest.mark.gpu
TOKEN = {torch.int32: "PARO_I32", torch.int64: "PARO_I64"}


def lookup(paro, n, dim, v, dtype, token, first=0, pad=0, scale=1.7, seed=1):
    g = rng(seed)
    table, wide = put(torch.randn(v, dim, generator=g), 0, dtype)
    tokens = torch.randint(first - 2, first + v + 2, (n,), generator=g).to(token)
    whole, out = rows(n, dim, pad, dtype, fill=7.0)
    dev = tokens.to(DEV)
    paro.paro_embed(table.data_ptr(), code(paro, dtype), v, dim, dev.data_ptr(), getattr(paro, TOKEN[token]), n, first, scale,
                    out.data_ptr(), dim + pad, stream())
    at = tokens.long() - first
    held = (at >= 0) & (at < v)
    ref = torch.where(held[:, None], wide[at.clamp(0, v - 1)] * scale, 0.0)
    check(out, ref, rounding(ref, dtype, EPS32 * 2 * ref.abs()), "lookup")     # scale in fp32, one product
    out.fill_(7.0)
    assert bool((whole == 7.0).all()), "wrote between the rows"


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [1, 3, 4, 7, 8, 9, 63, 768, 1601, 2048, 2056, 4099])
def test_lookup_of_any_width(paro, dim, dtype):
    lookup(paro, 37, dim, 50, dtype, torch.int64, pad=dim % 3)


@pytest.mark.parametrize("n,v,first,token", [(1, 1, 0, torch.int64), (2, 50257, 0, torch.int32), (5000, 11, 100, torch.int64), (300, 1000, -5, torch.int32)])
def test_lookup_of_any_count(paro, n, v, first, token):
    lookup(paro, n, 96, v, "bf16", token, first=first, pad=8)


def gradient(paro, tokens, dim, v, dtype, grad_dtype, first=0, pad=0, scale=0.6, seed=2):
    g, n = rng(seed), tokens.numel()
    dout, wide = put(torch.randn(n, dim, generator=g), pad, dtype) if n else (torch.empty(1, dim, device=DEV), torch.empty(0, dim).double())
    whole, grad = rows(v, dim, 0, grad_dtype)
    ws = workspace(paro.paro_embed_grad_workspace(n, v, dim))
    dev = tokens.to(DEV)
    call = [dout.data_ptr(), code(paro, dtype), dim + pad, dev.data_ptr(), getattr(paro, TOKEN[tokens.dtype]), n, first, scale, grad.data_ptr(),
            code(paro, grad_dtype), v, dim, ws.data_ptr(), ws.numel(), stream()]
    paro.paro_embed_grad(*call)
    at = tokens.long() - first
    held = (at >= 0) & (at < v)
    ref = torch.zeros(v, dim, dtype=torch.float64).index_add_(0, at[held], wide[held])
    size = torch.zeros(v, dim, dtype=torch.float64).index_add_(0, at[held], wide[held].abs())
    count = torch.bincount(at[held], minlength=v)[:, None].double()
    err = scale * EPS32 * (count + 2) * size               # count - 1 additions, whatever their order; the scale; one product
    check(grad, ref * scale, rounding(ref * scale, grad_dtype, err), "gradient")
    assert bool(whole[v * dim:].isnan().all()), "wrote past the gradient"
    first_bits = grad.clone()
    grad.fill_(3.0)
    ws.fill_(0x11)
    paro.paro_embed_grad(*call)
    assert torch.equal(grad, first_bits), "the same call gave other bits"


@pytest.mark.parametrize("dtype,grad_dtype", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("dim", [1, 5, 7, 8, 9, 64, 769, 1024, 2050])
def test_gradient_of_any_width(paro, dim, dtype, grad_dtype):
    tokens = torch.randint(-3, 60, (331,), generator=rng(dim))
    gradient(paro, tokens, dim, 57, dtype, grad_dtype, pad=dim % 2)


@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 1023, 1024, 1025, 4097, 20011])
@pytest.mark.parametrize("v", [1, 511, 512, 513, 2000])
def test_gradient_of_any_count(paro, n, v):
    u = torch.rand(n, generator=rng(n + v), dtype=torch.float64)
    tokens = (torch.exp(u * torch.log(torch.tensor(v + 4.0, dtype=torch.float64))) - 2).long()     # a few tokens have most of the places
    gradient(paro, tokens, 72, v, "bf16", "f32")


@pytest.mark.parametrize("where", ["front", "back", "one", "alternating", "none"])
def test_gradient_of_long_runs(paro, where):
    """Runs that begin and end inside the parts that are summed on their own, on either side of their length."""
    n, v = 4096, 9
    i = torch.arange(n)
    tokens = {"front": torch.where(i < 2111, 0, 1 + i % 8), "back": torch.where(i < 1999, i % 8, 8), "one": torch.full((n,), 4),
              "alternating": i // 65 % 9, "none": torch.full((n,), 9)}[where]
    for order in (i, torch.randperm(n, generator=rng(8))):
        gradient(paro, tokens[order].int(), 136, v, "f32", "f32", first=0)


def test_gradient_of_a_part_of_the_vocabulary(paro):
    tokens = torch.randint(0, 4000, (3000,), generator=rng(5))
    gradient(paro, tokens, 40, 1000, "f16", "f32", first=1500, pad=3)


def test_infinities_and_nan_stay_in_their_rows(paro):
    n, v, dim = 300, 20, 24
    tokens = torch.randint(0, v - 1, (n,), generator=rng(6))
    tokens[7], tokens[9] = v + 3, -1                        # masked tokens carry NaN
    tokens[100], tokens[200] = v - 1, v - 1
    x = torch.randn(n, dim, generator=rng(7))
    x[7], x[9] = float("nan"), float("inf")
    x[100, 3], x[200, 5] = float("inf"), float("nan")
    dout, _ = put(x, 0, "bf16")
    grad, ws, dev = torch.empty(v, dim, device=DEV), workspace(paro.paro_embed_grad_workspace(n, v, dim)), tokens.to(DEV)
    paro.paro_embed_grad(dout.data_ptr(), paro.PARO_BF16, 0, dev.data_ptr(), paro.PARO_I64, n, 0, 1.0, grad.data_ptr(), paro.PARO_F32, v, dim,
                         ws.data_ptr(), ws.numel(), stream())
    assert bool(grad[:-1].isfinite().all()) and bool(grad[-1, 3].isinf()) and bool(grad[-1, 5].isnan()) and int((~grad[-1].isfinite()).sum()) == 2


def test_gradient_against_differences_of_the_lookup(paro):
    """The gradient is the lookup's transpose: <lookup(table), dout> = <table, gradient(dout)>, here exactly (small whole numbers)."""
    g, n, v, dim = rng(11), 500, 40, 33
    table = torch.randint(-8, 9, (v, dim), generator=g).to(DEV, torch.float32)
    dout = torch.randint(-8, 9, (n, dim), generator=g).to(DEV, torch.float32)
    tokens = torch.randint(-4, v + 4, (n,), generator=g).to(DEV)
    out, grad = torch.empty(n, dim, device=DEV), torch.empty(v, dim, device=DEV)
    ws = workspace(paro.paro_embed_grad_workspace(n, v, dim))
    paro.paro_embed(table.data_ptr(), paro.PARO_F32, v, dim, tokens.data_ptr(), paro.PARO_I64, n, 0, 0.5, out.data_ptr(), 0, stream())
    paro.paro_embed_grad(dout.data_ptr(), paro.PARO_F32, 0, tokens.data_ptr(), paro.PARO_I64, n, 0, 0.5, grad.data_ptr(), paro.PARO_F32, v, dim,
                         ws.data_ptr(), ws.numel(), stream())
    assert float((out.double() * dout).sum()) == float((table.double() * grad).sum())


def test_on_another_stream_and_in_a_graph(paro):
    n, v, dim = 700, 130, 256
    tokens = torch.randint(0, v, (n,), generator=rng(3)).to(DEV)
    dout = torch.randn(n, dim, generator=rng(4)).to(DEV, torch.bfloat16)
    ws = workspace(paro.paro_embed_grad_workspace(n, v, dim))

    def grad_into(t):
        paro.paro_embed_grad(dout.data_ptr(), paro.PARO_BF16, 0, tokens.data_ptr(), paro.PARO_I64, n, 0, 1.0, t.data_ptr(), paro.PARO_BF16, v, dim,
                             ws.data_ptr(), ws.numel(), stream())
    ref, got = (torch.full((v, dim), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    grad_into(ref)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        grad_into(got)
    side.synchronize()
    assert torch.equal(ref, got)
    with torch.cuda.graph(graph):
        grad_into(got)
    for k in range(3):
        got.fill_(float(k))
        tokens.copy_(torch.randint(0, v, (n,), generator=rng(20 + k)))
        graph.replay()
        torch.cuda.synchronize()
        grad_into(ref)
        torch.cuda.synchronize()
        assert torch.equal(ref, got)


@pytest.mark.parametrize("dtype", ["f32"])
def test_offsets_beyond_32_bits(paro, dtype):
    """The last rows of a table, of activations and of a gradient whose bytes no 32-bit number counts."""
    v, dim = 300_007, 4096
    table = torch.zeros(v, dim, dtype=TORCH[dtype], device=DEV)
    table[-1] = 2.0
    tokens = torch.full((v,), v - 2, dtype=torch.int32, device=DEV)
    tokens[-1] = v - 1
    out = torch.full((v, dim), 9.0, dtype=TORCH[dtype], device=DEV)
    paro.paro_embed(table.data_ptr(), code(paro, dtype), v, dim, tokens.data_ptr(), paro.PARO_I32, v, 0, 3.0, out.data_ptr(), 0, stream())
    assert bool((out[-1] == 6.0).all()) and bool((out[-2] == 0.0).all()) and float(out.sum()) == 6.0 * dim
    ws = workspace(paro.paro_embed_grad_workspace(v, v, dim))
    paro.paro_embed_grad(out.data_ptr(), code(paro, dtype), 0, tokens.data_ptr(), paro.PARO_I32, v, 0, 0.5, table.data_ptr(), code(paro, dtype), v, dim,
                         ws.data_ptr(), ws.numel(), stream())
    assert bool((table[-1] == 3.0).all()) and float(table.sum()) == 3.0 * dim


@pytest.mark.parametrize("grad_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 7, 31, 64, 77])
@pytest.mark.parametrize("v,dim", [(1, 8), (2, 9), (700, 8), (300, 33), (513, 100), (40, 1031), (9, 5003)])
def test_rows_without_a_token_are_zeros_wherever_the_table_lies(paro, v, dim, offset, grad_dtype):
    """A gradient that begins at any element, few tokens or none: zeros in all other rows, nothing before and nothing behind."""
    for tokens in (torch.tensor([v // 2, v - 1, v // 2]), torch.tensor([v]), torch.arange(0, v, 2)):
        n, guard = tokens.numel(), 200
        whole = torch.full((guard + offset + v * dim + guard,), 9.0, dtype=TORCH[grad_dtype], device=DEV)
        grad = whole[guard - guard % 8 + offset:][:v * dim].view(v, dim)
        dout = torch.randn(n, dim, generator=rng(v)).to(torch.bfloat16)
        ws, dev, dout_dev = workspace(paro.paro_embed_grad_workspace(n, v, dim)), tokens.to(DEV), dout.to(DEV)
        paro.paro_embed_grad(dout_dev.data_ptr(), paro.PARO_BF16, dim, dev.data_ptr(), paro.PARO_I64, n, 0, 1.0, grad.data_ptr(),
                             code(paro, grad_dtype), v, dim, ws.data_ptr(), ws.numel(), stream())
        held = tokens < v
        ref = torch.zeros(v, dim, dtype=torch.float64).index_add_(0, tokens[held], dout[held].double())
        check(grad, ref, rounding(ref, grad_dtype, 4 * EPS32 * ref.abs() + 8 * EPS32), "gradient")     # at most two summands of size below 8
        assert bool((grad[ref.to(DEV).abs().sum(dim=1) == 0] == 0).all()), "a row without a token is not zeros"
        grad.fill_(9.0)
        assert bool((whole == 9.0).all()), "wrote beside the gradient"


@pytest.mark.parametrize("token", [torch.int32, torch.int64])
@pytest.mark.parametrize("dtype,grad_dtype", [("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("n,dim,v", [(1, 5000, 3), (7, 8, 1000), (32, 100, 31), (33, 2049, 9), (63, 4100, 40), (64, 64, 3000), (64, 1030, 1), (65, 1030, 1)])
def test_gradient_of_few_tokens(paro, n, dim, v, dtype, grad_dtype, token):
    tokens = torch.randint(-2, v + 2, (n,), generator=rng(n * dim)).to(token)
    gradient(paro, tokens + 11, dim, v, dtype, grad_dtype, first=11, pad=n % 3)


def test_as_many_tokens_as_the_call_takes(paro):
    """2^31 - 1 tokens: places among them, and 64 or a segment of 2^20 beyond, count in more than 32 bits.  One row's run ends in the last
    segment, the other's is the last 100 tokens; small whole numbers here and there make the sums exact."""
    n, dim, v = 2 ** 31 - 1, 8, 3
    tokens = torch.zeros(n, dtype=torch.int32, device=DEV)
    tokens[-100:] = 2
    dout = torch.zeros(n, dim, dtype=torch.bfloat16, device=DEV)
    ref = torch.zeros(v, dim)
    seg = 2 ** 20
    for i in (0, 5, seg - 1, seg, 700 * seg + 3, 2047 * seg - 1, 2047 * seg, 2047 * seg + 77, n - 101, n - 100, n - 64, n - 63, n - 37, n - 36, n - 1):
        dout[i, i % dim] = 1 + i % 5
        ref[2 if i >= n - 100 else 0, i % dim] += 1 + i % 5
    grad = torch.full((v, dim), 7.0, device=DEV)
    ws = workspace(paro.paro_embed_grad_workspace(n, v, dim))
    paro.paro_embed_grad(dout.data_ptr(), paro.PARO_BF16, 0, tokens.data_ptr(), paro.PARO_I32, n, 0, 1.0, grad.data_ptr(), paro.PARO_F32, v, dim,
                         ws.data_ptr(), ws.numel(), stream())
    assert torch.equal(grad.cpu(), ref)
