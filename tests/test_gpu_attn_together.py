"""The attention as programs use it: on another stream and in graphs, over arrays that pass 32 bits, one workspace for calls in turn, prompts and then tokens one by
one, and the example that trains a small model with every operator and the Update stage."""
import os
import sys

import pytest
import torch

from attn_ref import Case
from operators_ref import DEV, stream, workspace

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
KINDS = {"training, copies, bias": dict(lengths=[(200, 200), (77, 77)], hd=72, heads=4, kv=2, dtype="f16", window=60, sinks=3, buckets=7, pad=3),
         "training": dict(lengths=[(150, 150), (260, 260)], hd=64, heads=2, dtype="bf16"),
         "shared out": dict(lengths=[(900, 900)], hd=128, heads=2, kv=1, dtype="bf16", window=40, sinks=4),
         "new tokens, shared out": dict(lengths=[(2, 3000), (2, 4000)], hd=64, heads=4, kv=2, dtype="f16", buckets=16, far=100)}


def both_ways(case, backward):
    case.forward()
    outs = [case.out.whole, case.stats]
    if backward:
        case.backward()
        outs += [case.dq.whole, case.dk.whole, case.dv.whole] + ([case.dtable] if case.buckets else [])
    return outs


@pytest.mark.parametrize("kind", list(KINDS))
def test_in_a_graph_and_on_another_stream(paro, kind):
    c = Case(paro, **KINDS[kind])
    backward = kind != "new tokens, shared out"
    want = [t.clone() for t in both_ways(c, backward)]
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both_ways(c, backward)
    side.synchronize()
    assert all(bool(((a == b) | (a != a) & (b != b)).all()) for a, b in zip(want, got))
    d, room = c.plan(), max(16, paro.paro_attn_workspace(c.plan(), False), paro.paro_attn_workspace(c.plan(), True))
    ws = workspace(room)                                    # one for both: they follow each other
    fwd = [d, *(x.view.data_ptr() for x in (c.q, c.k, c.v)), *c.sequences(), c.out.view.data_ptr(), c.stats.data_ptr(), ws.data_ptr(), room]
    bwd = [d, c.dout.view.data_ptr(), *(x.view.data_ptr() for x in (c.q, c.k, c.v)), c.out.view.data_ptr(), c.stats.data_ptr(), *c.sequences(),
           *(x.view.data_ptr() for x in (c.dq, c.dk, c.dv)), c.address(c.dtable), ws.data_ptr(), room]
    with torch.cuda.graph(graph):
        paro.paro_attn(*fwd, stream())
        if backward:
            paro.paro_attn_grad(*bwd, stream())
    for i in range(3):                                      # other inputs, other garbage in the workspace, eager work in between
        c.q.view.mul_(0.8)
        c.dout.view.mul_(1.5)
        ws.fill_(0x11 * (i + 1))
        for t in got:
            t.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in got]
        for t in got:
            t.fill_(float(i))
        both_ways(c, backward)
        torch.cuda.synchronize()
        assert all(bool(((a == b) | (a != a) & (b != b)).all()) for a, b in zip(replayed, got)), i


def test_lengths_that_grow_between_replays(paro):
    """A captured step of a served batch: only the lengths on the device, and what the cache holds, change."""
    batch, room, heads, kv, hd = 3, 700, 4, 2, 64
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(batch * room, kv, hd, generator=g).half().to(DEV) for _ in range(2))
    q, out = torch.randn(batch, heads, hd, generator=g).half().to(DEV), torch.zeros(batch, heads, hd, dtype=torch.float16, device=DEV)
    lens = torch.zeros(batch, dtype=torch.int32, device=DEV)
    d = paro.make_attn(batch=batch, heads=heads, kv_heads=kv, head_dim=hd, len_q=1, len_k=room, dtype=paro.PARO_F16, window=90, sinks=2)
    ws = workspace(max(16, paro.paro_attn_workspace(d, False)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        paro.paro_attn(d, q.data_ptr(), k.data_ptr(), v.data_ptr(), 0, 0, lens.data_ptr(), 0, 0, out.data_ptr(), 0, ws.data_ptr(), ws.numel(), stream())
    for now in ([0, 1, 5], [1, 2, 6], [89, 90, 91], [92, 93, 700], [300, 699, 1]):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(now):
            seen = [j for j in range(n) if n - 1 - j < 90 or j < 2]
            kb, vb = (t.view(batch, room, kv, hd)[b, seen].double().cpu() for t in (k, v))
            for h in range(heads):
                p = torch.softmax(kb[:, h // 2] @ q[b, h].double().cpu() * hd ** -0.5, dim=0)
                want = p @ vb[:, h // 2] if seen else torch.zeros(hd, dtype=torch.float64)
                # fp16: a share and the result rounded, each by half a unit; fp32 sums of 64 and up to 92 terms
                assert bool(((out[b, h].double().cpu() - want).abs() <= 2.2 * 2.0 ** -11 * (p @ vb[:, h // 2].abs() if seen else want) + 2.0 ** -24).all()), (n, h)


def test_a_prompt_and_then_token_by_token(paro):
    """The rows of a whole sequence are those of the same tokens one by one over the cache, but for the roundings of shares (of other largest scores)."""
    n, heads, hd = 150, 3, 64
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(n, heads, hd, generator=g).half().to(DEV) for _ in range(3))
    whole, single = torch.empty_like(q), torch.empty_like(q)
    first = torch.tensor(paro.paro_rel_buckets(10, 50), dtype=torch.int32, device=DEV)
    table = torch.randn(10, heads, generator=g).to(DEV)
    common = dict(batch=1, heads=heads, head_dim=hd, dtype=paro.PARO_F16, window=40, sinks=1, buckets=10, table_dtype=paro.PARO_F32)
    paro.paro_attn(paro.make_attn(len_q=n, **common), q.data_ptr(), k.data_ptr(), v.data_ptr(), 0, 0, 0, table.data_ptr(), first.data_ptr(), whole.data_ptr(), 0, 0, 0,
                   stream())
    for i in range(n):
        d = paro.make_attn(len_q=1, len_k=i + 1, **common)
        ws = workspace(max(16, paro.paro_attn_workspace(d, False)))
        paro.paro_attn(d, q[i].data_ptr(), k.data_ptr(), v.data_ptr(), 0, 0, 0, table.data_ptr(), first.data_ptr(), single[i].data_ptr(), 0, ws.data_ptr(), ws.numel(),
                       stream())
    # each side: a share rounded (half a unit of a mean of |v|, which is below 4), the result rounded
    assert float((whole.double() - single.double()).abs().max()) <= 2 * (2.0 ** -11 * 4 + 2.0 ** -11 * 4)


@pytest.mark.parametrize("new", [1, 40])
def test_rows_past_32_bits(paro, new):
    """Keys, values and their gradients whose elements lie 2^31 and more from the first."""
    rows, ld, heads, hd, n = 70000, 1 << 15, 2, 64, 300
    k, v, dk, dv = (torch.empty(rows, ld, dtype=torch.bfloat16, device=DEV) for _ in range(4))
    g = torch.Generator().manual_seed(3)
    near_k, near_v = (torch.randn(n, heads * hd, generator=g).bfloat16().to(DEV) for _ in range(2))
    at, column = rows - n, ld - heads * hd
    k[at:, column:], v[at:, column:] = near_k, near_v
    assert (at * ld + column) > 2**31
    q = torch.randn(new, heads, hd, generator=g).bfloat16().to(DEV)
    starts = torch.tensor([at, rows], dtype=torch.int32, device=DEV)
    outs = []
    for kk, vv, gk, gv, start, step in ((k[:, column:], v[:, column:], dk[:, column:], dv[:, column:], starts, ld),
                                        (near_k, near_v, torch.empty_like(near_k), torch.empty_like(near_v), starts - at, heads * hd)):
        out, stats, dq = torch.empty_like(q), torch.empty(new, heads, 2, device=DEV), torch.empty_like(q)
        d = paro.make_attn(batch=1, heads=heads, head_dim=hd, len_q=new, len_k=n, rows_q=new, rows_k=rows if step == ld else n, ld_k=step, ld_v=step,
                           dtype=paro.PARO_BF16, window=100, sinks=5)
        ws = workspace(max(16, paro.paro_attn_workspace(d, True), paro.paro_attn_workspace(d, False)))
        paro.paro_attn(d, q.data_ptr(), kk.data_ptr(), vv.data_ptr(), 0, start.data_ptr(), 0, 0, 0, out.data_ptr(), stats.data_ptr(), ws.data_ptr(), ws.numel(), stream())
        paro.paro_attn_grad(d, q.data_ptr(), q.data_ptr(), kk.data_ptr(), vv.data_ptr(), out.data_ptr(), stats.data_ptr(), 0, start.data_ptr(), 0, 0, 0, dq.data_ptr(),
                            gk.data_ptr(), gv.data_ptr(), 0, ws.data_ptr(), ws.numel(), stream())
        outs.append([out, stats, dq, gk[at:, :heads * hd].clone() if step == ld else gk, gv[at:, :heads * hd].clone() if step == ld else gv])
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and bool(outs[0][3].isfinite().all())


@pytest.fixture(scope="module")
def example(paro):
    import attention_train
    return attention_train


@pytest.mark.parametrize("lengths,heads,kv,hd,window", [((40, 1, 33), 4, 2, 16, 12), ((129, 70), 2, 1, 24, 0)])
def test_the_examples_gradients_against_torch(example, lengths, heads, kv, hd, window):
    c = example.Shape(vocab=504, dim=40, hidden=72, heads=heads, kv_heads=kv, head_dim=hd, buckets=8, window=window, sinks=2 if window else 0, far=20)
    g = torch.Generator(device="cuda").manual_seed(5)
    T, k = 2.0, 9
    flat = example.random_parameters(c, g).to(torch.bfloat16)
    model, run = example.Model(flat, c), example.Pass(c, lengths, k, T)
    n = sum(lengths)
    tokens = torch.randint(0, c.vocab, (n,), generator=g, device="cuda")
    ids = torch.stack([torch.randperm(c.vocab, generator=g, device="cuda")[:k] for _ in range(n)])
    teacher = torch.randn(n, k, generator=g, device="cuda").to(torch.bfloat16)
    grads = example.Model(torch.full_like(flat, 7.0), c)
    loss = run.forward_backward(model, tokens, teacher, ids.int(), grads).clone()

    # in 32 bits on the host
    w = {name: getattr(model, name).float().cpu().requires_grad_() for name, *_ in c.parameters()}
    x = w["table"][tokens.cpu()] * c.dim ** 0.5
    q, kk, v = (x @ w["w_qkv"].t()).split([heads * hd, kv * hd, kv * hd], dim=1)
    rows, at = [], 0
    first = run.first.cpu()
    for size in lengths:
        far = torch.arange(size)[:, None] - torch.arange(size)
        seen = (far >= 0) & ((far < window) | (torch.arange(size) < c.sinks) if window else far >= 0)
        of = (first <= torch.arange(size)[:, None]).sum(1) - 1
        out = []
        for h in range(heads):
            a, b, d = q[at:at + size, h * hd:(h + 1) * hd], *(t[at:at + size, h // (heads // kv) * hd:(h // (heads // kv) + 1) * hd] for t in (kk, v))
            s = a @ b.t() * hd ** -0.5 + w["bias"][:, h][of][far.clamp(min=0)]
            out.append(torch.softmax(s.masked_fill(~seen, -torch.inf), 1) @ d)
        rows.append(torch.cat(out, 1))
        at += size
    z = x + torch.cat(rows) @ w["w_out"].t()
    y = z + (torch.nn.functional.silu(z @ w["w_gate"].t()) * (z @ w["w_up"].t())) @ w["w_down"].t()
    log_q = torch.log_softmax(y @ w["head"].t() / T, dim=1)
    log_p = torch.log_softmax(teacher.float().cpu() / T, dim=1)
    ref = (log_p.exp() * (log_p - log_q.gather(1, ids.cpu()))).sum(dim=1) * T * T
    ref.mean().backward()
    ref = ref.detach()
    # bf16 activations: each of the ten roundings on the way is 2^-9 of a value on average, 2^-8 at most
    assert float((loss.cpu() - ref).abs().max() / ref.abs().max()) < 10 * 2.0 ** -8
    for name, *_ in c.parameters():
        got, want = getattr(grads, name).float().cpu(), w[name].grad
        off = float((got - want).norm() / want.norm())
        assert off < 10 * 2.0 ** -8, (name, off)


def test_the_example_runs(example):
    losses = example.train(steps=4)
    assert len(losses) == 4 and all(x == x for x in losses)
    assert losses == example.train(steps=4), "another run gave other bits"
