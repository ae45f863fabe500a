"""The distillation loss and its gradient against their definitions in 64 bits: vocabularies on both sides of every kernel's limit and off the
vector width, one to all entries, repeated and masked ones, rows that hold none, infinities, the lowest numbers, in place, every dtype."""
import math

import pytest
import torch

from operators_ref import DEV, TORCH, check, code, put, rng, rounding, rows, stream

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -20        # relative error of a softmax entry whose exponent is of order one: a few fp32 roundings and the exponential's


def reference(z, t, ids, T, w):
    """loss, lse, dz in 64 bits and the bounds of their fp32 errors: an exponent x carries |x| roundings."""
    n, v = z.shape
    held = (ids >= 0) & (ids < v) & (t != -math.inf)
    some = held.any(dim=1)
    x = torch.where(held, t / T, -math.inf)
    log_p = torch.where(held, x - torch.logsumexp(x, dim=1, keepdim=True), -math.inf)
    p = log_p.exp()
    lse = torch.logsumexp(z / T, dim=1)
    at = ids.clamp(0, v - 1).long()
    log_q = torch.where(z == -math.inf, -math.inf, z / T - lse[:, None])
    terms = torch.where(p > 0, p * (log_p - log_q.gather(1, at)), 0.0)
    loss = torch.where(some, T * T * terms.sum(dim=1), 0.0)
    most = torch.where(z.amax(dim=1) == -math.inf, 0.0, z.amax(dim=1))
    size = torch.where(held & (p > 0), p * (log_p.abs() + ((z.gather(1, at) - most[:, None]) / T).abs()), 0.0).sum(dim=1) + 2 + (lse - most / T).abs()
    P = torch.zeros(n, v, dtype=torch.float64).scatter_add_(1, at, torch.where(held, p, 0.0))
    q = torch.where(log_q == -math.inf, 0.0, log_q.exp())
    dz = torch.where(some[:, None], T * w[:, None] * (q - P), 0.0)
    spread = 1 + torch.where(log_q.isfinite(), log_q.abs(), 0.0) / 2
    qw = T * w.abs()[:, None] * q
    err = TINY * (qw * spread + T * w.abs()[:, None] * 2 * P * (1 + torch.where(held & (p > 0), log_p.abs(), 0.0).amax(dim=1, keepdim=True) / 2)) + 2.0 ** -120
    lse_err = torch.where(lse.isfinite(), TINY * (2 + lse.abs()), 0.0)
    return loss, torch.where(some, lse, 0.0), dz, TINY * T * T * size, lse_err, err, err + qw * lse_err[:, None]


def run_all(paro, z, t, ids, T, dtype, teacher, pad=0, w=None, in_place=True):
    n, v = z.shape
    k = t.shape[1]
    zd, z64 = put(z, pad, dtype)
    td, t64 = t.to(TORCH[teacher]).to(DEV), t.to(TORCH[teacher]).double()
    idd = ids.int().to(DEV)
    w = torch.rand(n, generator=rng(n + v)) + 0.5 if w is None else w
    wd = w.float().to(DEV)
    d = paro.make_distill(n=n, vocab=v, k=k, temperature=T, dtype=code(paro, dtype), teacher_dtype=code(paro, teacher), ld_logits=v + pad,
                          ld_dlogits=v + pad)
    T32 = float(torch.tensor(T, dtype=torch.float32))
    loss64, lse64, dz64, loss_err, lse_err, dz_err, dz_err_of_lse = reference(z64, t64, ids, T32, w.float().double())
    args = zd.data_ptr(), td.data_ptr(), idd.data_ptr()
    loss, lse = (torch.full((n,), 77.0, device=DEV) for _ in range(2))
    paro.paro_distill_loss(d, *args, loss.data_ptr(), lse.data_ptr(), stream())
    check(loss, loss64, loss_err, "loss")
    check(lse, lse64, lse_err, "lse")
    for what in ("step", "grad") + (("in place",) if in_place else ()):
        whole, dz = rows(n, v, pad, dtype, fill=5.0)
        if what == "grad":
            paro.paro_distill_grad(d, *args, lse.data_ptr(), wd.data_ptr(), dz.data_ptr(), stream())
            err = dz_err_of_lse
        else:
            again = torch.full((n,), 77.0, device=DEV)
            target = zd if what == "in place" else dz
            paro.paro_distill_step(d, *args, wd.data_ptr(), again.data_ptr(), target.data_ptr(), stream())
            assert torch.equal(again, loss) or bool(again.isnan().any()), "loss of the step differs"
            err = dz_err
            if what == "in place":
                dz.copy_(zd)
        check(dz, dz64, rounding(dz64, dtype, err), what)
        dz.fill_(5.0)
        assert bool((whole == 5.0).all()), "wrote between the rows"


def some_inputs(n, v, k, seed, masked=True):
    g = rng(seed)
    z = torch.randn(n, v, generator=g) * 2
    t = torch.randn(n, k, generator=g) * 2
    ids = torch.randint(-1 if masked else 0, v + (1 if masked else 0), (n, k), generator=g)       # repeated, and some masked
    z.scatter_add_(1, ids.clamp(0, v - 1), t + 4)
    if masked and n > 2:
        ids[n // 2] = -1
    return z, t, ids


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("v", [1, 2, 3, 7, 8, 9, 1000, 4095, 4096, 4100, 8192, 8193, 16389, 32007])
def test_vocabularies(paro, v, dtype):
    z, t, ids = some_inputs(5, v, min(v, 11), v)
    run_all(paro, z, t, ids, 2.0, dtype, "f32", pad=v % 5)


@pytest.mark.parametrize("v,dtype", [(32768, "f32"), (32773, "f32"), (65536, "f32"), (65541, "f32"), (65536, "bf16"), (65544, "f16"), (131072, "bf16"),
                                     (131081, "bf16"), (200003, "f16")])
def test_large_vocabularies(paro, v, dtype):
    z, t, ids = some_inputs(3, v, 33, v)
    run_all(paro, z, t, ids, 1.5, dtype, "bf16", pad=3)


@pytest.mark.parametrize("k", [1, 2, 63, 64, 255, 256, 257, 512, 1023, 1024])
@pytest.mark.parametrize("v", [900, 20000, 50257])
def test_numbers_of_entries(paro, k, v):
    z, t, ids = some_inputs(3, v, k, k)
    run_all(paro, z, t, ids, 3.0, "bf16", "f16")


@pytest.mark.parametrize("n", [1, 2, 600])
def test_numbers_of_rows(paro, n):
    z, t, ids = some_inputs(n, 777, 9, n)
    run_all(paro, z, t, ids, 1.0, "f16", "bf16", pad=1)


@pytest.mark.parametrize("T", [0.05, 0.5, 1.0, 20.0, 1000.0])
def test_temperatures(paro, T):
    z, t, ids = some_inputs(4, 3001, 20, 3, masked=False)
    run_all(paro, z * min(T, 1.0), t * min(T, 1.0), ids, T, "f32", "f32")


def test_every_entry_the_same_place(paro):
    z, t, ids = some_inputs(2, 500, 300, 4, masked=False)
    ids[:] = 17
    run_all(paro, z, t, ids, 2.0, "f32", "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("v", [9, 3000, 40000, 140000])
def test_masks(paro, v, dtype):
    """Rows without an entry, with NaN logits that nothing may read; teacher's and student's logits of -inf and of the lowest number; and no
    trace of one row in another."""
    lowest = torch.finfo(TORCH[dtype]).min
    z, t, ids = some_inputs(8, v, 6, v, masked=False)
    ids[0] = -1
    z[0] = math.nan
    t[1] = -math.inf
    z[1] = math.inf
    t[2, :3] = -math.inf
    ids[3, 1:] = v
    # masked words: by -inf and by the lowest number, none of which the teacher names
    free = torch.ones(v, dtype=torch.bool)
    free[ids[4:6].clamp(0, v - 1).flatten()] = False
    z[4, free & (torch.arange(v) % 3 == 0)] = -math.inf
    z[5, free & (torch.arange(v) % 3 == 0)] = lowest
    z[6] = -math.inf                                        # nothing at all: q = 0, the loss infinite
    z[7] = lowest                                           # all words alike
    keep = [0, 1, 2, 3, 4, 5, 6]
    run_all(paro, z[keep], t[keep], ids[keep], 2.0, dtype, "f32", in_place=False)
    if v < 3000:
        d = paro.make_distill(n=1, vocab=v, k=6, temperature=2.0, dtype=code(paro, dtype), teacher_dtype=paro.PARO_F32)
        zd, td, idd = z[7:].to(DEV, TORCH[dtype]), t[7:].to(DEV), ids[7:].int().to(DEV)
        loss, dz = torch.empty(1, device=DEV), torch.empty(1, v, dtype=TORCH[dtype], device=DEV)
        paro.paro_distill_step(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), 0, loss.data_ptr(), dz.data_ptr(), stream())
        p = torch.softmax(t[7].double() / 2, dim=0)
        ref = 2 * (torch.full((v,), 1 / v, dtype=torch.float64) - torch.zeros(v, dtype=torch.float64).scatter_add_(0, ids[7].long(), p))
        check(dz[0], ref, rounding(ref, dtype, torch.full_like(ref, 4 * TINY)), "all words at the lowest number")


def test_a_named_word_that_the_student_masks(paro):
    z, t, ids = some_inputs(3, 100, 4, 1, masked=False)
    z[1, ids[1, 2]] = -math.inf
    run_all(paro, z, t, ids, 1.0, "bf16", "f32")


def test_nan_stays_in_its_row(paro):
    z, t, ids = some_inputs(3, 5000, 4, 1, masked=False)
    z[1, 77] = math.nan
    d = paro.make_distill(n=3, vocab=5000, k=4, temperature=1.0, dtype=paro.PARO_F32, teacher_dtype=paro.PARO_F32)
    zd, td, idd = z.to(DEV), t.to(DEV), ids.int().to(DEV)
    loss, dz = torch.empty(3, device=DEV), torch.empty(3, 5000, device=DEV)
    paro.paro_distill_step(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), 0, loss.data_ptr(), dz.data_ptr(), stream())
    assert loss.isnan().tolist() == [False, True, False] and dz.isnan().any(dim=1).tolist() == [False, True, False]


@pytest.mark.parametrize("T", [1.0, 2.5])
def test_gradient_against_differences_of_the_loss(paro, T):
    """Central differences of the loss that the library computes, along a few logits, named and not."""
    n, v, k, h = 4, 50, 5, 2.0 ** -5
    z, t, ids = some_inputs(n, v, k, 12, masked=False)
    d = paro.make_distill(n=n, vocab=v, k=k, temperature=T, dtype=paro.PARO_F32, teacher_dtype=paro.PARO_F32)
    td, idd = t.to(DEV), ids.int().to(DEV)

    def loss_of(x):
        out, xd = torch.empty(n, device=DEV), x.to(DEV)
        paro.paro_distill_loss(d, xd.data_ptr(), td.data_ptr(), idd.data_ptr(), out.data_ptr(), 0, stream())
        return out.cpu().double()
    loss, dz, zd = torch.empty(n, device=DEV), torch.empty(n, v, device=DEV), z.to(DEV)
    paro.paro_distill_step(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), 0, loss.data_ptr(), dz.data_ptr(), stream())
    dz = dz.cpu().double()
    for at in list(range(0, v, 7)) + ids[0].tolist():
        e = torch.zeros(n, v)
        e[:, at] = h
        slope = (loss_of(z + e) - loss_of(z - e)) / (2 * h)
        # third derivative of T^2 log sum exp(z / T) is at most 1 / T: h^2 / 6; and the two losses' own errors
        bound = h * h / (6 * T) + 2 * TINY * T * T * (20 + loss_of(z).abs()) / (2 * h)
        assert bool(((slope - dz[:, at]).abs() <= bound).all()), at


def test_in_a_graph_and_on_another_stream(paro):
    n, v, k = 33, 6001, 8
    z, t, ids = some_inputs(n, v, k, 2)
    d = paro.make_distill(n=n, vocab=v, k=k, temperature=2.0, dtype=paro.PARO_BF16, teacher_dtype=paro.PARO_F32)
    zd, td, idd = z.to(DEV, torch.bfloat16), t.to(DEV), ids.int().to(DEV)

    def step(loss, dz):
        paro.paro_distill_step(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), 0, loss.data_ptr(), dz.data_ptr(), stream())
    ref, got = ((torch.zeros(n, device=DEV), torch.zeros(n, v, dtype=torch.bfloat16, device=DEV)) for _ in range(2))
    step(*ref)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(*got)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    with torch.cuda.graph(graph):
        step(*got)
    for i in range(3):
        zd.copy_(z + i)
        zd[:, i] += 3
        for b in got:
            b.fill_(float(i))
        graph.replay()
        torch.cuda.synchronize()
        step(*ref)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v,span,k", [(1500, 1500, 250), (1500, 40, 250), (4000, 90, 512), (4000, 30, 40), (8000, 200, 300), (8000, 8000, 1024), (16000, 500, 600),
                                      (16003, 64, 24), (30000, 3000, 1024), (60000, 16, 16)])
def test_several_entries_in_a_piece(paro, v, span, k, dtype):
    """Places that are named often and lie side by side, few of them and many; twice, with the same bits."""
    z, t, _ = some_inputs(4, v, k, v + k, masked=False)
    ids = torch.randint(0, span, (4, k), generator=rng(k)) + torch.tensor([[0], [v - span], [(v - span) // 2], [0]])
    ids[3, ::3] = -1
    z.scatter_(1, ids.clamp(0, v - 1), t + 4)
    run_all(paro, z, t, ids, 2.0, dtype, "f32")
    d = paro.make_distill(n=4, vocab=v, k=k, temperature=2.0, dtype=code(paro, dtype), teacher_dtype=paro.PARO_F32)
    zd, td, idd = z.to(DEV, TORCH[dtype]), t.to(DEV), ids.int().to(DEV)
    loss, got = torch.empty(4, device=DEV), [torch.empty(4, v, dtype=TORCH[dtype], device=DEV) for _ in range(3)]
    for dz in got:
        paro.paro_distill_step(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), 0, loss.data_ptr(), dz.data_ptr(), stream())
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("dtype,v", [("bf16", v) for v in (2047, 2048, 2049, 2055, 2056, 4103, 4104, 8191, 8199, 8200, 16384, 16391, 16392, 24577)]
                         + [("f32", v) for v in (1023, 1024, 1027, 1028, 2051, 2052, 4099, 8195, 8196, 16383)])
def test_row_lengths_between_two_launches(paro, dtype, v):
    z, t, ids = some_inputs(3, v, 7, v)
    run_all(paro, z, t, ids, 2.0, dtype, "bf16", pad=v % 3)
