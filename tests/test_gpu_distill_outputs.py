"""Outputs of the distillation calls that the definition's tests leave open: the step's own loss where rows hold NaN, and the gradient written
over the logits by paro_distill_grad."""
import math

import pytest
import torch

from operators_ref import DEV, TORCH, code, rng, rows, stream
from test_gpu_distill import run_all, some_inputs

pytestmark = pytest.mark.gpu


def some(n, v, k, seed):
    g = rng(seed)
    z, t = torch.randn(n, v, generator=g) * 2, torch.randn(n, k, generator=g)
    ids = torch.randint(-1, v, (n, k), generator=g)
    ids[n // 2] = -1
    return z, t, ids


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [7, 500, 5000, 30011, 140003])
def test_loss_of_the_step_is_the_loss(paro, v, dtype):
    """Bit for bit, row by row, NaN where the loss is NaN and nowhere else."""
    z, t, ids = some(7, v, 6, v)
    ids[1, 0] = ids[2, 0] = 0
    z[1, v // 2], z[2, 0] = math.nan, -math.inf
    z[3] = math.nan                                         # a row that holds no entry
    d = paro.make_distill(n=7, vocab=v, k=6, temperature=2.0, dtype=code(paro, dtype), teacher_dtype=paro.PARO_F32)
    zd, td, idd = z.to(DEV, TORCH[dtype]), t.to(DEV), ids.int().to(DEV)
    loss, step = (torch.full((7,), 77.0, device=DEV) for _ in range(2))
    dz = torch.empty(7, v, dtype=TORCH[dtype], device=DEV)
    paro.paro_distill_loss(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), loss.data_ptr(), 0, stream())
    paro.paro_distill_step(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), 0, step.data_ptr(), dz.data_ptr(), stream())
    assert loss.isnan().tolist() == [False, True] + [False] * 5 and bool(loss[2].isposinf()) and float(loss[3]) == 0.0
    assert bool(((loss == step) | (loss.isnan() & step.isnan())).all())


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("dtype,v", [(d, v) for d in ("bf16", "f16", "f32") for v in (5, 1000, 9001, 50257)] + [("f32", 65541), ("bf16", 131081)])
def test_gradient_over_the_logits(paro, dtype, v, pad):
    """The same bits as into an array of its own, nothing written between the rows."""
    z, t, ids = some(5, v, 9, v)
    d = paro.make_distill(n=5, vocab=v, k=9, temperature=2.0, dtype=code(paro, dtype), teacher_dtype=paro.PARO_F32, ld_logits=v + pad, ld_dlogits=v + pad)
    whole, zd = rows(5, v, pad, dtype, fill=5.0)
    zd.copy_(z.to(TORCH[dtype]))
    td, idd, w = t.to(DEV), ids.int().to(DEV), torch.rand(5, generator=rng(1)).to(DEV)
    loss, lse = torch.empty(5, device=DEV), torch.empty(5, device=DEV)
    paro.paro_distill_loss(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), loss.data_ptr(), lse.data_ptr(), stream())
    apart = rows(5, v, pad, dtype)[1]
    for target in (apart, zd):
        paro.paro_distill_grad(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), lse.data_ptr(), w.data_ptr(), target.data_ptr(), stream())
    assert torch.equal(apart, zd)
    zd.fill_(5.0)
    assert bool((whole == 5.0).all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("v,k", [(900, 1024), (1500, 600), (4096, 513)])
def test_many_entries_in_short_rows(paro, dtype, v, k):
    """More entries than the few threads of a short row would have taken: more threads."""
    z, t, ids = some_inputs(3, v, k, v + k)
    run_all(paro, z, t, ids, 2.0, dtype, "f32", pad=v % 3)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", [0.05, 0.25, 0.5, 1.0, 2.0])
@pytest.mark.parametrize("v", [40, 5000, 140003])
def test_loss_of_a_named_word_at_the_lowest_number(paro, v, T, dtype):
    """The student masks a word that the teacher names with the lowest number of a type: the loss, about T p times that, mostly is a number of fp32,
    although the logit by T may be none.  Where it is beyond them it is infinite."""
    n, k = 6, 5
    z, t, ids = torch.randn(n, v, generator=rng(v)), torch.randn(n, k, generator=rng(v + 1)) * T, torch.stack([torch.randperm(v, generator=rng(i))[:k] for i in range(n)])
    for row in range(1, n):
        z[row, ids[row, row - 1]] = torch.finfo(TORCH[dtype]).min
    t[:, 0] += 2 * T                        # the others' shares are small
    z[1, ids[1, 0]], z[1, ids[1, 1]] = z[0, 0], torch.finfo(TORCH[dtype]).min
    d = paro.make_distill(n=n, vocab=v, k=k, temperature=T, dtype=code(paro, dtype), teacher_dtype=paro.PARO_F32)
    zd, td, idd = z.to(DEV, TORCH[dtype]), t.to(DEV), ids.int().to(DEV)
    loss, step, dz = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, v, dtype=TORCH[dtype], device=DEV)
    paro.paro_distill_loss(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), loss.data_ptr(), 0, stream())
    paro.paro_distill_step(d, zd.data_ptr(), td.data_ptr(), idd.data_ptr(), 0, step.data_ptr(), dz.data_ptr(), stream())
    assert torch.equal(loss, step)
    T64 = float(torch.tensor(T, dtype=torch.float32))
    log_p, log_q = torch.log_softmax(t.double() / T64, dim=1), torch.log_softmax(z.to(TORCH[dtype]).double() / T64, dim=1).gather(1, ids)
    terms = log_p.exp() * (log_p - log_q)
    ref, size = T64 * T64 * terms.sum(dim=1), T64 * T64 * (log_p.exp() * (log_p.abs() + log_q.abs() + 2)).sum(dim=1)
    ref = ref.float().double()
    # as in the tests of the operator: an exponent carries its own size in roundings
    got = loss.cpu().double()
    assert bool(((got == ref) | ((got - ref).abs() <= 2.0 ** -20 * size * (1 + log_p.abs().amax(dim=1) / 2)) & ref.isfinite()).all()), (loss, ref)
