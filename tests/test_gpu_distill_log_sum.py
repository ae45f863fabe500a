"""The distillation gradient from the stored log-sum: as exact as its argument lets it be where logits are large, and the same as the step's
where a log-sum in 32 bits says nothing about the row any more."""
import pytest
import torch

from operators_ref import DEV, EPS32, TORCH, check, code, put, rng, rounding, rows, stream

pytestmark = pytest.mark.gpu
STORED = 1024.0          # log-sums below this size are taken as they are stored; of larger ones the row's own is formed anew
TINY = 2.0 ** -20        # as in the tests of the operator: a few fp32 roundings and the exponential's


def entries(n, v, k, seed):
    g = rng(seed)
    return torch.randn(n, k, generator=g), torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(n)])


def calls(paro, z, t, ids, T, dtype):
    """lse, gradient from it, gradient of the step, in that order; and the logits as the dtype holds them."""
    n, v = z.shape
    zd, z64 = put(z, 3, dtype)
    td, idd, w = t.to(DEV), ids.int().to(DEV), torch.rand(n, generator=rng(n + v)) + 0.5
    wd = w.to(DEV)
    d = paro.make_distill(n=n, vocab=v, k=t.shape[1], temperature=T, dtype=code(paro, dtype), teacher_dtype=paro.PARO_F32, ld_logits=v + 3, ld_dlogits=v + 3)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    args = zd.data_ptr(), td.data_ptr(), idd.data_ptr()
    paro.paro_distill_loss(d, *args, loss.data_ptr(), lse.data_ptr(), stream())
    grad, step = rows(n, v, 3, dtype)[1], rows(n, v, 3, dtype)[1]
    paro.paro_distill_grad(d, *args, lse.data_ptr(), wd.data_ptr(), grad.data_ptr(), stream())
    paro.paro_distill_step(d, *args, wd.data_ptr(), loss.data_ptr(), step.data_ptr(), stream())
    return lse.cpu().double(), grad, step, z64, w.double()


def teacher_at(t, ids, T, v):
    p = torch.softmax(t.double() / T, dim=1)
    return torch.zeros(t.shape[0], v, dtype=torch.float64).scatter_add_(1, ids.long(), p)


@pytest.mark.parametrize("v", [40, 3000, 30000, 70001])
@pytest.mark.parametrize("T", [1.0, 2.0, 3.0, 0.7])
@pytest.mark.parametrize("around", [0.0, 100.0, -100.0, 1000.0, -1000.0, 30000.0])
def test_large_logits(paro, around, T, v):
    """q = exp(z / T - lse) for the log-sum as it is stored, or, where that is large, in 64 bits.  Beside a few roundings of the exponent's own size, what 1 / T is off by in 32
    bits counts at the size of z / T; nothing else does."""
    t, ids = entries(4, v, 5, v)
    z = around + 3 * torch.randn(4, v, generator=rng(v + 1))
    lse, grad, _, z64, w = calls(paro, z, t, ids, T, "f32")
    T32 = torch.tensor(T, dtype=torch.float32)
    off = abs(float((1 / T32).double() * T32.double()) - 1)
    T64 = float(T32)
    lse = torch.where(lse.abs() < STORED, lse, torch.logsumexp(z64 / T64, dim=1))
    x = z64 / T64 - lse[:, None]
    P, wT = teacher_at(t, ids, T64, v), w[:, None] * T64
    ref = wT * (x.exp() - P)
    err = wT * (x.exp() * ((z64 / T64).abs() * off * 1.001 + TINY * (1 + x.abs() / 2)) + 4 * TINY * P) + 2.0 ** -120
    check(grad, ref, rounding(ref, "f32", err), "gradient")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T", [0.25, 1.0, 1.4, 2.0])
@pytest.mark.parametrize("v", [9, 3000, 40000, 140000])
def test_all_words_at_the_lowest_number(paro, v, T, dtype):
    """A mask over the whole row, entries held: every word has 1 / V."""
    t, ids = entries(3, v, 4, v)
    z = torch.full((3, v), torch.finfo(TORCH[dtype]).min)
    z[1] = 1.0
    _, grad, step, _, w = calls(paro, z, t, ids, T, dtype)
    T64 = float(torch.tensor(T, dtype=torch.float32))
    P, wT = teacher_at(t, ids, T64, v), w[:, None] * T64
    ref = wT * (1 / v - P)
    err = wT * 4 * TINY * (1 / v + P)
    check(step, ref, rounding(ref, dtype, err), "step")
    check(grad, ref, rounding(ref, dtype, err + wT / v * EPS32 * 32), "gradient")       # the ordinary row's log-sum: below 32


@pytest.mark.parametrize("v", [9, 3000, 40000, 70003])
@pytest.mark.parametrize("T,around", [(1.0, 3e6), (3.0, -3e6), (1e-5, 0.0), (2.0, 1e30)])
def test_log_sums_that_32_bits_do_not_resolve(paro, v, T, around):
    """Neighbouring numbers far out: their differences are exact, the log-sum's last place is worth more than they are."""
    t, ids = entries(3, v, 4, v)
    g = rng(v + 2)
    z = torch.randint(0, 4, (3, v), generator=g).float() * (T if T < 1 else 1.0) * 0.5
    z = (z + around).float()
    lse, grad, step, z64, w = calls(paro, z, t * min(T, 1.0), ids, T, "f32")
    T64 = float(torch.tensor(T, dtype=torch.float32))
    q, P, wT = torch.softmax(z64 / T64, dim=1), teacher_at(t * min(T, 1.0), ids, T64, v), w[:, None] * T64
    ref = wT * (q - P)
    # where the log-sum is small it counts as stored: 2^-24 of it
    err = wT * (q * (4 * TINY + EPS32 * torch.where(lse.abs() < STORED, lse.abs(), 0.0)[:, None]) + 8 * TINY * P) + 2.0 ** -120
    check(step, ref, rounding(ref, "f32", err), "step")
    check(grad, ref, rounding(ref, "f32", err), "gradient")


@pytest.mark.parametrize("which", ["grad", "step"])
def test_the_teachers_share_is_as_exact_as_its_roundings(paro, which):
    """Named words that the student masks: their gradient is -T w p alone.  Over many rows p is off, in the mean square, by what its own roundings
    make up: the exponent's (at a size of 3 about 5e-8), the exponential's (7e-8), the sum's, its reciprocal's and the product's (4 to 5e-8
    each), 1.2e-7 together.  Divided by its sum through a logarithm it would be off by that logarithm's rounding too, at its size."""
    n, v, k, T = 512, 2000, 100, 2.0
    g = rng(5)
    t, ids = torch.randn(n, k, generator=g) * 2, torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(n)])
    z = torch.randn(n, v, generator=g).scatter_(1, ids, float("-inf"))
    zd, td, idd = z.to(DEV), t.to(DEV), ids.int().to(DEV)
    d = paro.make_distill(n=n, vocab=v, k=k, temperature=T, dtype=paro.PARO_F32, teacher_dtype=paro.PARO_F32)
    loss, lse, dz = torch.empty(n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, v, device=DEV)
    args = zd.data_ptr(), td.data_ptr(), idd.data_ptr()
    paro.paro_distill_loss(d, *args, loss.data_ptr(), lse.data_ptr(), stream())
    if which == "grad":
        paro.paro_distill_grad(d, *args, lse.data_ptr(), 0, dz.data_ptr(), stream())
    else:
        paro.paro_distill_step(d, *args, 0, loss.data_ptr(), dz.data_ptr(), stream())
    got, ref = -dz.cpu().double().gather(1, ids) / T, torch.softmax(t.double() / T, dim=1)
    assert float((got - ref).norm() / ref.norm()) < 1.5e-7
