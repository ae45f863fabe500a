"""The example that trains a small model with the operators and the Update stage together: its gradients against torch's own in 32 bits, and
that it learns."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example(paro):
    import distill_train
    return distill_train


@pytest.mark.parametrize("n,vocab,dim,hidden,k", [(100, 504, 64, 136, 7), (33, 1000, 40, 88, 20)])
def test_gradients_against_torch(example, n, vocab, dim, hidden, k):
    g = torch.Generator(device="cuda").manual_seed(5)
    T = 2.0
    flat = example.random_parameters(vocab, dim, hidden, g).to(torch.bfloat16)
    model, run = example.Model(flat, vocab, dim, hidden), example.Pass(n, vocab, dim, hidden, k, T)
    tokens = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    ids = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:k] for _ in range(n)])
    teacher = torch.randn(n, k, generator=g, device="cuda").to(torch.bfloat16)
    grads = example.Model(torch.full_like(flat, 7.0), vocab, dim, hidden)
    loss = run.forward_backward(model, tokens, teacher, ids.int(), grads).clone()

    w = {name: getattr(model, name).float().requires_grad_() for name in model.NAMES}
    x = w["table"][tokens] * dim ** 0.5
    h = torch.nn.functional.silu(x @ w["w_gate"].t()) * (x @ w["w_up"].t())
    log_q = torch.log_softmax((x + h @ w["w_down"].t()) @ w["head"].t() / T, dim=1)
    log_p = torch.log_softmax(teacher.float() / T, dim=1)
    ref = (log_p.exp() * (log_p - log_q.gather(1, ids))).sum(dim=1) * T * T
    ref.mean().backward()
    ref = ref.detach()
    # bf16 activations: each of the six roundings on the way is 2^-9 of a value on average, 2^-8 at most
    assert float((loss - ref).abs().max() / ref.abs().max()) < 6 * 2.0 ** -8
    for name in model.NAMES:
        got, want = getattr(grads, name).float(), w[name].grad
        off = float((got - want).norm() / want.norm())
        assert off < 6 * 2.0 ** -8, (name, off)


def test_it_learns(example):
    losses = example.train(steps=25, ranks=2, tokens=256, vocab=1000, dim=64, hidden=128)
    assert all(b == b for b in losses) and losses[-1] < 0.5 * losses[0]
    assert losses == example.train(steps=25, ranks=2, tokens=256, vocab=1000, dim=64, hidden=128), "another run gave other bits"
