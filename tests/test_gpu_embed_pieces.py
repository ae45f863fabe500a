"""The table's gradient of thousands of tokens, at the widths and types for which a lane takes two and four pieces of a row: runs of every length
beside tokens that the table does not hold, widths on and off the piece, rows apart."""
import pytest
import torch

from operator_sizes import TABLE_GRADIENT
from operators_ref import rng
from test_gpu_embed import gradient

pytestmark = pytest.mark.gpu


def text(n, v, seed):
    """Token numbers of which few have most of the places, a few of them below and beyond the table."""
    u = torch.rand(n, generator=rng(seed), dtype=torch.float64)
    return (torch.exp(u * torch.log(torch.tensor(v + 4.0, dtype=torch.float64))) - 2).long()


@pytest.mark.parametrize("dtype,grad_dtype,n,v,dim", list(TABLE_GRADIENT))
def test_gradient_in_wide_pieces(paro, dtype, grad_dtype, n, v, dim):
    tokens = text(n, v, n + dim)
    gradient(paro, tokens, dim, v, dtype, grad_dtype, pad=n % 3)


@pytest.mark.parametrize("where", ["front", "back", "one", "alternating", "none"])
@pytest.mark.parametrize("dtype,grad_dtype,n,dim", [("bf16", "bf16", 6500, 1001), ("f16", "f32", 6500, 1030), ("bf16", "bf16", 6500, 2050)])
def test_long_runs_in_wide_pieces(paro, dtype, grad_dtype, n, dim, where):
    """Runs that begin and end inside the parts that are summed on their own, in order and out of it."""
    i = torch.arange(n)
    tokens = {"front": torch.where(i < 2111, 0, 1 + i % 8), "back": torch.where(i < 1999, i % 8, 8), "one": torch.full((n,), 4),
              "alternating": i // 65 % 9, "none": torch.full((n,), 9)}[where]
    for order in (i, torch.randperm(n, generator=rng(8))):
        gradient(paro, tokens[order].int(), dim, 9, dtype, grad_dtype, pad=1)
