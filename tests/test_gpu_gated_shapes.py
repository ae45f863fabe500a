"""The gated projections at sizes that take the forms of the kernels that small ones do not: tiles of 256 x 256 and 128 x 128 of each product, whole
and split over the inner dimension, each product in a launch of its own; and backward passes of few tokens over several blocks of columns and
several rounds of hidden elements."""
import pytest

from operator_sizes import BACKWARD, FEW_BACKWARD, FORWARD
from test_gpu_gated import backward, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,dim,hidden,dtype,act,pad", list(FORWARD))
def test_forward_tiles(paro, n, dim, hidden, dtype, act, pad):
    forward(paro, n, dim, hidden, dtype, act, pad=pad)


@pytest.mark.parametrize("n,dim,hidden,dtype,act,pad", list(BACKWARD))
def test_backward_tiles(paro, n, dim, hidden, dtype, act, pad):
    backward(paro, n, dim, hidden, dtype, act, pad=pad)


@pytest.mark.parametrize("n,dim,hidden,dtype,act,pad", list(FEW_BACKWARD))
def test_backward_of_few_tokens(paro, n, dim, hidden, dtype, act, pad):
    backward(paro, n, dim, hidden, dtype, act, pad=pad)
