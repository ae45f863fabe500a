"""Attention whose last bucket begins beyond 1024 tokens, where each tile looks its distances up, over sequences that reach beyond it: forward, for new tokens over a cache, and backward."""
import pytest
import torch

from attn_ref import Case
from test_gpu_attn import forward
from test_gpu_attn_grad import backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,dtype,table", [(64, "bf16", "f32"), (128, "bf16", "bf16"), (128, "f16", "f16"), (72, "f16", "f32")])
@pytest.mark.parametrize("buckets,far", [(40, 1500), (256, 1600), (2, 2500)])
def test_tiles_in_front_of_and_beyond_the_last_bucket(paro, buckets, far, hd, dtype, table):
    kw = dict(hd=hd, dtype=dtype, buckets=buckets, far=far, table=table)
    c = forward(paro, [(1700, 1700)], heads=1, **kw)
    assert (c.first_list[-1] > 1024) == (buckets > 2)
    forward(paro, [(5, 1800), (1, 1300), (16, 40)], heads=4, kv=2, **kw)
    forward(paro, [(100, 2500), (17, 30)], heads=2, kv=1, **kw)
    backward(paro, [(1700, 1700)], heads=1, **kw)
    backward(paro, [(130, 1500), (300, 300), (200, 150)], heads=4, kv=2, **kw)
    backward(paro, [(500, 1500)], heads=2, kv=1, window=1300, sinks=70, **kw)


@pytest.mark.parametrize("value", [-1e9, -torch.inf, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("far", [100, 1500])
def test_a_last_bucket_that_hides(paro, far, hd, value):
    """Tiles beyond the last bucket's beginning whose bias is no usual number; some queries see others too, with sinks."""
    for lengths in ([(1400, 1400)], [(3, 1400), (16, 1300)]):
        c = Case(paro, lengths, heads=2, kv=1, hd=hd, buckets=40, far=far)
        c.table[-1] = value
        c.table[7] = value
        c.forward()
        c.check_forward()
        if lengths[0][0] > 16:
            c.set_forward()
            c.backward()
            c.check_backward()
