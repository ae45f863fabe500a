"""Attention and its gradient where there are no queries, no keys or no sequences, against the definition: what is there is written, nothing else."""
import pytest

from test_gpu_attn_grad import backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("buckets", [0, 5])
@pytest.mark.parametrize("window,sinks", [(0, 0), (10, 0), (10, 4), (1, 1), (10, 140), (99, 500)])
def test_keys_without_queries(paro, window, sinks, buckets, dtype):
    """len_q is zero: the gradients of keys and values are zeros, those of the keys with sinks too."""
    for hd, lengths in ((64, [(0, 100)]), (128, [(0, 300), (0, 31)]), (72, [(0, 700)])):
        c = backward(paro, lengths, hd=hd, heads=4, kv=2, dtype=dtype, buckets=buckets, window=window, sinks=sinks)
        assert all(bool((x.view[x.held] == 0).all()) for x in (c.dk, c.dv))


def test_sequences_without_queries_among_others(paro):
    backward(paro, [(0, 300), (200, 300), (0, 5), (40, 40)], heads=4, kv=2, window=30, sinks=5, buckets=6, dtype="f16")
