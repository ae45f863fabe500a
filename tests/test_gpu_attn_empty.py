"""Attention and its gradient where there are no queries, no keys or no sequences, against the definition: what is there is written, nothing else."""
import pytest
import torch

from attn_ref import Case
from operators_ref import DEV, TORCH, code, stream
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


@pytest.mark.parametrize("dtype,table", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
def test_no_sequence_leaves_a_table_without_gradient(paro, dtype, table):
    """batch 0, at once and in a graph: zeros, without a workspace."""
    kinds = dict(batch=0, heads=5, head_dim=64, len_q=300, dtype=code(paro, dtype), window=10, sinks=4, buckets=7, table_dtype=code(paro, table))
    d = paro.make_attn(**kinds)
    assert paro.paro_attn_workspace(d, True) == 0
    whole = torch.full((40,), 7.0, dtype=TORCH[table], device=DEV)

    def check():
        assert bool((whole[:35] == 0).all()) and bool((whole[35:] == 7).all())
        whole[:35] = 7.0
    paro.paro_attn_grad(d, *[0] * 14, whole.data_ptr(), 0, 0, stream())
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        paro.paro_attn_grad(d, *[0] * 14, whole.data_ptr(), 0, 0, stream())
    for _ in range(3):
        graph.replay()
        check()
    paro.paro_attn_grad(d, *[0] * 15, 0, 0, stream())                          # not wanted
    paro.paro_attn(d, *[0] * 10, 0, 0, stream())
    assert bool((whole == 7).all())


@pytest.mark.parametrize("hd,dtype,buckets", [(64, "bf16", 0), (128, "f16", 5), (77, "bf16", 3)])
def test_arrays_of_no_rows_are_null(paro, hd, dtype, buckets):
    """What an empty tensor's address is, 0, in the place of the queries' arrays, and of the keys'."""
    empty = torch.empty(0, 4, hd, dtype=TORCH[dtype], device=DEV)
    assert empty.data_ptr() == 0
    c = Case(paro, [(0, 100), (0, 40)], hd=hd, heads=4, kv=2, dtype=dtype, buckets=buckets, window=10, sinks=4)
    for x in (c.q, c.dout, c.out, c.dq):
        x.view = empty
    c.stats = torch.empty(0, 4, 2, device=DEV)
    c.forward()
    c.backward()
    c.check_backward()
    c = Case(paro, [(40, 0), (100, 0)], hd=hd, heads=4, kv=2, dtype=dtype, buckets=buckets, window=10, sinks=4)
    for x in (c.k, c.v, c.dk, c.dv):
        x.view = empty[:, :2]
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
