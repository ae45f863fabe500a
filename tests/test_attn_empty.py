"""Attention over nothing, on the CPU: which kernels are launched where a batch, its queries or its keys are none, and which arrays such a call may do without.  The built
library runs against a runtime that only writes down what it is asked to launch; every pointer is made up."""
import os
import subprocess

import pytest

from test_attn_launches import RUNTIME
from test_operator_launches import Launch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# bit i of `none`: argument i of the call is NULL; room: of the workspace, -1: what paro_attn_workspace says
MAIN = RUNTIME + r"""
int main() {
    char call[32];
    long batch, heads, kv, hd, n, m, window, sinks, buckets, dtype, none, room;
    while (std::scanf("%31s %ld %ld %ld %ld %ld %ld %ld %ld %ld %ld %ld %ld", call, &batch, &heads, &kv, &hd, &n, &m, &window, &sinks, &buckets, &dtype, &none, &room) == 13) {
        const auto at = [&](int i) { return none >> i & 1 ? nullptr : reinterpret_cast<void *>((uintptr_t)(i + 1) << 40); };
        const auto ints = [&](int i) { return static_cast<int32_t *>(at(i)); };
        const auto floats = [&](int i) { return static_cast<float *>(at(i)); };
        paro_attn_t d = {};
        d.batch = batch; d.heads = heads; d.kv_heads = kv; d.head_dim = hd; d.len_q = n; d.len_k = m;
        d.window = window; d.sinks = sinks; d.scale = 1.0f; d.dtype = (int32_t)dtype; d.buckets = (int32_t)buckets; d.table_dtype = PARO_F32;
        const bool grad = std::string(call) == "grad";
        const int64_t bytes = room >= 0 ? room : paro_attn_workspace(&d, grad);
        const int rc = grad ? paro_attn_grad(&d, at(0), at(1), at(2), at(3), at(4), floats(5), ints(6), ints(7), ints(8), at(9), ints(10), at(11), at(12), at(13), at(14),
                                             at(15), bytes, nullptr)
                            : paro_attn(&d, at(0), at(1), at(2), ints(3), ints(4), ints(5), at(6), ints(7), at(8), floats(9), at(10), bytes, nullptr);
        if (rc != PARO_OK) { std::printf("%s\n", paro_last_error()); return 3; }
        std::printf("end\n");
    }
    return 0;
}
"""
GRAD = ("dout", "q", "k", "v", "out", "stats", "q_starts", "k_starts", "k_lens", "table", "first", "dq", "dk", "dv", "dtable", "workspace")
FORWARD = ("q", "k", "v", "q_starts", "k_starts", "k_lens", "table", "first", "out", "stats", "workspace")
BF16, F16 = 0, 2


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    from __graft_entry__ import ensure_built
    ensure_built()
    where = tmp_path_factory.mktemp("attn_empty")
    (where / "main.cpp").write_text(MAIN)
    lib = os.path.join(ROOT, "paper_2310_06003_amd")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), str(where / "main.cpp"), "-o", str(where / "launches"),
                        os.path.join(lib, "libparo.so"), "-Wl,-rpath," + lib, "-Wl,--allow-shlib-undefined", "-rdynamic"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def ask(call, *, batch=1, heads=2, kv=0, hd=64, n, m, window=0, sinks=0, buckets=0, dtype=BF16, given=None, room=-1):
        """given: the arrays that are not NULL."""
        names = GRAD if call == "grad" else FORWARD
        given = [x for x in names if not x.endswith(("starts", "lens"))] if given is None else given
        none = sum(1 << i for i, name in enumerate(names) if name not in given)
        line = " ".join(str(x) for x in (call, batch, heads, kv or heads, hd, n, m, window, sinks, buckets, dtype, none, room))
        r = subprocess.run([str(where / "launches")], input=line, capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, (r.returncode, r.stdout[-500:] + r.stderr)
        lines = r.stdout.splitlines()
        assert lines[-1] == "end"
        got = [Launch(x) for x in lines[:-1]]
        assert all(x.x and x.y for x in got), "a launch of nothing"
        return got
    return ask


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("window,sinks", [(0, 0), (10, 0), (10, 4), (1, 1), (99, 100), (10, 200)])
@pytest.mark.parametrize("m", [1, 100, 300, 3000])
def test_keys_without_queries_have_gradients(launches, m, window, sinks, dtype):
    """No query, but keys: each tile of 128 of them has a block at least, which writes its zeros."""
    got = launches("grad", batch=3, n=0, m=m, window=window, sinks=sinks, dtype=dtype)
    blocks = [x.x for x in got if x.kernel == "k_grads"]
    assert len(blocks) == 1 and blocks[0] >= 3 * 2 * -(-m // 128)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hd,m,window,sinks", [(64, 100, 0, 0), (128, 5000, 0, 0), (64, 300, 10, 4), (128, 5000, 200, 300)])
def test_no_sequence_leaves_a_table_without_gradient(launches, hd, m, window, sinks, dtype):
    """batch 0: no array but the table's gradient is needed, nor a workspace; its zeros are one launch."""
    for n in (0, 1, 300):
        got = launches("grad", batch=0, hd=hd, n=n, m=m, window=window, sinks=sinks, buckets=9, dtype=dtype, given=["dtable"])
        assert [(x.kernel, x.x) for x in got] == [("k_table_grad", 2)]
        assert launches("grad", batch=0, hd=hd, n=n, m=m, window=window, sinks=sinks, buckets=9, dtype=dtype, given=[]) == []
        assert launches("grad", batch=0, hd=hd, n=n, m=m, window=window, sinks=sinks, dtype=dtype, given=["dtable"]) == []      # of no bucket


@pytest.mark.parametrize("buckets", [0, 9])
@pytest.mark.parametrize("window,sinks", [(0, 0), (10, 4)])
def test_arrays_without_rows_may_be_null(launches, window, sinks, buckets):
    """An empty tensor's address is 0: arrays of queries are not looked at where len_q is 0, arrays of keys where len_k is."""
    of_q, of_k, more = ["dout", "q", "out", "stats", "dq"], ["k", "v", "dk", "dv"], ["workspace"] + (["table", "first", "dtable"] if buckets else [])
    size = dict(batch=3, window=window, sinks=sinks, buckets=buckets)
    for n, m, given in ((0, 100, of_k), (50, 0, of_q), (1, 0, of_q), (0, 0, [])):
        kernels = [x.kernel for x in launches("grad", n=n, m=m, given=given + more, **size)]
        assert kernels == ["k_dots"] * (n > 0) + ["k_grads"] * (n + m > 0) + ["k_table_grad"] * (buckets > 0)
    for n, m, given in ((0, 100, []), (50, 0, ["q", "out", "stats"]), (1, 0, ["q", "out"]), (0, 0, [])):
        kernels = [x.kernel for x in launches("attn", n=n, m=m, given=given + more, **size)]
        assert kernels == (["k_attend" if n > 16 else "k_attend_few"] if n else [])
