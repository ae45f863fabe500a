"""Which kernels the attention launches, with how many blocks, on the CPU: the built library runs against a runtime of a few lines that only writes down what it is
asked to launch.  Every pointer is made up.  Holds the sizes by which the tests on the GPU reach each kernel to the kernels that they are there for."""
import os
import subprocess

import pytest

from test_operator_launches import MAIN as OTHERS, Launch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
RUNTIME = OTHERS[:OTHERS.index("int main()")]
MAIN = RUNTIME + r"""
int main() {
    char call[32];
    long batch, heads, kv, hd, n, m, window, sinks, buckets, dtype, pad;
    while (std::scanf("%31s %ld %ld %ld %ld %ld %ld %ld %ld %ld %ld %ld", call, &batch, &heads, &kv, &hd, &n, &m, &window, &sinks, &buckets, &dtype, &pad) == 12) {
        const auto at = [](int i) { return reinterpret_cast<void *>((uintptr_t)(i + 1) << 40); };
        const auto ints = [&](int i) { return static_cast<int32_t *>(at(i)); };
        paro_attn_t d = {};
        d.batch = batch; d.heads = heads; d.kv_heads = kv; d.head_dim = hd; d.len_q = n; d.len_k = m;
        d.ld_q = d.ld_out = heads * hd + pad; d.ld_k = d.ld_v = kv * hd + pad;
        d.window = window; d.sinks = sinks; d.scale = 1.0f; d.dtype = (int32_t)dtype; d.buckets = (int32_t)buckets; d.table_dtype = PARO_F32;
        const int64_t room = (int64_t)1 << 50;
        float *stats = static_cast<float *>(at(4));
        const int rc = std::string(call) == "attn"
            ? paro_attn(&d, at(0), at(1), at(2), nullptr, nullptr, nullptr, at(5), ints(6), at(3), stats, at(7), room, nullptr)
            : paro_attn_grad(&d, at(8), at(0), at(1), at(2), at(3), stats, nullptr, nullptr, nullptr, at(5), ints(6), at(9), at(10), at(11), at(12), at(7), room, nullptr);
        if (rc != PARO_OK) { std::printf("%s\n", paro_last_error()); return 3; }
        std::printf("end\n");
    }
    return 0;
}
"""
BF16, F16 = 0, 2


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    from __graft_entry__ import ensure_built
    ensure_built()
    where = tmp_path_factory.mktemp("attn_launches")
    (where / "main.cpp").write_text(MAIN)
    lib = os.path.join(ROOT, "paper_2310_06003_amd")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), str(where / "main.cpp"), "-o", str(where / "launches"),
                        os.path.join(lib, "libparo.so"), "-Wl,-rpath," + lib, "-Wl,--allow-shlib-undefined", "-rdynamic"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def ask(call, *, batch=1, heads=2, kv=0, hd=64, n, m=0, window=0, sinks=0, buckets=0, dtype=BF16, pad=0):
        line = " ".join(str(x) for x in (call, batch, heads, kv or heads, hd, n, m or n, window, sinks, buckets, dtype, pad))
        r = subprocess.run([str(where / "launches")], input=line, capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stdout[-500:] + r.stderr
        lines = r.stdout.splitlines()
        assert lines[-1] == "end"
        return [Launch(x) for x in lines[:-1]]
    return ask


def names(got):
    return [x.kernel for x in got]


@pytest.mark.parametrize("n,kernel", [(1, "k_attend_few"), (16, "k_attend_few"), (17, "k_attend"), (2047, "k_attend")])
def test_few_queries_and_many(launches, n, kernel):
    assert names(launches("attn", n=n)) == [kernel]


@pytest.mark.parametrize("heads,kv,n,rows", [(2, 2, 1, 16), (16, 1, 1, 16), (17, 1, 1, 32), (8, 4, 8, 16), (8, 4, 9, 32), (40, 4, 16, 160)])
def test_rows_of_few_queries(launches, heads, kv, n, rows):
    """Heads of a group, query by query, in tiles of 16 rows; of two tiles a block beyond."""
    got, = launches("attn", heads=heads, kv=kv, n=n, m=100)
    assert got.flags[3] == ("1" if rows == 16 else "2") and got.x == kv * -(-rows // (16 if rows == 16 else 32))


@pytest.mark.parametrize("size,shares", [(dict(m=700, heads=12), 1), (dict(m=770, heads=12), 2), (dict(m=4000, heads=2), 6), (dict(m=5000, heads=4, kv=2, hd=128, window=3001), 4),
                                         (dict(m=100000, batch=4, heads=32, kv=8, hd=128), 16), (dict(m=4096, batch=32, heads=32, kv=8, hd=128, window=1024, sinks=4), 1)])
def test_shares_of_long_caches(launches, size, shares):
    got = launches("attn", n=1, **size)
    whole = size.get("batch", 1) * (size.get("kv") or size["heads"])
    assert got[0].x == whole * shares and names(got) == ["k_attend_few"] + ["k_attend_join"] * (shares > 1)


@pytest.mark.parametrize("size,blocks,shares", [(dict(n=64, m=5000), 2, 4), (dict(n=17, m=20500, batch=5, heads=3, kv=1), 15, 16), (dict(n=33, m=9000, batch=2, heads=4, kv=2, window=5001, sinks=40), 8, 5),
                                                (dict(n=2200, heads=1), 18, 2), (dict(n=64, m=100000, heads=32, kv=8, hd=128), 32, 16), (dict(n=64, m=2047), 2, 1),
                                                (dict(n=64, m=100000, window=1024, sinks=4), 2, 1), (dict(n=4096, m=4096, heads=12), 384, 1), (dict(n=8192, heads=4, hd=128), 256, 2)])
def test_shares_of_keys(launches, size, blocks, shares):
    got = launches("attn", **size)
    assert got[0].x == blocks * shares and names(got) == ["k_attend"] + ["k_attend_join"] * (shares > 1)
    assert shares == 1 or got[1].x == blocks * 32


@pytest.mark.parametrize("change,arrays", [({}, 0), (dict(pad=8), 0), (dict(pad=4), 2), (dict(hd=72), 0), (dict(hd=70), 2)])
def test_rows_off_sixteen_bytes_are_copied(launches, change, arrays):
    forward, backward = (launches(call, n=100, **change) for call in ("attn", "grad"))
    assert [x.y for x in forward if x.kernel == "k_align"] == [arrays] * (arrays > 0)
    assert [x.y for x in backward if x.kernel == "k_align"] == [2 * arrays] * (arrays > 0)
    assert "k_align" not in names(launches("attn", n=3, m=100, **change))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("buckets", [0, 9])
def test_passes_of_the_gradient(launches, dtype, buckets):
    want = ["k_dots"] + ["k_times"] * (dtype == F16) + ["k_grads"] + ["k_table_grad"] * (buckets > 0)
    got = launches("grad", batch=3, heads=64, n=300, buckets=buckets, dtype=dtype)
    assert names(got) == want


# sizes that tests on the GPU have: tiles of keys that are shared out, of one head (0: none; fewer than all: those with sinks)
@pytest.mark.parametrize("size,joined", [(dict(n=300), 3), (dict(n=1100, heads=1, hd=128, window=100, sinks=4), 9), (dict(n=1500, heads=2, kv=1, window=200, sinks=140), 12),
                                         (dict(n=900, heads=2, kv=1, hd=128, window=40, sinks=4), 8), (dict(n=900, heads=8, hd=128, window=40), 0),
                                         (dict(n=700, heads=6, window=40, sinks=4), 1), (dict(n=700, heads=6, window=40, sinks=140), 2),
                                         (dict(n=1500, heads=16, kv=1, hd=64), 12), (dict(n=1024, batch=8, heads=12), 0)])
def test_shared_tiles_of_keys(launches, size, joined):
    got = [x for x in launches("grad", **size) if x.kernel == "k_grad_join"]
    assert [x.x for x in got] == ([joined * size.get("batch", 1) * (size.get("kv") or size.get("heads", 2))] if joined else [])
