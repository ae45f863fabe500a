"""Which kernels the operators beside the Update stage launch, with how many blocks, on the CPU: the built library runs against a runtime of a few
lines that only writes down what it is asked to launch.  Every pointer is made up.  Holds the sizes by which the tests on the GPU reach each
of the kernels' forms to the forms they were chosen for, so that another rule cannot take them off unseen."""
import os
import subprocess

import pytest

import operator_sizes as sizes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = r"""
#include <cxxabi.h>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include "paro.h"

struct dim3 { uint32_t x, y, z; };
static dim3 grid_, block_;
static size_t lds_;
static std::map<const void *, std::string> &kernels() { static std::map<const void *, std::string> k; return k; }
extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *handle; return &handle; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) {
    int status;
    char *plain = abi::__cxa_demangle(name, nullptr, nullptr, &status);
    std::string n = status == 0 ? plain : name;
    std::free(plain);
    for (size_t at; (at = n.find("(anonymous namespace)::")) != std::string::npos;) n.erase(at, 23);
    kernels()[host] = n.rfind("void ", 0) == 0 ? n.substr(5) : n;
}
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, void *) { grid_ = grid; block_ = block; lds_ = lds; return 0; }
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, void **st) { *grid = grid_; *block = block_; *lds = lds_; *st = nullptr; return 0; }
int hipLaunchKernel(const void *f, dim3 grid, dim3, void **, size_t, void *) {
    std::printf("%s\t%u\t%u\n", kernels()[f].c_str(), grid.x, grid.y);
    return 0;
}
int hipFuncSetAttribute(const void *, int, int) { return 0; }
int hipGetDevice(int *d) { *d = 0; return 0; }
int hipDeviceGetAttribute(int *v, int, int) { *v = 160 * 1024; return 0; }
int hipMalloc(void **p, size_t n) { return (*p = std::malloc(n)) ? 0 : 2; }
int hipFree(void *p) { std::free(p); return 0; }
int hipMemcpy(void *to, const void *from, size_t n, int) { std::memcpy(to, from, n); return 0; }
int hipGetLastError() { return 0; }
const char *hipGetErrorString(int) { return "?"; }
int hipGetSymbolAddress(void **p, const void *) { static double one; *p = &one; return 0; }
}

int main() {
    char call[32];
    long n, a, b, dtype, other, pad;
    while (std::scanf("%31s %ld %ld %ld %ld %ld %ld", call, &n, &a, &b, &dtype, &other, &pad) == 7) {
        const auto at = [](int i) { return reinterpret_cast<void *>((uintptr_t)(i + 1) << 40); };
        int rc;
        const std::string what = call;
        const int64_t room = (int64_t)1 << 50;
        if (what == "embed_grad") {                                 // rows a, dim b
            rc = paro_embed_grad(at(0), (int)dtype, b + pad, at(1), PARO_I64, n, 0, 1.0f, at(2), (int)other, a, b, at(3), room, nullptr);
        } else if (what.rfind("distill", 0) == 0) {                 // vocab a, k b
            paro_distill_t d = {n, a, b, a + pad, 0, a + pad, 2.0f, (int32_t)dtype, (int32_t)other, 0};
            const int32_t *ids = (const int32_t *)at(2);
            float *loss = (float *)at(3), *lse = (float *)at(4);
            if (what == "distill_loss") rc = paro_distill_loss(&d, at(0), at(1), ids, loss, lse, nullptr);
            else if (what == "distill_grad") rc = paro_distill_grad(&d, at(0), at(1), ids, lse, nullptr, at(6), nullptr);
            else rc = paro_distill_step(&d, at(0), at(1), ids, nullptr, loss, at(6), nullptr);
        } else {                                                    // dim a, hidden b
            paro_gated_t d = {n, a, b, a + pad, b + pad, (int32_t)dtype, (int32_t)other};
            if (what == "gated") rc = paro_gated(&d, at(0), at(1), at(2), at(3), at(4), at(5), at(6), room, nullptr);
            else rc = paro_gated_grad(&d, at(0), at(1), at(2), at(3), at(4), at(5), at(6), at(7), at(8), at(9), room, nullptr);
        }
        if (rc != PARO_OK) { std::printf("%s\n", paro_last_error()); return 3; }
        std::printf("end\n");
    }
    return 0;
}
"""
BF16, F32, F16 = 0, 1, 2
SILU, GELU = 0, 1


class Launch:
    def __init__(self, line):
        name, x, y = line.split("\t")
        self.name = name[:name.index("(")]
        self.kernel, self.x, self.y = self.name.split("<")[0], int(x), int(y)
        self.flags = [f.strip() for f in self.name[self.name.index("<") + 1:-1].split(",")] if "<" in self.name else []


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    from __graft_entry__ import ensure_built
    ensure_built()
    where = tmp_path_factory.mktemp("launches")
    (where / "main.cpp").write_text(MAIN)
    lib = os.path.join(ROOT, "paper_2310_06003_amd")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), str(where / "main.cpp"), "-o", str(where / "launches"),
                        os.path.join(lib, "libparo.so"), "-Wl,-rpath," + lib, "-Wl,--allow-shlib-undefined", "-rdynamic"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def ask(call, n, a, b, dtype, other=0, pad=0):
        r = subprocess.run([str(where / "launches")], input=f"{call} {n} {a} {b} {dtype} {other} {pad}", capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stdout[-500:] + r.stderr
        lines = r.stdout.splitlines()
        assert lines[-1] == "end"
        return [Launch(x) for x in lines[:-1]]
    return ask


def tiles_of(got, mode):
    """Side of a product's tiles, and how many of them are split."""
    product, = [x for x in got if x.kernel == "k_product" and x.flags[1] == str(mode)]
    side = int(product.flags[3])
    split = [x.x for x in got if x.kernel == "k_join" and x.flags[1] == str(mode)]
    at_once = 256 if side == 256 else 512
    return f"{side} " + ("unsplit" if not split else "rest split" if product.x > at_once else "all split")


DTYPES, ACTS = {"bf16": BF16, "f16": F16, "f32": F32}, {"silu": SILU, "gelu": GELU}


@pytest.mark.parametrize("size", list(sizes.FORWARD))
def test_forms_of_the_forward_pass(launches, size):
    n, dim, hidden, dtype, act, pad = size
    assert tiles_of(launches("gated", n, dim, hidden, DTYPES[dtype], ACTS[act], pad), 0) == sizes.FORWARD[size]


@pytest.mark.parametrize("size", list(sizes.BACKWARD))
def test_forms_of_the_backward_pass(launches, size):
    n, dim, hidden, dtype, act, pad = size
    got = launches("gated_grad", n, dim, hidden, DTYPES[dtype], ACTS[act], pad)
    assert (tiles_of(got, 1), tiles_of(got, 2)) == sizes.BACKWARD[size]


def test_every_form_of_every_product_has_a_size():
    forms = {f"{side} {how}" for side in (256, 128) for how in ("unsplit", "rest split", "all split")}
    assert set(sizes.FORWARD.values()) == forms
    assert {dx for dx, _ in sizes.BACKWARD.values()} == forms and {dw for _, dw in sizes.BACKWARD.values()} == forms


@pytest.mark.parametrize("size", list(sizes.FEW_BACKWARD))
def test_forms_of_few_tokens_backward(launches, size):
    n, dim, hidden, dtype, act, pad = size
    grad, join = launches("gated_grad", n, dim, hidden, DTYPES[dtype], ACTS[act], pad)
    assert (grad.kernel, join.kernel) == ("k_few_grad", "k_few_join")
    assert (grad.y, -(-hidden // grad.x)) == sizes.FEW_BACKWARD[size]


@pytest.mark.parametrize("size", list(sizes.TABLE_GRADIENT))
def test_pieces_of_the_table_gradient(launches, size):
    dtype, grad_dtype, n, rows, dim = size
    sums, = [x for x in launches("embed_grad", n, rows, dim, DTYPES[dtype], DTYPES[grad_dtype]) if x.kernel == "k_sums"]
    assert int(sums.flags[2]) == sizes.TABLE_GRADIENT[size]
