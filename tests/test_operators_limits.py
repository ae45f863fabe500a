"""The largest sizes that the operators beside the Update stage take, and one more, on the host: what is taken gets to a later check (an array that is
missing, a workspace that is too small), what is not is refused for its size.  Every pointer is made up."""
import pytest

import paper_2310_06003_amd as paro

P = 1 << 12          # an address that nothing follows


def refusal(call):
    with pytest.raises(paro.ParoError) as e:
        call()
    return e.value.code, str(e.value)


@pytest.mark.parametrize("name,most", [("n", 2 ** 31 - 1), ("rows", 2 ** 30), ("dim", 2 ** 24)])
def test_embed_limits(name, most):
    sizes = dict(n=5, rows=7, dim=8)
    for value, taken in ((most, True), (most + 1, False), (-1, False)):
        a = {**sizes, name: value}
        code, text = refusal(lambda: paro.paro_embed(P, paro.PARO_BF16, a["rows"], a["dim"], P, paro.PARO_I32, a["n"], 0, 1.0, 0))
        assert ("out is NULL" if taken else f"{name} must be") in text and code == paro.PARO_EINVAL
        code, text = refusal(lambda: paro.paro_embed_grad(P, paro.PARO_BF16, 0, P, paro.PARO_I32, a["n"], 0, 1.0, P, paro.PARO_F32, a["rows"], a["dim"], P, 0))
        assert (code, "workspace" in text) == (paro.PARO_ERANGE, True) if taken else (code, f"{name} must be" in text) == (paro.PARO_EINVAL, True)
        if taken:
            assert paro.paro_embed_grad_workspace(a["n"], a["rows"], a["dim"]) >= 4 * (a["rows"] + 1 + 2 * a["n"])


@pytest.mark.parametrize("name,most,text", [("n", 2 ** 22 - 1, "n must be"), ("vocab", 2 ** 31 - 1 - 8192, "vocab"), ("k", paro.PARO_DISTILL_MAX_K, "k must be")])
def test_distill_limits(name, most, text):
    sizes = dict(n=4, vocab=2000, k=8, temperature=1.0, dtype=paro.PARO_F32, teacher_dtype=paro.PARO_F32)
    for value, taken in ((most, True), (most + 1, False)):
        d = paro.make_distill(**{**sizes, name: value})
        for call in (lambda: paro.paro_distill_loss(d, P, P, P, 0), lambda: paro.paro_distill_step(d, P, P, P, 0, 0, P),
                     lambda: paro.paro_distill_grad(d, P, P, P, 0, 0, P)):
            assert ("is NULL" if taken else text) in refusal(call)[1]


@pytest.mark.parametrize("temperature,taken", [(1e-6, True), (1e6, True), (9.9e-7, False), (1.01e6, False)])
def test_temperature_limits(temperature, taken):
    d = paro.make_distill(n=4, vocab=10, k=2, temperature=temperature, dtype=paro.PARO_F32, teacher_dtype=paro.PARO_F32)
    assert ("loss is NULL" if taken else "temperature") in refusal(lambda: paro.paro_distill_loss(d, P, P, P, 0))[1]


@pytest.mark.parametrize("name,most,text", [("n", 2 ** 22, "n must be"), ("dim", 2 ** 20, "dim"), ("hidden", 2 ** 20, "hidden"), ("ld_x", 2 ** 21, "2^21"),
                                            ("ld_h", 2 ** 21, "2^21")])
def test_gated_limits(name, most, text):
    sizes = dict(n=40, dim=64, hidden=32, dtype=paro.PARO_F16)
    for value, taken in ((most, True), (most + 1, False)):
        d = paro.make_gated(**{**sizes, name: value})
        if taken:
            assert all(paro.paro_gated_workspace(d, grad) >= 16 for grad in (False, True))
        else:
            assert text in refusal(lambda: paro.paro_gated_workspace(d, False))[1]
        code, got = refusal(lambda: paro.paro_gated(d, P, P, P, 0, 0, 0, P, 1 << 50))
        assert ("h is NULL" if taken else text) in got and code == paro.PARO_EINVAL
        code, got = refusal(lambda: paro.paro_gated_grad(d, *[P] * 9, P, 0))
        assert (code == paro.PARO_ERANGE) if taken else text in got
