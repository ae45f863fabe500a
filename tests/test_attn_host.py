"""The attention on the host: what its calls refuse, before anything touches a GPU, and with which code; workspaces; the first distances of the buckets; the
extension that reads the usual arguments against the ctypes forms.  Every pointer is made up."""
import itertools
import math
from fractions import Fraction

import pytest

import paper_2310_06003_amd as paro

P = 1 << 12          # an address that nothing follows
ROOM = 1 << 40
ATTN = dict(batch=2, heads=4, kv_heads=2, head_dim=64, len_q=100, len_k=100, dtype=paro.PARO_BF16, buckets=8, table_dtype=paro.PARO_F32)
NAMES = ("q", "k", "v", "q_starts", "k_starts", "k_lens", "table", "first", "out", "stats")
GRAD_NAMES = ("dout", "q", "k", "v", "out", "stats", "q_starts", "k_starts", "k_lens", "table", "first", "dq", "dk", "dv", "dtable")


def refused(call, code, text):
    with pytest.raises(paro.ParoError) as e:
        call()
    assert e.value.code == code and text in str(e.value), str(e.value)


@pytest.mark.parametrize("change,text", [
    (dict(dtype=paro.PARO_F32), "dtype"), (dict(dtype=9), "dtype"), (dict(batch=-1), "batch"), (dict(batch=2**20 + 1), "batch"), (dict(heads=0), "heads"),
    (dict(heads=1026), "heads"), (dict(heads=5), "multiple of kv_heads"), (dict(kv_heads=-2), "heads"), (dict(head_dim=0), "head_dim"), (dict(head_dim=7), "head_dim"), (dict(head_dim=129), "head_dim"),
    (dict(len_q=-2), "len_q"), (dict(len_q=2**30 + 1), "len_q"), (dict(len_k=2**31), "len_q"), (dict(rows_q=-1), "rows_q"), (dict(rows_k=2**31), "rows_q"),
    (dict(batch=4, len_q=2**30), "rows of queries"), (dict(batch=4, len_k=2**30), "rows of keys"), (dict(window=-1), "window"), (dict(sinks=-1), "window"),
    (dict(scale=-1.0), "scale"), (dict(scale=1e-19), "scale"), (dict(scale=1e19), "scale"), (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"), (dict(buckets=-1), "buckets"), (dict(buckets=257), "buckets"),
    (dict(table_dtype=paro.PARO_F16), "table_dtype"), (dict(ld_q=255), "longer"), (dict(ld_k=127), "longer"), (dict(ld_v=1), "longer"), (dict(ld_out=-256), "longer"),
    (dict(head_q=63), "longer"), (dict(head_k=-64), "longer"), (dict(head_v=65, ld_v=128), "longer"), (dict(head_out=80, ld_out=300), "longer"),
    (dict(ld_k=2**24 + 1), "2^24"), (dict(head_v=2**50 + 1), "2^50"), (dict(heads=1024, kv_heads=1, batch=2, len_q=2**29, len_k=1), "2^34"),
    (dict(rows_q=199), "rows_q holds"), (dict(rows_k=199), "rows_k holds")])
def test_refuses(change, text):
    d = paro.make_attn(**{**ATTN, **change})
    if "holds" not in text:
        for grad in (False, True):
            refused(lambda: paro.paro_attn_workspace(d, grad), paro.PARO_EINVAL, text)
    refused(lambda: paro.paro_attn(d, P, P, P, 0, 0, 0, P, P, P, P, P, ROOM), paro.PARO_EINVAL, text)
    refused(lambda: paro.paro_attn_grad(d, P, P, P, P, P, P, 0, 0, 0, P, P, P, P, P, P, P, ROOM), paro.PARO_EINVAL, text)


def test_refuses_pointers():
    d = paro.make_attn(**ATTN)
    for which, name in enumerate(NAMES):
        args = [P] * len(NAMES)
        args[which] = P + 1
        refused(lambda: paro.paro_attn(d, *args, P, ROOM), paro.PARO_EALIGN, name)
        args[which] = 0
        if name not in ("q_starts", "k_starts", "k_lens", "stats"):
            refused(lambda: paro.paro_attn(d, *args, P, ROOM), paro.PARO_EINVAL, name)
    for which, name in enumerate(GRAD_NAMES):
        args = [P] * len(GRAD_NAMES)
        args[which] = P + 1
        refused(lambda: paro.paro_attn_grad(d, *args, P, ROOM), paro.PARO_EALIGN, name)
        args[which] = 0
        if name not in ("q_starts", "k_starts", "k_lens", "dtable"):
            refused(lambda: paro.paro_attn_grad(d, *args, P, ROOM), paro.PARO_EINVAL, name)
    room = paro.paro_attn_workspace(d, True)
    for ws, size, code in ((0, room, paro.PARO_EINVAL), (P + 8, room, paro.PARO_EALIGN), (P, room - 1, paro.PARO_ERANGE), (P, -1, paro.PARO_ERANGE)):
        refused(lambda: paro.paro_attn_grad(d, *[P] * 15, ws, size), code, "workspace")
    long = paro.make_attn(**{**ATTN, "len_q": 1, "len_k": 10000})
    room = paro.paro_attn_workspace(long, False)
    assert room > 0
    refused(lambda: paro.paro_attn(long, *[P] * 10, P, room - 1), paro.PARO_ERANGE, "workspace")
    assert paro._lib.paro_attn(None, *[P] * 11, 0, 0) == paro.PARO_EINVAL and paro._lib.paro_attn_workspace(None, 0) == paro.PARO_EINVAL
    assert paro._lib.paro_attn_grad(None, *[P] * 16, 0, 0) == paro.PARO_EINVAL


def test_refuses_more_than_a_launch_takes():
    """Launches count their threads in 32 bits."""
    room = 2**62
    for change in (dict(batch=2**17, heads=256, kv_heads=256, head_dim=8, len_q=60, len_k=60), dict(batch=2**17, heads=128, kv_heads=128, head_dim=8, len_q=1, len_k=60),
                   dict(batch=2**20, heads=1, kv_heads=1, head_dim=9, len_q=1000, len_k=1000)):
        d = paro.make_attn(**{**ATTN, "buckets": 0, **change})
        refused(lambda: paro.paro_attn(d, P, P, P, 0, 0, 0, 0, 0, P, P, P, room), paro.PARO_ERANGE, "a launch")
        refused(lambda: paro.paro_attn_grad(d, P, P, P, P, P, P, 0, 0, 0, 0, 0, P, P, P, 0, P, room), paro.PARO_ERANGE, "a launch")


def test_rows_on_sixteen_bytes_lie_there():
    """Where a head and its distances are whole pieces, the arrays that go to shared memory as they are lie on 16 bytes; others are copied."""
    d = paro.make_attn(**{**ATTN, "buckets": 0})
    for which, name in enumerate(("q", "k", "v")):
        args = [P] * 3
        args[which] = P + 8
        if name != "q":
            refused(lambda: paro.paro_attn(d, *args, 0, 0, 0, 0, 0, P, P, P, ROOM), paro.PARO_EALIGN, "16-byte")
        refused(lambda: paro.paro_attn_grad(d, P, *args, P, P, 0, 0, 0, 0, 0, P, P, P, 0, P, ROOM), paro.PARO_EALIGN, "16-byte")
    refused(lambda: paro.paro_attn_grad(d, P + 2, P, P, P, P, P, 0, 0, 0, 0, 0, P, P, P, 0, P, ROOM), paro.PARO_EALIGN, "16-byte")
    whole, odd = (paro.make_attn(**{**ATTN, **x}) for x in (dict(head_dim=72), dict(head_dim=70)))
    copy_k, copy_q = (-(-2 * 100 * heads * 72 * 2 // 256) * 256 for heads in (2, 4))
    assert paro.paro_attn_workspace(whole, False) == 0 and paro.paro_attn_workspace(odd, False) == 2 * copy_k
    assert paro.paro_attn_workspace(odd, True) == paro.paro_attn_workspace(whole, True) + 2 * copy_k + 2 * copy_q
    apart = paro.make_attn(**{**ATTN, "ld_k": 131})                      # one of the four
    assert paro.paro_attn_workspace(apart, False) == -(-2 * 100 * 2 * 64 * 2 // 256) * 256
    few = paro.make_attn(**{**ATTN, "head_dim": 70, "len_q": 3})         # few queries take rows as they lie
    assert paro.paro_attn_workspace(few, False) == 0


def test_nothing_to_do_needs_no_arrays():
    for change in (dict(batch=0), dict(len_q=0)):
        d = paro.make_attn(**{**ATTN, **change})
        paro.paro_attn(d, *[0] * 10, 0, 0)
    d = paro.make_attn(**{**ATTN, "batch": 0})
    paro.paro_attn_grad(d, *[0] * 15, 0, 0)


def test_defaults():
    d = paro.make_attn(batch=3, heads=6, head_dim=16, len_q=7, dtype=paro.PARO_F16)
    assert (d.kv_heads, d.len_k, d.scale, d.window, d.sinks, d.buckets) == (6, 7, 0.25, 0, 0, 0)
    assert paro.make_attn(batch=3, heads=6, head_dim=16, len_q=7, len_k=0, dtype=paro.PARO_F16).len_k == 0


def test_workspaces():
    """Forward: only where few blocks look at many keys; backward: a few words a row and head, and the sums of what is shared out."""
    for heads, len_q, len_k, window, sinks in itertools.product((1, 32), (1, 16, 17, 4096), (0, 1, 4096, 100_000), (0, 1, 1024), (0, 4, 5000)):
        d = paro.make_attn(batch=2, heads=heads, head_dim=128, len_q=len_q, len_k=len_k, dtype=paro.PARO_F16, window=window, sinks=sinks)
        some = heads == 1 or len_q < 4096                              # of 17 queries and more: blocks for less than the chip, and 2048 keys that they see
        most = 200 << 20 if len_q <= 16 else 512 * 128 * 130 * 4 if some and len_k >= 2048 and (window == 0 or window + 128 + sinks >= 2048) else 0
        assert paro.paro_attn_workspace(d, False) <= most
        small = 2 * len_q * heads * 8
        assert small <= paro.paro_attn_workspace(d, True) <= small + (400 << 20)


@pytest.mark.parametrize("buckets", list(range(1, 70)) + [128, 255, 256])
def test_first_distances(buckets):
    """The smallest whole number d with (d / h)^m >= (D / h)^k, in whole numbers."""
    h = (buckets + 1) // 2
    m = buckets - h
    for far in (h, h + 1, 128, 2000, 2**30 - 1):
        if far < h:
            refused(lambda: paro.paro_rel_buckets(buckets, far), paro.PARO_EINVAL, "max_distance")
            continue
        first = paro.paro_rel_buckets(buckets, far)
        assert first[:h] == list(range(h))
        for k, d in enumerate(first[h:]):
            reaches = lambda x: Fraction(x, h) ** m >= Fraction(far, h) ** k     # noqa: E731
            assert reaches(d) and not (d and reaches(d - 1)), (k, d)


def test_first_distances_refused():
    for buckets, far in ((0, 5), (-1, 5), (257, 1000), (8, 3), (8, 2**30), (8, -1)):
        refused(lambda: paro.paro_rel_buckets(buckets, far), paro.PARO_EINVAL, "must be in")
    assert paro._lib.paro_rel_buckets(8, 100, None) == paro.PARO_EINVAL


def outcome(call):
    try:
        return "returned", call()
    except paro.ParoError as e:
        return "refused", e.code, str(e)
    except Exception as e:
        return "raised", type(e)


CALLS = {"paro_attn": [paro.make_attn(**ATTN)] + [P] * 9 + [P + 1, P, ROOM, 0],
         "paro_attn_grad": [paro.make_attn(**ATTN)] + [P] * 14 + [P + 1, P, ROOM, 0]}


@pytest.mark.skipif(__import__("torch").cuda.is_available(), reason="calls with made-up addresses are for machines without a GPU")
@pytest.mark.parametrize("name", list(CALLS))
def test_extension_reads_what_ctypes_reads(name):
    """Each argument replaced by others, of its kind and not: returned, refused or raised alike."""
    fast, slow, args = getattr(paro, name), paro._through_ctypes[name], CALLS[name]
    assert fast is not slow and outcome(lambda: fast(*args))[0] == "refused" and outcome(lambda: fast(*args)) == outcome(lambda: slow(*args))
    for k in range(len(args)):
        for other in (0, 1, -1, 2**31, 2**63, -2**63, 2**64, 0.5, None, "x", True, [], P + 1, paro.make_gated(n=1, dim=1, hidden=1, dtype=0)):
            changed = args[:k] + [other] + args[k + 1:]
            a, b = outcome(lambda: fast(*changed)), outcome(lambda: slow(*changed))
            assert a == b or (a[0] == b[0] == "raised"), (k, other, a, b)
    for few in range(len(args) - 1):
        a, b = outcome(lambda: fast(*args[:few])), outcome(lambda: slow(*args[:few]))
        assert a == b, (few, a, b)
