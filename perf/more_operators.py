"""The attention half of a language model's block, as cases that can be timed and compared: attention with a sliding window and a few first
tokens that stay visible, over prompts and training batches, for new tokens over a cache, and its gradient; and the learned relative position bias
by buckets that is added to its scores, with the gradient of its table.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` makes one pass - in plain torch operations,
held in 32 bits and rounded once at the end, or, where `own` is true, through the library's entry points - and `exact` says in 64 bits what
that pass returns.  Heads and lengths are those of the models that this repository is benchmarked and tested on (12 heads of 64 over 1024
tokens; 32 heads of 128), or lie around them.

The last query of a sequence stands where its last key stands; with p its place, a query sees key j where
    0 <= j <= p  and  (window == 0  or  p - j < window  or  j < sinks)
and its score is  scale * q . k + table[bucket of p - j][head].

Fields of a case
  op      "attn"        out, and for the backward pass the largest score of each row and the log of its sum
          "attn_grad"   gradients of q, k, v, and of the table where there is one
          "attn_new"    out of n new tokens of each sequence over a cache
  batch   sequences;  n: queries of the longest;  m: keys of the longest, and of "attn_new" the cache's room for a sequence
  ragged  sequences are of different lengths (of "attn": packed one behind the other)
  heads, kv, hd         query heads, key heads, elements of a head
  window, sinks         in tokens; window 0: none
  buckets               rows of the table, 0: no bias;  table: dtype of it and of its gradient
  dtype   of activations;  pad: elements that a token's row of them is longer than its heads
  layout  of a cache: "rows" (heads side by side for each token) or "heads" (tokens one behind the other for each head)
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
CODE = {"bf16": 0, "f32": 1, "f16": 2}        # the library's dtype codes
SCORES_LARGEST = 32 * 8192 * 8192             # of attn_grad_large: scores over all heads
CACHE_LARGEST = 4 * 100000 * 8 * 128          # elements of attn_new_long's keys


def listed():
    return [
        # One new token of a single served sequence: latency alone.
        dict(name="attn_new_one", op="attn_new", batch=1, n=1, m=700, ragged=False, heads=12, kv=12, hd=64, window=0, sinks=0, buckets=0,
             dtype="bf16", pad=0, layout="rows"),
        # A batch of served sequences whose model looks back 1024 tokens.
        dict(name="attn_new_window", op="attn_new", batch=32, n=1, m=4096, ragged=True, heads=32, kv=8, hd=128, window=1024, sinks=4, buckets=0,
             dtype="bf16", pad=0, layout="rows"),
        # Few long documents: reading the cache is all.
        dict(name="attn_new_long", op="attn_new", batch=4, n=1, m=100000, ragged=True, heads=32, kv=8, hd=128, window=0, sinks=0, buckets=0,
             dtype="bf16", pad=0, layout="rows"),
        # Five drafted tokens a sequence, looked at together, with the bias; a cache with a head's tokens side by side.
        dict(name="attn_new_drafts", op="attn_new", batch=7, n=5, m=1531, ragged=True, heads=12, kv=12, hd=64, window=512, sinks=4, buckets=32,
             table="f32", dtype="f16", pad=0, layout="heads"),
        # A micro-batch of the GPT-2-shaped model, forward, with the bias.
        dict(name="attn_gpt2_bias", op="attn", batch=8, n=1024, m=1024, ragged=False, heads=12, kv=12, hd=64, window=0, sinks=0, buckets=32,
             table="f32", dtype="bf16", pad=0),
        # Sequences of different lengths, packed, four query heads to a key head.
        dict(name="attn_window", op="attn", batch=8, n=2048, m=2048, ragged=True, heads=32, kv=8, hd=128, window=1024, sinks=4, buckets=0,
             dtype="bf16", pad=0),
        # Odd in every size, fp16, padded rows.
        dict(name="attn_odd", op="attn", batch=3, n=1999, m=1999, ragged=True, heads=10, kv=5, hd=77, window=333, sinks=7, buckets=17,
             table="f16", dtype="f16", pad=3),
        # A long training sequence, forward.
        dict(name="attn_long", op="attn", batch=1, n=8192, m=8192, ragged=False, heads=32, kv=32, hd=128, window=4096, sinks=16, buckets=0,
             dtype="bf16", pad=0),
        # Backward of the same four.
        dict(name="attn_grad_gpt2_bias", op="attn_grad", batch=8, n=1024, m=1024, ragged=False, heads=12, kv=12, hd=64, window=0, sinks=0, buckets=32,
             table="f32", dtype="bf16", pad=0),
        dict(name="attn_grad_window", op="attn_grad", batch=8, n=2048, m=2048, ragged=True, heads=32, kv=8, hd=128, window=1024, sinks=4, buckets=0,
             dtype="bf16", pad=0),
        dict(name="attn_grad_odd", op="attn_grad", batch=3, n=1999, m=1999, ragged=True, heads=10, kv=5, hd=77, window=333, sinks=7, buckets=17,
             table="f16", dtype="f16", pad=3),
        # The largest: every earlier token is seen.
        dict(name="attn_grad_large", op="attn_grad", batch=1, n=8192, m=8192, ragged=False, heads=32, kv=32, hd=128, window=0, sinks=0, buckets=0,
             dtype="bf16", pad=0),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no costlier than the largest listed."""
    op = rng.choice(["attn", "attn_grad", "attn_new"])
    kv, group = _log(rng, 1, 32), rng.choice([1, 1, 2, 4, 8])
    heads = kv * group if kv * group <= 64 else kv
    hd = rng.choice([64, 128, 64, 128, 32, 80, 96, _log(rng, 16, 128), _log(rng, 16, 128)])
    dtype, pad = rng.choice(["bf16", "bf16", "f16"]), rng.choice([0, 0, 0, 8, 5])
    c = dict(op=op, heads=heads, kv=kv, hd=hd, dtype=dtype, pad=pad, ragged=rng.random() < 0.6)
    if op == "attn_new":
        n, m = rng.choice([1, 1, 1, rng.randint(2, 16)]), _log(rng, 16, 131072)
        batch = _log(rng, 1, max(1, min(64, CACHE_LARGEST // (m * kv * hd))))
        c.update(batch=batch, n=n, m=min(m, max(16, CACHE_LARGEST // (kv * hd))), layout=rng.choice(["rows", "rows", "heads"]))
    else:
        n = min(_log(rng, 1, 8192), int(math.sqrt(SCORES_LARGEST / 2 / heads)))
        c.update(n=n, m=n, batch=_log(rng, 1, max(1, min(32, SCORES_LARGEST // 2 // (heads * n * n)))))
    window = 0 if rng.random() < 0.35 else _log(rng, 1, max(2, c["m"]))
    c.update(window=window, sinks=rng.choice([0, 1, 4, _log(rng, 1, 200)]) if window else 0)
    buckets = 0 if rng.random() < 0.5 else _log(rng, 2, 128)
    return dict(c, buckets=buckets, **(dict(table=rng.choice(["f32", dtype])) if buckets else {}))


# ------------------------------------------------------------------------------ inputs
def _lengths(c):
    """Queries and keys of each sequence: the case's, whatever the seed."""
    batch, n, m = c["batch"], c["n"], c["m"]
    rng = random.Random(batch * 1000003 + m * 31 + n)
    if c["op"] == "attn_new":
        keys = [rng.randint(max(n, m // 2), max(n, m)) if c["ragged"] and b else max(n, m) for b in range(batch)]
        return [n] * batch, keys
    keys = [rng.randint((n + 1) // 2, n) if c["ragged"] and b else n for b in range(batch)]
    return keys, keys


def _rows(n, heads, hd, pad, dtype):
    """n tokens' rows of heads side by side, each `pad` elements from the next."""
    return torch.empty(n, heads * hd + pad, dtype=TORCH[dtype], device=DEV)[:, :heads * hd].unflatten(1, (heads, hd))


def _filled(g, t, size):
    return t.copy_(torch.randn(t.shape, generator=g, device=DEV).mul_(size))


def _first_distances(buckets, far=128):
    """The first distance of each bucket: half of the buckets take a distance each, the others grow by a ratio up to `far`."""
    single = (buckets + 1) // 2
    far = max(far, 2 * single)
    more = buckets - single
    grown = [math.ceil(single * (far / single) ** (k / more) - 1e-9) for k in range(more)] if more else []
    return list(range(single)) + grown


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    c, op = dict(case), case["op"]
    batch, heads, kv, hd, dtype, pad = c["batch"], c["heads"], c["kv"], c["hd"], c["dtype"], c["pad"]
    nq, nk = _lengths(c)
    s = {"case": c, "scale": 1 / math.sqrt(hd)}
    to = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)                # noqa: E731
    starts = np.concatenate([[0], np.cumsum(nq)]).tolist()
    s["rows"], s["nq"], s["nk"], s["q_starts"] = starts[-1], to(nq), to(nk), to(starts)
    s["q"] = _filled(g, _rows(starts[-1], heads, hd, pad, dtype), 1.5)
    if op == "attn_new":                       # the cache behind a sequence's end holds what was there before
        m = max(nk)
        if c["layout"] == "rows":
            s["k"], s["v"] = (_filled(g, _rows(batch * m, kv, hd, 0, dtype), 1.0) for _ in range(2))
            s["k_starts"] = to([b * m for b in range(batch)])
        else:                                  # a row is hd long; a head's rows lie m rows from the next one's
            s["k"], s["v"] = (_filled(g, torch.empty(batch, kv, m, hd, dtype=TORCH[dtype], device=DEV), 1.0) for _ in range(2))
            s["k_starts"] = to([b * kv * m for b in range(batch)])
        s["k_lens"] = to(nk)
    else:
        s["k"], s["v"] = (_filled(g, _rows(starts[-1], kv, hd, pad, dtype), 1.0) for _ in range(2))
        s["k_starts"] = s["q_starts"]
    s["table"] = _filled(g, torch.empty(c["buckets"], heads, dtype=TORCH[c["table"]], device=DEV), 1.0) if c["buckets"] else None
    s["first"] = to(_first_distances(c["buckets"])) if c["buckets"] else None
    s["out"] = _rows(starts[-1], heads, hd, pad, dtype)
    s["stats"] = torch.empty(starts[-1], heads, 2, device=DEV)
    if op == "attn_grad":
        out, stats = _plain_attn(s)
        s["out"].copy_(out)
        s["stats"].copy_(stats)
        s["dout"] = _filled(g, _rows(starts[-1], heads, hd, pad, dtype), 0.1 * (1024 if dtype == "f16" else 1))       # fp16: with loss scaling
        s["dq"], s["dk"], s["dv"] = (_rows(starts[-1], h, hd, pad, dtype) for h in (heads, kv, kv))
        s["dtable"] = torch.empty_like(s["table"]) if c["buckets"] else None
    return s


# ------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _own(s)
    if s["case"]["op"] == "attn_grad":
        return _plain_grad(s)
    out, stats = _plain_attn(s)
    return [out] if s["case"]["op"] == "attn_new" else [out, stats]


def _dense(rows, starts, lengths, most):
    """[batch, heads, most, hd] of packed rows, zeros behind a sequence's end."""
    at = torch.arange(most, device=DEV)
    held = at < lengths[:, None]
    return torch.where(held[:, :, None, None], rows[torch.where(held, starts[:, None] + at, 0).long()].float(), 0.0).transpose(1, 2)


def _keys(s, t):
    c = s["case"]
    if c["op"] != "attn_new":
        return _dense(t, s["k_starts"][:-1], s["nk"], c["m"])
    t = t if c["layout"] == "heads" else t.unflatten(0, (c["batch"], -1)).transpose(1, 2)
    held = torch.arange(t.shape[2], device=DEV) < s["nk"][:, None]
    return torch.where(held[:, None, :, None], t.float(), 0.0)


def _scores(s, q, k):
    """Scores of every query head [batch, heads, n, m], -inf where a key is not seen; the distances [batch, n, m]."""
    c = s["case"]
    batch, heads, n, hd = q.shape
    kv, m = k.shape[1], k.shape[2]
    z = (q.reshape(batch, kv, heads // kv * n, hd) @ k.transpose(2, 3)).view(batch, heads, n, m).mul_(s["scale"])
    i, j = torch.arange(n, device=DEV)[:, None], torch.arange(m, device=DEV)
    nq, nk = s["nq"][:, None, None], s["nk"][:, None, None]
    far = (nk - nq) + i - j
    seen = (far >= 0) & (j < nk) & (i < nq)
    if c["window"]:
        seen &= (far < c["window"]) | (j < c["sinks"])
    if c["buckets"]:
        of = (s["first"] <= torch.arange(max(1, m), device=DEV)[:, None]).sum(dim=1) - 1       # bucket of each distance
        by_distance = s["table"].float()[of].t().contiguous()                                 # [heads, distances]
        z += by_distance[:, far.clamp(0, m - 1)].transpose(0, 1)
    return z.masked_fill_(~seen[:, None], -math.inf), far


def _plain_attn(s):
    c, dt = s["case"], TORCH[s["case"]["dtype"]]
    q = _dense(s["q"], s["q_starts"][:-1], s["nq"], c["n"])
    k, v = _keys(s, s["k"]), _keys(s, s["v"])
    z, _ = _scores(s, q, k)
    most = z.amax(dim=3, keepdim=True)
    p = torch.exp(z - most.masked_fill(most == -math.inf, 0.0))
    total = p.sum(dim=3, keepdim=True)
    p /= torch.where(total > 0, total, 1.0)
    batch, heads, n, m = p.shape
    kv = k.shape[1]
    out = (p.view(batch, kv, heads // kv * n, m) @ v).view(batch, heads, n, -1)
    held = torch.arange(n, device=DEV) < s["nq"][:, None]
    stats = torch.cat([most, torch.where(total > 0, torch.log(total), 0.0)], dim=3)
    return out.transpose(1, 2)[held].to(dt), stats.transpose(1, 2)[held]


def _plain_grad(s):
    c, dt = s["case"], TORCH[s["case"]["dtype"]]
    starts, nq, n = s["q_starts"][:-1], s["nq"], c["n"]
    q, dout, out = (_dense(s[x], starts, nq, n) for x in ("q", "dout", "out"))
    stats = _dense(s["stats"], starts, nq, n)
    k, v = _keys(s, s["k"]), _keys(s, s["v"])
    z, far = _scores(s, q, k)
    batch, heads, n, m = z.shape
    kv = k.shape[1]
    group = lambda t: t.reshape(batch, kv, heads // kv * n, t.shape[3])         # noqa: E731
    p = torch.exp(z - stats[..., :1] - stats[..., 1:])
    dv = group(p).transpose(2, 3).contiguous() @ group(dout)
    dp = (group(dout) @ v.transpose(2, 3)).view(batch, heads, n, m)
    dz = p.mul_(dp.sub_((dout * out).sum(dim=3, keepdim=True)))
    dq = (group(dz) @ k).view(batch, heads, n, -1) * s["scale"]
    dk = group(dz).transpose(2, 3).contiguous() @ group(q) * s["scale"]
    held = torch.arange(n, device=DEV) < nq[:, None]
    grads = [t.transpose(1, 2)[held].to(dt) for t in (dq, dk, dv)]
    if c["buckets"]:
        # sums along diagonals first (place i, j of a row goes to i - j + m - 1), then over the distances of a bucket
        wide = torch.nn.functional.pad(dz.flip(3), (0, n)).flatten(2)[:, :, :n * (m + n - 1)]
        along = wide.view(batch, heads, n, m + n - 1).sum(dim=2, dtype=torch.float64)
        at = (s["nk"] - nq)[:, None] + torch.arange(n + m - 1, device=DEV) - (m - 1)
        of = (s["first"] <= at.clamp(min=0)[..., None]).sum(dim=2) - 1
        sums = torch.zeros(c["buckets"], heads, dtype=torch.float64, device=DEV)
        sums.index_add_(0, of.flatten(), torch.where(at[:, None] >= 0, along, 0.0).transpose(1, 2).flatten(0, 1))
        grads.append(sums.to(TORCH[c["table"]]))
    return grads


def _own(s):
    import paper_2310_06003_amd as paro
    c, op = s["case"], s["case"]["op"]
    stream = torch.cuda.current_stream().cuda_stream
    address = lambda t: 0 if t is None else t.data_ptr()                         # noqa: E731
    heads_first = op == "attn_new" and c["layout"] == "heads"
    ragged = op != "attn_new" and c["ragged"]
    ld = lambda t: t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]    # noqa: E731
    room = s["k"].shape[2] if heads_first else s["k"].shape[0] // c["batch"] if op == "attn_new" else c["m"]
    d = paro.make_attn(batch=c["batch"], heads=c["heads"], kv_heads=c["kv"], head_dim=c["hd"], len_q=c["n"], len_k=room,
                       rows_q=s["rows"], rows_k=s["k"].numel() // c["hd"] if heads_first else s["k"].shape[0],
                       ld_q=ld(s["q"]), ld_k=c["hd"] if heads_first else ld(s["k"]), ld_v=c["hd"] if heads_first else ld(s["v"]), ld_out=ld(s["out"]),
                       head_k=room * c["hd"] if heads_first else 0, head_v=room * c["hd"] if heads_first else 0,
                       window=c["window"], sinks=c["sinks"], scale=s["scale"], dtype=CODE[c["dtype"]], buckets=c["buckets"],
                       table_dtype=CODE[c["table"]] if c["buckets"] else 0)
    if "work" not in s:                        # a program keeps it from call to call
        s["work"] = torch.empty(paro.paro_attn_workspace(d, op == "attn_grad"), dtype=torch.uint8, device=DEV)
    q_starts = s["q_starts"].data_ptr() if ragged else 0
    k_starts = s["k_starts"].data_ptr() if ragged or heads_first else 0
    k_lens = address(s.get("k_lens"))
    q, k, v, table, first = s["q"].data_ptr(), s["k"].data_ptr(), s["v"].data_ptr(), address(s["table"]), address(s["first"])
    work, size = s["work"].data_ptr(), s["work"].numel()
    if op == "attn_grad":
        paro.paro_attn_grad(d, s["dout"].data_ptr(), q, k, v, s["out"].data_ptr(), s["stats"].data_ptr(), q_starts, k_starts, k_lens, table, first,
                            s["dq"].data_ptr(), s["dk"].data_ptr(), s["dv"].data_ptr(), address(s["dtable"]), work, size, stream)
        return [s["dq"], s["dk"], s["dv"]] + ([s["dtable"]] if c["buckets"] else [])
    paro.paro_attn(d, q, k, v, q_starts, k_starts, k_lens, table, first, s["out"].data_ptr(), 0 if op == "attn_new" else s["stats"].data_ptr(),
                   work, size, stream)
    return [s["out"]] if op == "attn_new" else [s["out"], s["stats"]]


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """Sequence by sequence and key head by key head, without padding."""
    s, c, op = prepare(case, seed), case, case["op"]
    lengths, f64 = list(zip(*_lengths(c))), torch.float64
    group = c["heads"] // c["kv"]
    outs = [torch.zeros(t.shape, dtype=f64, device=DEV) for t in ((s["out"], s["stats"]) if op != "attn_grad" else (s["dq"], s["dk"], s["dv"]))]
    dtable = torch.zeros(c["buckets"], c["heads"], dtype=f64, device=DEV)
    at = 0
    for b, (n, m) in enumerate(lengths):
        rows = slice(at, at + n)
        at += n
        place = torch.arange(m - n, m, device=DEV)[:, None]
        far = place - torch.arange(m, device=DEV)
        hidden = far < 0
        if c["window"]:
            hidden |= (far >= c["window"]) & (torch.arange(m, device=DEV) >= c["sinks"])
        if c["buckets"]:
            of = torch.searchsorted(s["first"], torch.arange(max(m, 1), device=DEV, dtype=torch.int32), right=True) - 1
        for h in range(c["kv"]):
            k, v = ((s[x][b, h] if c.get("layout") == "heads" else s[x].unflatten(0, (c["batch"], -1))[b, :, h])[:m].double() if op == "attn_new"
                    else s[x][rows, h].double() for x in ("k", "v"))
            for e in range(h * group, (h + 1) * group):
                q = s["q"][rows, e].double()
                z = (q @ k.t()) * s["scale"]
                if c["buckets"]:
                    z += s["table"][:, e].double()[of][far.clamp(min=0)]
                z.masked_fill_(hidden, -math.inf)
                if op != "attn_grad":
                    most = z.amax(dim=1)
                    outs[0][rows, e] = torch.softmax(z, dim=1) @ v
                    outs[1][rows, e, 0] = most
                    outs[1][rows, e, 1] = torch.logsumexp(z - most[:, None], dim=1)
                    continue
                p = torch.exp(z - s["stats"][rows, e].double().sum(dim=1, keepdim=True))
                dout = s["dout"][rows, e].double()
                dz = p * (dout @ v.t() - (dout * s["out"][rows, e].double()).sum(dim=1, keepdim=True))
                outs[0][rows, e] = dz @ k * s["scale"]
                outs[1][rows, h] += dz.t() @ q * s["scale"]
                outs[2][rows, h] += p.t() @ dout
                if c["buckets"]:
                    by_distance = torch.zeros(m + 1, dtype=f64, device=DEV).index_add_(0, torch.where(hidden, m, far).flatten(), dz.flatten())
                    dtable[:, e].index_add_(0, of, by_distance[:-1])
    return outs[:1] if op == "attn_new" else outs + [dtable] if op == "attn_grad" and c["buckets"] else outs


# ------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    """Keys and values that some query sees, queries and gradients once; the products over the pairs that see each other."""
    c, e = case, SIZE[case["dtype"]]
    window, sinks, pairs, keys, queries = c["window"], c["sinks"], 0, 0, 0
    for n, m in zip(*_lengths(c)):
        p = np.arange(m - n, m, dtype=np.int64) + 1                          # keys up to a query's own place
        queries += n
        if window:
            pairs += int((np.minimum(p, window) + np.clip(p - window, 0, sinks)).sum())
            before = max(0, m - n + 1 - window)                              # keys in front of the first query's window
            keys += m - before + min(before, sinks)
        else:
            pairs += int(p.sum())
            keys += m
    of_q, of_k = queries * c["heads"] * c["hd"] * e, keys * c["kv"] * c["hd"] * e
    table = c["buckets"] * (c["heads"] * SIZE[c["table"]] + 4) if c["buckets"] else 0
    if c["op"] == "attn_grad":
        return {"bytes": 4 * of_q + 4 * of_k + 8 * queries * c["heads"] + 2 * table, "flops": 10 * pairs * c["heads"] * c["hd"]}
    return {"bytes": 2 * of_q + 2 * of_k + (8 * queries * c["heads"] if c["op"] == "attn" else 0) + table, "flops": 4 * pairs * c["heads"] * c["hd"]}
