"""What the tests of the attention share: sequences of any lengths in any layout, the definition in 64 bits with what fp32 sums and the roundings of
16-bit products may add to it, and the calls.  Holds no arithmetic of the library's."""
import math

import torch

from operators_ref import DEV, EPS32, HALF_ULP, TORCH, check, code, rng, rounding, stream, workspace

F64 = torch.float64


def first_distances(buckets, far):
    single = (buckets + 1) // 2
    more = buckets - single
    return list(range(single)) + [math.ceil(single * (far / single) ** (k / more) - 1e-9) for k in range(more)]


def check_rounded(got, ref, bound, dtype, what):
    """fp16 rounds what lies from 65520 = 65504 + half a step on to infinity: where the value may lie there, infinity is its rounding."""
    got = got.detach().cpu().double()
    if dtype == "f16":
        got = torch.where(got.isinf() & (got.sign() == ref.sign()) & (ref.abs() + bound >= 65520), ref, got)
    check(got, ref, bound, what)


class Array:
    """Rows of heads somewhere in a buffer full of `fill`: packed, `pad` elements apart, from an odd element on where pad is odd; or head by head (planes)."""

    def __init__(self, rows, heads, hd, pad, dtype, planes=False, fill=float("nan")):
        self.whole = torch.full((rows * heads * hd + rows * pad + 64 + 2 * hd,), fill, dtype=TORCH[dtype], device=DEV)
        at = 1 if pad % 2 else 0
        if planes:
            self.ld, self.head = hd, rows * hd + pad
            self.whole = torch.full((heads * self.head + 64,), fill, dtype=TORCH[dtype], device=DEV)
        else:
            self.ld, self.head = heads * hd + pad, hd
        self.view = self.whole[at:].as_strided((rows, heads, hd), (self.ld, self.head, 1))
        self.mask = torch.zeros_like(self.whole, dtype=torch.bool)
        self.held = self.mask[at:].as_strided((rows, heads, hd), (self.ld, self.head, 1))

    def put(self, rows, values):
        self.view[rows] = values.to(self.view.dtype).to(DEV)

    def untouched(self, fill, what):
        """Nothing but what the sequences hold was written."""
        rest = self.whole[~self.mask]
        assert bool((rest.isnan() if fill != fill else rest == fill).all()), f"{what}: wrote beside its rows"


class Case:
    """lengths: (queries, keys) of each sequence.  layout: "packed" (with gaps between sequences), "dense" (padded to the longest: queries by q_starts where
    they differ), "planes" (as packed, keys and values head by head).  shared: queries and keys have the same rows (training)."""

    def __init__(self, paro, lengths, heads=2, kv=0, hd=64, dtype="bf16", window=0, sinks=0, buckets=0, far=40, table="f32", pad=0, layout="packed",
                 seed=1, size=1.0, use_lens=False, spread=1.0):
        g = rng(seed)
        kv = kv or heads
        self.paro, self.lengths, self.heads, self.kv, self.hd, self.dtype = paro, lengths, heads, kv, hd, dtype
        self.window, self.sinks, self.buckets, self.table_dtype, self.pad = window, sinks, buckets, table, pad
        self.scale, self.batch = 0.9 / math.sqrt(hd), len(lengths)
        len_q, len_k = (max(x[i] for x in lengths) for i in (0, 1))
        gap = 0 if layout == "dense" else 3
        self.q_at, self.k_at, at_q, at_k = [], [], gap, gap
        for nq, nk in lengths:
            self.q_at.append(at_q)
            self.k_at.append(at_k)
            at_q += len_q if layout == "dense" else nq
            at_k += len_k if layout == "dense" else nk + (gap if use_lens else 0)
        self.rows_q, self.rows_k = at_q + gap, at_k + gap
        to = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)           # noqa: E731
        if layout == "dense":
            assert all(nq == len_q for nq, _ in lengths)
            self.q_starts = self.k_starts = None
            self.k_lens = to([nk for _, nk in lengths]) if use_lens or any(nk != len_k for _, nk in lengths) else None
        else:
            self.q_starts = to(self.q_at + [at_q])
            self.k_lens = to([nk for _, nk in lengths]) if use_lens else None
            self.k_starts = to(self.k_at + ([] if use_lens else [at_k]))
        self.len_q, self.len_k = len_q, len_k
        planes = layout == "planes"
        n = max(self.rows_q, 1), max(self.rows_k, 1)
        self.q, self.dout, self.out, self.dq = (Array(n[0], heads, hd, pad, dtype, fill=f) for f in (float("nan"), float("nan"), 5.0, 5.0))
        self.k, self.v, self.dk, self.dv = (Array(n[1], kv, hd, pad, dtype, planes, fill=f) for f in (float("nan"), float("nan"), 5.0, 5.0))
        for b, (nq, nk) in enumerate(lengths):
            rq, rk = slice(self.q_at[b], self.q_at[b] + nq), slice(self.k_at[b], self.k_at[b] + nk)
            self.q.put(rq, torch.randn(nq, heads, hd, generator=g) * size)
            most = torch.finfo(TORCH[dtype]).max              # no infinities: the definition below would form their multiples by zero
            self.dout.put(rq, (torch.randn(nq, heads, hd, generator=g) * spread).clamp(-most, most))
            self.k.put(rk, torch.randn(nk, kv, hd, generator=g))
            self.v.put(rk, torch.randn(nk, kv, hd, generator=g))
            for x in (self.out, self.dq):
                x.held[rq] = True
            for x in (self.dk, self.dv):
                x.held[rk] = True
        self.stats = torch.full((n[0], heads, 2), 5.0, device=DEV)
        self.table = self.first = self.dtable = None
        if buckets:
            self.table = torch.randn(buckets, heads, generator=g).to(TORCH[table]).to(DEV)
            self.first_list = first_distances(buckets, max(far, (buckets + 1) // 2))
            self.first = to(self.first_list)
            self.dtable = torch.full_like(self.table, 7.0)

    def plan(self, **change):
        p = dict(batch=self.batch, heads=self.heads, kv_heads=self.kv, head_dim=self.hd, len_q=self.len_q, len_k=self.len_k, rows_q=self.rows_q, rows_k=self.rows_k,
                 ld_q=self.q.ld, ld_k=self.k.ld, ld_v=self.v.ld, ld_out=self.out.ld, head_k=self.k.head, head_v=self.v.head, window=self.window, sinks=self.sinks,
                 scale=self.scale, dtype=code(self.paro, self.dtype), buckets=self.buckets, table_dtype=code(self.paro, self.table_dtype))
        return self.paro.make_attn(**{**p, **change})

    @staticmethod
    def address(t):
        return 0 if t is None else t.data_ptr()

    def sequences(self):
        return [self.address(t) for t in (self.q_starts, self.k_starts, self.k_lens, self.table, self.first)]

    def forward(self, stats=True):
        d = self.plan()
        ws = workspace(max(16, self.paro.paro_attn_workspace(d, False)))
        self.paro.paro_attn(d, *(x.view.data_ptr() for x in (self.q, self.k, self.v)), *self.sequences(), self.out.view.data_ptr(),
                            self.stats.data_ptr() if stats else 0, ws.data_ptr(), ws.numel(), stream())

    def backward(self, want_table=True):
        d = self.plan()
        ws = workspace(max(16, self.paro.paro_attn_workspace(d, True)))
        self.paro.paro_attn_grad(d, self.dout.view.data_ptr(), *(x.view.data_ptr() for x in (self.q, self.k, self.v)), self.out.view.data_ptr(),
                                 self.stats.data_ptr(), *self.sequences(), *(x.view.data_ptr() for x in (self.dq, self.dk, self.dv)),
                                 self.address(self.dtable) if want_table else 0, ws.data_ptr(), ws.numel(), stream())

    # ------------------------------------------------------------------------------ the definition
    def rows_of(self, array, at, n):
        return array.view[at:at + n].double().cpu()

    def pairs(self, nq, nk):
        """Distances, and which pairs see each other."""
        place = torch.arange(nk - nq, nk)[:, None]
        far = place - torch.arange(nk)
        seen = far >= 0
        if self.window:
            seen &= (far < self.window) | (torch.arange(nk) < self.sinks)
        return far, seen

    def scores(self, b, h):
        """Of head h of sequence b: scores with -inf where unseen, a bound on what an fp32 score is off, distances."""
        nq, nk = self.lengths[b]
        q = self.rows_of(self.q, self.q_at[b], nq)[:, h]
        k = self.rows_of(self.k, self.k_at[b], nk)[:, h // (self.heads // self.kv)]
        far, seen = self.pairs(nq, nk)
        s = q @ k.t() * self.scale
        off = 2 * (self.hd + 4) * EPS32 * (q.abs() @ k.abs().t()) * self.scale + 4 * EPS32 * s.abs()
        if self.buckets:
            of = (torch.tensor(self.first_list)[None] <= torch.arange(nk + 1)[:, None]).sum(1) - 1
            bias = self.table[:, h].double().cpu()[of][far.clamp(min=0)]
            s = s + bias
            off = off + 2 * EPS32 * (s.abs().clamp(max=1e39) + bias.abs().clamp(max=1e39))          # of -inf a share is zero, whatever this says
        return s.masked_fill(~seen, -math.inf), off, far, seen

    def check_forward(self, stats=True):
        for b, (nq, nk) in enumerate(self.lengths):
            if nq == 0:
                continue
            out = torch.zeros(nq, self.heads, self.hd, dtype=F64)
            bound = torch.zeros_like(out)
            st, st_bound = torch.zeros(nq, self.heads, 2, dtype=F64), torch.zeros(nq, self.heads, 2, dtype=F64)
            st[..., 0] = -math.inf
            v_all = self.rows_of(self.v, self.k_at[b], nk)
            for h in range(self.heads):
                if nk == 0:
                    continue
                s, off, _far, seen = self.scores(b, h)
                some = (s > -math.inf).any(1)
                most = torch.where(some, s.amax(1), 0.0)
                p = torch.exp(s - most[:, None])
                total = torch.where(some, p.sum(1), 1.0)
                P = p / total[:, None]
                off = torch.where(seen & (s > -math.inf), off, 0.0).amax(1)
                size = torch.where(seen & (s > -math.inf), (s - most[:, None]).abs(), 0.0).amax(1).clamp(max=200)
                # a share: the score's and the largest's error, the argument in powers of two rounded thrice, an exponential of one unit
                share = 2 * off + EPS32 * (6 * size + 6 * most.abs().clamp(max=1e6) * (0 if self.buckets else 1) + 16)
                sums = (nk + 16) * EPS32
                rel = HALF_ULP[self.dtype] + 2 * share + 3 * sums
                floor = 2.0 ** -32 if self.dtype == "f16" else 0.0
                v = v_all[:, h // (self.heads // self.kv)]
                out[:, h] = P @ v
                bound[:, h] = rel[:, None] * (P @ v.abs()) + floor * torch.where(seen, 1.0, 0.0).double() @ v.abs()
                st[:, h, 0] = torch.where(some, most, -math.inf)
                st_bound[:, h, 0] = off + 2 * EPS32 * most.abs()
                st[:, h, 1] = torch.where(some, torch.log(total), 0.0)
                st_bound[:, h, 1] = share + off + sums + 8 * EPS32 * (torch.log(total).abs() + 16)
            got = self.out.view[self.q_at[b]:self.q_at[b] + nq]
            check(got, out, rounding(out, self.dtype, bound), f"out of sequence {b}")
            if stats:
                check(self.stats[self.q_at[b]:self.q_at[b] + nq], st, st_bound, f"stats of sequence {b}")
        self.out.untouched(5.0, "out")

    def set_forward(self):
        """out and stats as the definition has them, rounded: what the gradient is taken from."""
        for b, (nq, nk) in enumerate(self.lengths):
            v = self.rows_of(self.v, self.k_at[b], nk)
            for h in range(self.heads):
                rows = slice(self.q_at[b], self.q_at[b] + nq)
                if nk == 0:
                    self.out.view[rows, h] = 0
                    self.stats[rows, h] = torch.tensor([-math.inf, 0.0], device=DEV)
                    continue
                s, *_ = self.scores(b, h)
                some = (s > -math.inf).any(1)
                most = torch.where(some, s.amax(1), 0.0)
                p = torch.exp(s - most[:, None])
                total = torch.where(some, p.sum(1), 1.0)
                self.out.view[rows, h] = ((p / total[:, None]) @ v[:, h // (self.heads // self.kv)]).to(TORCH[self.dtype]).to(DEV)
                self.stats[rows, h, 0] = torch.where(some, most, -math.inf).float().to(DEV)
                self.stats[rows, h, 1] = torch.where(some, torch.log(total), 0.0).float().to(DEV)

    def check_backward(self, want_table=True):
        half, group = HALF_ULP[self.dtype], self.heads // self.kv
        dtable, table_bound = torch.zeros(max(1, self.buckets), self.heads, dtype=F64), torch.zeros(max(1, self.buckets), self.heads, dtype=F64)
        # fp16: dS is scaled so that twice the largest |dout| |v| is at least 2^12; half the smallest subnormal of that
        most_dout = max([self.rows_of(self.dout, self.q_at[b], n[0]).norm(dim=2).max().item() for b, n in enumerate(self.lengths) if n[0]] + [0.0])
        most_v = max([self.rows_of(self.v, self.k_at[b], n[1]).norm(dim=2).max().item() for b, n in enumerate(self.lengths) if n[1]] + [0.0])
        floor_s = 2.0 ** -25 * 2 * most_dout * most_v * 2.0 ** -12 if self.dtype == "f16" else 2.0 ** -133
        self.bounds = []                              # of dq, dk, dv of each sequence, and of dtable
        floor_p = 2.0 ** -40 if self.dtype == "f16" else 2.0 ** -133
        for b, (nq, nk) in enumerate(self.lengths):
            q, dout, out = (self.rows_of(x, self.q_at[b], nq) for x in (self.q, self.dout, self.out))
            k, v = (self.rows_of(x, self.k_at[b], nk) for x in (self.k, self.v))
            ref = [torch.zeros(nq, self.heads, self.hd, dtype=F64), torch.zeros(nk, self.kv, self.hd, dtype=F64), torch.zeros(nk, self.kv, self.hd, dtype=F64)]
            bound = [torch.zeros_like(x) for x in ref]
            stats = self.stats[self.q_at[b]:self.q_at[b] + nq].double().cpu()
            of = (torch.tensor(self.first_list)[None] <= torch.arange(nk + 1)[:, None]).sum(1) - 1 if self.buckets else None
            for h in range(self.heads):
                if nq == 0 or nk == 0:
                    continue
                s, off, far, seen = self.scores(b, h)
                kh, vh = k[:, h // group], v[:, h // group]
                most, log_sum = stats[:, h, :1], stats[:, h, 1:]
                P = torch.where(seen & (most > -math.inf), torch.exp(s - most - log_sum), 0.0)
                # what P is off, relative: the score, the argument (its parts rounded; without a bias scaled first), the exponential
                size = torch.where(seen & (s > -math.inf), s.abs() + 2 * most.abs(), 0.0).clamp(max=1e6)
                part = torch.where(seen, off + EPS32 * (6 * size * (0 if self.buckets else 1) + 8 * (s - most).abs().clamp(max=200) + 6 * log_sum.abs() + 32), 0.0)
                D = (dout[:, h] * out[:, h]).sum(1, keepdim=True)
                dP = dout[:, h] @ vh.t()
                e = 2 * (self.hd + 4) * EPS32 * (dout[:, h].abs() @ vh.abs().t() + (dout[:, h] * out[:, h]).abs().sum(1, keepdim=True))
                dS = P * (dP - D)
                eS = dS.abs() * (part + 4 * EPS32) + P * (1 + part) * e
                eP = P * part
                rS, rP = eS + half * (dS.abs() + eS) + floor_s * seen, eP + half * (P + eP) + floor_p * seen
                ref[0][:, h] = self.scale * dS @ kh
                bound[0][:, h] = self.scale * (rS @ kh.abs() + 2 * (nk + 8) * EPS32 * ((dS.abs() + rS) @ kh.abs()))
                ref[1][:, h // group] += self.scale * dS.t() @ q[:, h]
                bound[1][:, h // group] += self.scale * (rS.t() @ q[:, h].abs() + 2 * (nq * group + 80) * EPS32 * ((dS.abs() + rS).t() @ q[:, h].abs()))
                ref[2][:, h // group] += P.t() @ dout[:, h]
                bound[2][:, h // group] += rP.t() @ dout[:, h].abs() + 2 * (nq * group + 80) * EPS32 * ((P + rP).t() @ dout[:, h].abs())
                if self.buckets:
                    flat = of[far.clamp(min=0)].flatten()
                    dtable[:, h].index_add_(0, flat, torch.where(seen, dS, 0.0).flatten())
                    table_bound[:, h].index_add_(0, flat, torch.where(seen, eS + floor_s * 2.0 ** -20 + (nq + nk + 200) * EPS32 * dS.abs(), 0.0).flatten())
            for x, r, e, at, n, what in zip((self.dq, self.dk, self.dv), ref, bound, (self.q_at, self.k_at, self.k_at), (nq, nk, nk), ("dq", "dk", "dv")):
                self.bounds.append(rounding(r, self.dtype, e + 2 * EPS32 * r.abs()))
                check_rounded(x.view[at[b]:at[b] + n], r, self.bounds[-1], self.dtype, f"{what} of sequence {b}")
        for x, what in ((self.dq, "dq"), (self.dk, "dk"), (self.dv, "dv")):
            x.untouched(5.0, what)
        if self.buckets and want_table:
            more = self.batch * EPS32 * 2
            self.bounds.append(rounding(dtable, self.table_dtype, table_bound * (1 + more) + more * dtable.abs()))
            check_rounded(self.dtable, dtable, self.bounds[-1], self.table_dtype, "dtable")
