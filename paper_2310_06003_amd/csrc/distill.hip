// Distillation from a teacher's top logits, forward and backward (gfx950).
//
// For a row of student logits z[0 .. V) with the teacher's logits t[0 .. k) at the places id[0 .. k), at temperature T:
//   p = softmax(t / T) over the row's held entries,   q = softmax(z / T) over the vocabulary
//   loss = T^2 * sum_j p_j (log p_j - log q_{id_j}),   d loss / d z_v = T (q_v - sum of p_j over id_j = v)
//
// Bound by memory: the row is read once and, for the gradient, written once.  A block takes a row and holds it in registers as
// it came, so that the gradient needs no second read; each thread runs one pass with its own running maximum and sum, and one
// exchange joins them.  All sums are fp32.  The few elements that the teacher names get their values in the registers of the thread that
// holds them: each piece has a list of its entries in shared memory, nearly always empty (16384 rows of 32000 with 128 entries, 366 us without
// any: written a second time after the row 457, each entry looking for its likes among all 468, so 370).
#include "operators.hpp"

namespace {

constexpr int MAX_K = PARO_DISTILL_MAX_K;
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }      // 1 ulp; flushes below 2^-126
constexpr float NOTHING = -__builtin_inff();

// A stored log-sum L is off by up to 2^-24 L, which is what q = exp(z / T - L) is off by, relative.  From this size on (6e-5) the gradient forms
// the row's own maximum and sum again, as the step does: at the lowest numbers of a type, which programs mask whole rows with, the stored one
// holds nothing of the sum, or is infinite.
constexpr float STORED_SERVES = 1024.0f;

// Running maximum m of the logits and sum s of exp((x - m) / T), c = log2(e) / T.  m stays a logit, undivided: the lowest number of
// a type, which programs mask with, does not overflow.  Nothing yet: m = -inf, s = 0.  fmaxf passes a NaN over; it reaches s.
struct MaxSum {
    float m, s;
    template <int N>
    __device__ __forceinline__ void take(const float (&x)[N], float c) {
        const float before = m;
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, x[e]);
        const float from = m == NOTHING ? 0.0f : m;
        s *= before == NOTHING ? 1.0f : exp2_fast((before - from) * c);
#pragma unroll
        for (int e = 0; e < N; ++e) s += exp2_fast((x[e] - from) * c);
    }
};
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c) {
    MaxSum r;
    r.m = fmaxf(a.m, b.m);
    const float ka = a.m == NOTHING ? 1.0f : exp2_fast((a.m - r.m) * c), kb = b.m == NOTHING ? 1.0f : exp2_fast((b.m - r.m) * c);
    r.s = a.s * ka + b.s * kb;
    return r;
}
// ... over the block, in every thread, in a fixed shape.
template <int THREADS>
__device__ __forceinline__ MaxSum block_join(MaxSum v, MaxSum *room, float c) {
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) v = join(v, MaxSum{__shfl_xor(v.m, step), __shfl_xor(v.s, step)}, c);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = join(v, room[w], c);
    return v;
}

// Between two pieces: the compiler neither works on both at once nor keeps what it unpacked from one, either of which costs it the
// registers that the row needs (and 2 waves a SIMD instead of 8, or spills).
__device__ __forceinline__ void apart(u32x4 &piece) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned w = piece[i];
        asm volatile("" : "+v"(w));
        piece[i] = w;
    }
    __builtin_amdgcn_sched_barrier(0);
}

struct Row {
    int64_t vocab, k, ld_logits, ld_teacher, ld_dlogits;
    float temperature;
    int teacher_dtype;
};

__device__ __forceinline__ float teacher_of(const void *t, int64_t at, int dtype) {
    return dtype == PARO_F32 ? static_cast<const float *>(t)[at] : bits16_to_f32(dtype, static_cast<const unsigned short *>(t)[at]);
}

// HELD pieces of the row a thread, in registers; 0: the row is read again for the gradient.  Of 16, no more than 128 registers (two
// more, and so one block of 512 threads a compute unit: 666 rows of 60179 43 us, so 38); of 8 in the gradient alone no more than 72, seven waves a SIMD.
template <int DT, int THREADS, int HELD, bool LOSS, bool GRAD>
__global__ __launch_bounds__(THREADS, HELD == 16 ? 4 : HELD == 8 && !LOSS ? 7 : 1) void k_distill(const void *logits, const void *teacher, const int32_t *ids, const float *dloss, float *loss,
                                                     float *lse, void *dlogits, Row d) {
    constexpr int E = Elem<DT>::E, ROOM = 4 * THREADS < MAX_K ? 4 * THREADS : MAX_K;      // for entries
    constexpr unsigned MINUS_INF = DT == PARO_F32 ? 0xFF800000u : DT == PARO_F16 ? 0xFC00FC00u : 0xFF80FF80u;
    __shared__ __attribute__((aligned(16))) int s_id[ROOM];
    __shared__ float s_p[ROOM];
    __shared__ MaxSum s_teacher[THREADS / 64], s_student[THREADS / 64];
    __shared__ float s_loss[THREADS / 64];
    constexpr int LISTS = GRAD && HELD ? HELD * THREADS + 1 : 1;
    __shared__ int s_list[LISTS];                                // of each piece, and of the short one: an entry + 1, or none
    __shared__ short s_next[GRAD && HELD ? ROOM : 1];           // the entry + 1 after an entry
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid & ~63);
    const int k = (int)d.k;
    const char *z = static_cast<const char *>(logits) + row * d.ld_logits * Elem<DT>::BYTES;
    char *dz = GRAD ? static_cast<char *>(dlogits) + row * d.ld_dlogits * Elem<DT>::BYTES : nullptr;
    const float inverse_t = 1.0f / d.temperature, c = LOG2E * inverse_t;
    float stored = 0.0f;                                         // the row's log-sum, on its way beside the teacher's entries
    if constexpr (!LOSS) stored = lse[row];

    if constexpr (GRAD && HELD > 0)
        for (int i = tid; i < LISTS; i += THREADS) s_list[i] = 0;

    // The teacher's entries.  One is masked where its place is outside the vocabulary, or its logit -inf.
    MaxSum top{NOTHING, 0.0f};
    for (int j = tid; j < k; j += THREADS) {
        const int id = ids[row * d.ld_teacher + j];
        const float t = teacher_of(teacher, row * d.ld_teacher + j, d.teacher_dtype);
        const bool held = id >= 0 && id < d.vocab && t != NOTHING;
        s_id[j] = held ? id : -1;
        s_p[j] = t;
        if (held) top = join(top, MaxSum{t, 1.0f}, c);
    }
    if (tid < 4 && k + tid < ROOM) s_id[k + tid] = -1;
    top = block_join<THREADS>(top, s_teacher, c);
    const bool some = top.s != 0.0f;                             // NaN counts as something

    const int64_t pieces = d.vocab / E;
    const int rest = (int)(d.vocab - pieces * E);                // elements of a last, shorter piece
    if (!some) {
        if (LOSS && tid == 0) {
            loss[row] = 0.0f;
            if (lse) lse[row] = 0.0f;
        }
        if constexpr (GRAD) {
            for (int64_t i = tid; i < pieces; i += THREADS) store_piece<DT>(dz, i * E, u32x4{0, 0, 0, 0});
            if (tid < rest) store_one<DT>(dz, pieces * E + tid, 0.0f);
        }
        return;
    }

    // The student's row.
    u32x4 held[HELD ? HELD : 1];
    float last = 0.0f;                                           // the short piece: an element a thread
    if constexpr (HELD > 0) {
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            const int64_t i = h * THREADS + tid;
            held[h] = u32x4{MINUS_INF, MINUS_INF, MINUS_INF, MINUS_INF};
            // streamed where it is the last reader: 8000 rows of 32000 in fp16 167 us, not 183, 2047 of 50257 in fp32 131 and 141; with the
            // loss 16384 rows 380 and 360
            if (i < pieces) held[h] = LOSS ? load_piece<DT>(z, i * E) : load_stream<DT>(z, i * E);
        }
    }
    if (tid < rest) last = load_one<DT>(z, pieces * E + tid);
    // The student's logits at the teacher's places, before anything is overwritten.
    constexpr int OWN = ROOM / THREADS;
    float at_id[OWN];
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int j = o * THREADS + tid;
        at_id[o] = j < k && s_id[j] >= 0 ? load_one<DT>(z, s_id[j]) : 0.0f;
    }

    // Maximum and sum of the row.
    const auto of_row = [&]() {
        MaxSum mine{NOTHING, 0.0f};
        const auto take = [&](u32x4 raw) {
            float x[E];
            unpack<DT>(raw, x);
            mine.take(x, c);
        };
        if constexpr (HELD > 0 && LOSS) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                if (h * THREADS + wave < pieces) take(held[h]);     // 4000 rows of 17000 60 us without, 53
                apart(held[h]);
            }
        } else if constexpr (HELD > 0) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {        // of copies: what is unpacked here, by few rows, is not kept for all of them
                u32x4 piece = held[h];
                if constexpr (DT != PARO_F32) apart(piece);
                take(piece);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            for (int64_t i = tid; i < pieces; i += 4 * THREADS) {
                u32x4 raw[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i + u * THREADS < pieces) raw[u] = load_piece<DT>(z, (i + u * THREADS) * E);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i + u * THREADS < pieces) take(raw[u]);
            }
        }
        if (tid < rest && last != NOTHING) mine = join(mine, MaxSum{last, 1.0f}, c);
        return block_join<THREADS>(mine, s_student, c);
    };
    float most, norm;                                            // q = 2^((z - most) c - norm)
    if (LOSS || fabsf(stored) >= STORED_SERVES) {                // a stored NaN stays NaN
        const MaxSum all = of_row();
        most = all.m == NOTHING ? 0.0f : all.m;
        norm = all.s == 0.0f ? 0.0f : __log2f(all.s);            // a row of -inf alone: q = 0
        if (LOSS && lse && tid == 0) lse[row] = all.s == 0.0f ? NOTHING : most * inverse_t + norm * LN2;
    } else {
        // The stored log-sum as a logit, subtracted before anything is scaled: scaled first, both sides are rounded at their full size.  What that
        // logit is off by, from 1 / T in two parts, goes into norm.
        most = stored * d.temperature;
        norm = (fmaf(-most, inverse_t, stored) - most * (fmaf(-d.temperature, inverse_t, 1.0f) * inverse_t)) * LOG2E;
    }

    // p, and this row's loss.  p is divided by its sum itself, not in the exponent, where the sum's logarithm would be rounded at its size.
    // loss = T sum p (T log p - T log q) in logits, undivided: a named word that the student masks with the lowest number is not infinite at T < 1.
    const float share = 1.0f / top.s, norms = (norm - __log2f(top.s)) * LN2 * d.temperature;
    float sum = 0.0f;
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
        const int j = o * THREADS + tid;
        if (j < k) {
            const float below = s_p[j] - top.m, p = s_id[j] >= 0 ? exp2_fast(below * c) * share : 0.0f;
            s_p[j] = p;
            if (LOSS && p != 0.0f) sum += p * (below - (at_id[o] - most) + norms);
        }
    }
    if constexpr (LOSS) {
#pragma unroll
        for (int step = 32; step >= 1; step /= 2) sum += __shfl_xor(sum, step);
        if ((tid & 63) == 0) s_loss[tid >> 6] = sum;
        __syncthreads();                                         // s_p too
        if (tid == 0) {
            float all = 0.0f;
            for (int w = 0; w < THREADS / 64; ++w) all += s_loss[w];
            loss[row] = all * d.temperature;
        }
    } else {
        __syncthreads();
    }

    if constexpr (GRAD) {
        const float w = (dloss ? dloss[row] : 1.0f) * d.temperature;
        const auto q = [&](float x) { return exp2_fast(fmaf(x - most, c, -norm)); };
        // The entries in order, four at a time; those past k are masked.
        const auto each = [&](auto &&visit) {
            for (int i = 0; i < k; i += 4) {
                const int4 id = *reinterpret_cast<const int4 *>(&s_id[i]);
                visit(i, id.x);
                visit(i + 1, id.y);
                visit(i + 2, id.z);
                visit(i + 3, id.w);
            }
        };
        if constexpr (HELD > 0) {
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                const int j = o * THREADS + tid;
                if (j < k && s_id[j] >= 0) s_next[j] = (short)atomicExch(&s_list[s_id[j] / E], j + 1);
            }
            __syncthreads();
            // What the entries of piece i take off, added up in their order, not the list's.  Of a few the next one is looked for in the list, which
            // takes their square of reads that wait for one another; otherwise all entries are visited, four a read (always so: 20 rows of
            // 2000 with 1000 entries 69 us, so 10; 4000 of 12512 in fp32 with 132 314 and 81; up to 8 from the list whatever k is: 1196
            // of 1584 with 10 entries 12 us, so 9).
            const auto take_off = [&](int i, float (&x)[E]) {
                const int entry = s_list[i];
                if (!entry) return;
                float p[E] = {};
                const auto add = [&](int id, float of) {
#pragma unroll
                    for (int e = 0; e < E; ++e) p[e] += (id & (E - 1)) == e ? of : 0.0f;
                };
                const int second = s_next[entry - 1];
                if (!second) {
                    add(s_id[entry - 1], s_p[entry - 1]);
                } else {
                    int count = 1;
                    for (int j = second; j && 4 * count * count <= k; j = s_next[j - 1]) ++count;
                    if (4 * count * count <= k) {
                        for (int before = 0; count > 0; --count) {
                            int next = ROOM + 1;
                            for (int j = entry; j; j = s_next[j - 1]) next = j > before && j < next ? j : next;
                            add(s_id[next - 1], s_p[next - 1]);
                            before = next;
                        }
                    } else {
                        each([&](int j, int id) {
                            if (id >= 0 && id / E == i) add(id, s_p[j]);
                        });
                    }
                }
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] -= p[e] * w;
            };
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                const int i = h * THREADS + tid;
                if (i < pieces) {
                    float x[E];
                    unpack<DT>(held[h], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = q(x[e]) * w;
                    take_off(i, x);
                    store_stream<DT>(dz, (int64_t)i * E, pack<DT>(x));      // 2047 rows of 50257 in fp32 148 us, so 141
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (tid < rest) {
                float x[E] = {};
                take_off((int)pieces, x);
                float off = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) off = e == tid ? x[e] : off;
                store_one<DT>(dz, pieces * E + tid, q(last) * w + off);
            }
        } else {
            for (int64_t i = tid; i < pieces; i += 4 * THREADS) {
                u32x4 raw[4];
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i + u * THREADS < pieces) raw[u] = load_piece<DT>(z, (i + u * THREADS) * E);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (i + u * THREADS >= pieces) continue;
                    float x[E];
                    unpack<DT>(raw[u], x);
#pragma unroll
                    for (int e = 0; e < E; ++e) x[e] = q(x[e]) * w;
                    store_piece<DT>(dz, (i + u * THREADS) * E, pack<DT>(x));
                }
            }
            if (tid < rest) store_one<DT>(dz, pieces * E + tid, q(last) * w);
            __syncthreads();                                     // the row is written: now what the teacher names
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                const int j = o * THREADS + tid;
                if (j >= k || s_id[j] < 0) continue;
                float p = 0.0f;
                bool first = true;                               // a place that is named twice: its first entry stores it
                each([&](int i, int id) {
                    if (id != s_id[j]) return;
                    p += s_p[i];
                    first = first && i >= j;
                });
                if (first) store_one<DT>(dz, s_id[j], (q(at_id[o]) - p) * w);
            }
        }
    }
}

// ---------------------------------------------------------------- host
template <int DT, bool LOSS, bool GRAD>
void launch(const paro_distill_t &d, const void *logits, const void *teacher, const int32_t *ids, const float *dloss, float *loss, float *lse,
            void *dlogits, hipStream_t st) {
    const Row r{d.vocab, d.k, d.ld_logits ? d.ld_logits : d.vocab, d.ld_teacher ? d.ld_teacher : d.k, d.ld_dlogits ? d.ld_dlogits : d.vocab,
                d.temperature, d.teacher_dtype};
    const int64_t pieces = d.vocab / Elem<DT>::E;
#define PARO_DISTILL(THREADS, HELD)                                                                                                        \
    hipLaunchKernelGGL((k_distill<DT, THREADS, HELD, LOSS, GRAD>), dim3((unsigned)d.n), dim3(THREADS), 0, st, logits, teacher, ids, dloss, \
                       loss, lse, dlogits, r)
    // Few threads a row, so that many rows are under way and each thread has work: 12008 rows of 1717, loss alone, by 256 threads 31 us, by 64 15;
    // 6000 of 6000 by 256 23, by 128 18; 5602 of 12509 in fp16 in 16 pieces a thread 73, in 8 63; 16384 of 32000 by 512 threads 409, by 256
    // 380.  But entries enough for a thread, four: 30 rows of 2000 with 1000 entries by 64 threads 22, by 256 10.
    if (pieces <= 64 * 4 && d.k <= 4 * 64) PARO_DISTILL(64, 4);
    else if (pieces <= 128 * 4 && d.k <= 4 * 128) PARO_DISTILL(128, 4);
    else if (pieces <= 128 * 8 && d.k <= 4 * 128) PARO_DISTILL(128, 8);
    else if (pieces <= 256 * 4) PARO_DISTILL(256, 4);
    else if (pieces <= 256 * 8) PARO_DISTILL(256, 8);
    else if (pieces <= 256 * 16) PARO_DISTILL(256, 16);
    else if (pieces <= 512 * 16) PARO_DISTILL(512, 16);
    else if (pieces <= 1024 * 16) PARO_DISTILL(1024, 16);
    else PARO_DISTILL(1024, 0);
#undef PARO_DISTILL
}

int check(const std::string &f, const paro_distill_t *d, const void *logits, const void *teacher, const int32_t *ids) {
    int rc;
    if (!d) return fail(PARO_EINVAL, f + "d is NULL");
    if (d->n < 0 || d->n >= ((int64_t)1 << 22)) return fail(PARO_EINVAL, f + "n must be in [0, 2^22)");
    if (d->vocab < 1 || d->vocab > INT32_MAX - 8192) return fail(PARO_EINVAL, f + "bad vocab");
    if (d->k < 1 || d->k > MAX_K) return fail(PARO_EINVAL, f + "k must be in [1, PARO_DISTILL_MAX_K]");
    if (!(d->temperature >= 1e-6f && d->temperature <= 1e6f)) return fail(PARO_EINVAL, f + "temperature must be in [1e-6, 1e6]");
    if (!is_dtype(d->dtype) || !is_dtype(d->teacher_dtype)) return fail(PARO_EINVAL, f + "bad dtype");
    if ((d->ld_logits && d->ld_logits < d->vocab) || (d->ld_dlogits && d->ld_dlogits < d->vocab) || (d->ld_teacher && d->ld_teacher < d->k))
        return fail(PARO_EINVAL, f + "a row is longer than its distance to the next");
    if (too_large(d->n, d->ld_logits, 4) || too_large(d->n, d->ld_dlogits, 4) || too_large(d->n, d->ld_teacher, 4))
        return fail(PARO_EINVAL, f + "too large");
    if (d->n == 0) return PARO_OK;
    if ((rc = check_array(logits, size_of(d->dtype), f + "logits"))) return rc;
    if ((rc = check_array(teacher, size_of(d->teacher_dtype), f + "teacher"))) return rc;
    return check_array(ids, 4, f + "ids");
}

// dlogits may be logits itself (each element is read before it is written), with the same distance between rows.
int check_dlogits(const std::string &f, const paro_distill_t *d, const void *logits, const float *dloss, void *dlogits) {
    int rc;
    if ((rc = check_array(dlogits, size_of(d->dtype), f + "dlogits"))) return rc;
    if (dloss && (rc = check_array(dloss, 4, f + "dloss"))) return rc;
    if (dlogits == logits && (d->ld_logits ? d->ld_logits : d->vocab) != (d->ld_dlogits ? d->ld_dlogits : d->vocab))
        return fail(PARO_EINVAL, f + "in place, ld_dlogits must be ld_logits");
    return PARO_OK;
}

template <bool LOSS, bool GRAD>
int run(const char *what, const paro_distill_t *d, const void *logits, const void *teacher, const int32_t *ids, const float *dloss, float *loss,
        float *lse, void *dlogits, void *stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (d->dtype == PARO_F32) launch<PARO_F32, LOSS, GRAD>(*d, logits, teacher, ids, dloss, loss, lse, dlogits, st);
    else if (d->dtype == PARO_F16) launch<PARO_F16, LOSS, GRAD>(*d, logits, teacher, ids, dloss, loss, lse, dlogits, st);
    else launch<PARO_BF16, LOSS, GRAD>(*d, logits, teacher, ids, dloss, loss, lse, dlogits, st);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PARO_OK : fail(PARO_EHIP, std::string(what) + hipGetErrorString(e));
}

}  // namespace

extern "C" {

int paro_distill_loss(const paro_distill_t *d, const void *logits, const void *teacher, const int32_t *ids, float *loss, float *lse, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_distill_loss: ";
        int rc;
        if ((rc = check(f, d, logits, teacher, ids)) || d->n == 0) return rc;
        if ((rc = check_array(loss, 4, f + "loss")) || (lse && (rc = check_array(lse, 4, f + "lse")))) return rc;
        return run<true, false>("paro_distill_loss: ", d, logits, teacher, ids, nullptr, loss, lse, nullptr, stream);
    });
}

int paro_distill_grad(const paro_distill_t *d, const void *logits, const void *teacher, const int32_t *ids, const float *lse, const float *dloss,
                      void *dlogits, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_distill_grad: ";
        int rc;
        if ((rc = check(f, d, logits, teacher, ids)) || d->n == 0) return rc;
        if ((rc = check_array(lse, 4, f + "lse")) || (rc = check_dlogits(f, d, logits, dloss, dlogits))) return rc;
        return run<false, true>("paro_distill_grad: ", d, logits, teacher, ids, dloss, nullptr, const_cast<float *>(lse), dlogits, stream);
    });
}

int paro_distill_step(const paro_distill_t *d, const void *logits, const void *teacher, const int32_t *ids, const float *dloss, float *loss,
                      void *dlogits, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_distill_step: ";
        int rc;
        if ((rc = check(f, d, logits, teacher, ids)) || d->n == 0) return rc;
        if ((rc = check_array(loss, 4, f + "loss")) || (rc = check_dlogits(f, d, logits, dloss, dlogits))) return rc;
        return run<true, true>("paro_distill_step: ", d, logits, teacher, ids, dloss, loss, nullptr, dlogits, stream);
    });
}

}  // extern "C"
