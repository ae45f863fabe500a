// Attention with a sliding window, sinks and a relative position bias by buckets, forward (gfx950):
//
//   s_ij = scale q_i . k_j + table[bucket(p_i - j)][head],  out_i = sum_j softmax(s_i)_j v_j   over the keys j that query i sees
//
// in one pass over the keys: a row keeps its largest score m, l = sum exp(s - m) and the sum of exp(s - m) v in fp32; where m grows by more than a factor of
// 2^8 in exp(m), l and the sum are scaled down (until then exp(s - m) is above one, which costs nothing).  The products run on the matrix cores
// with the scores transposed: a lane has a query's scores of 16 keys of 32, rounded to 16 bits they are the operand of the second product as they
// stand, and maximum and sum of a row need one exchange between the two halves of a wave.  fp16 shares are multiplied by 2^7 (divided out at the end), so that
// those below 2^-14 of the largest keep their bits.
//
// k_attend: 8192 tokens of 32 heads of 128, window 4096, 437 us at best (945 TF), 479 in the middle: the matrix cores are busy 50 % of the cycles, the vector unit (16 exponents,
// 84 other instructions for 32 x 32 scores) a third, at the clock that power allows (1.8 GHz).  8 x 1024 tokens of 12 heads of 64 with bias 35 us: the way from score to exponent to
// product, with a barrier behind eight matrix instructions; waves wait 41 %, matrix cores are busy 13 %.  64 tokens over 100000 keys, 8 key heads of 128, shared: 203 us and 7 to join.
// k_attend_few: 4 tokens over 50000 to 100000 keys, 8 key heads of 128, 271 us at best, 4.9 TB/s: memory.
#include "attn.hpp"

namespace {

constexpr int QUERIES = 128, KEYS = 32;      // of a block, of a tile
constexpr int MOST_SHARES = 256;
constexpr float GROWS = 8.0f;                // powers of two that a row's shares may exceed one by
template <int DT>
constexpr float SHIFT = DT == PARO_F16 ? 7.0f : 0.0f;

struct Few {                              // of blocks that share a tile's keys, whose sums k_attend_join adds
    int shares, row_tiles;                // row_tiles: of a sequence's key head
    float *sums, *stats;                  // of a share: [block][ROWS][HD], and [block][ROWS][2]: largest score, sum
};

// SHARED: the block has one share of its tile's keys.  (Unshared: 64 tokens over 100000 keys, 8 key heads of 128, 1793 us, so 221; 8192 tokens of one head of 64 123, so 37; 2048 of
// four 37, so 29.)
template <int DT, int HD, bool BIAS, bool SHARED>
__global__ __launch_bounds__(256, 2) void k_attend(Attn a, Few f) {
    using T = Tile<HD>;
    constexpr int BYTES = KEYS * T::ROW, STEPS = HD / 16, RING = 4;
    __shared__ __attribute__((aligned(1024))) char tiles[RING][2][BYTES];    // [part of the ring][keys, values]
    __shared__ Bias bias;
    const int group = a.heads / a.kv_heads;
    int unit_of, tile_of, of_group, share = 0;
    if constexpr (SHARED) {                // shares of the same keys stay on one XCD where there are eight, or a multiple
        const int block = blockIdx.x / f.shares;
        share = blockIdx.x % f.shares;
        unit_of = block / f.row_tiles;
        tile_of = block % f.row_tiles / group;
        of_group = block % f.row_tiles % group;
    } else {
        const Work work(blockIdx.x, a.batch * a.kv_heads, a.tiles * group, a.bunch, group);
        unit_of = work.unit;
        tile_of = a.tiles - 1 - work.within / group;                                   // the longest first
        of_group = work.within % group;
    }
    const int kv = unit_of % a.kv_heads, b = unit_of / a.kv_heads, head = kv * group + of_group, i0 = tile_of * QUERIES;
    const Sequence seq(a, b);
    if (i0 >= seq.nq) return;
    const int lane = threadIdx.x & 63, w = wave_of(), h = lane >> 5;
    const int off = seq.nk - seq.nq, first = i0 + off, last = (i0 + QUERIES < seq.nq ? i0 + QUERIES : seq.nq) - 1 + off;
    const Seen<KEYS> seen(a, first, last);
    const int from_tile = SHARED ? (int)((int64_t)seen.tiles * share / f.shares) : 0, to_tile = SHARED ? (int)((int64_t)seen.tiles * (share + 1) / f.shares) : seen.tiles;
    const int of_wave = first + w * 32, place = of_wave + (lane & 31), i = i0 + w * 32 + (lane & 31);     // of the lane's query

    const int64_t row_k = a.copied_k ? (int64_t)b * a.len_k : seq.k0, row_v = a.copied_v ? (int64_t)b * a.len_k : seq.k0;
    const char *const keys_at = a.keys.of(row_k, kv), *const values_at = a.values.of(row_v, kv);
    const int64_t k_step = a.keys.ld * (2 * KEYS), v_step = a.values.ld * (2 * KEYS);
    const Filled<HD, KEYS> fill_k(a.keys.ld, a.hd), fill_v(a.values.ld, a.hd);
    constexpr int FILLS = 2 * Filled<HD, KEYS>::FILLS;
    Distances by_distance{};
    const auto lowest = [&](int k0) { return first - (k0 + KEYS - 1); };
    const auto is_far = [&](int k0) { return BIAS && by_distance.usual && by_distance.beyond(lowest(k0)); };
    const auto fill = [&](int t, int part) __attribute__((always_inline)) {
        const int tile = seen.tile(t), k0 = tile * KEYS;
        if constexpr (BIAS) by_distance.look_up(bias, lowest(k0), part, a.buckets);
        const u32x4 k_from = fill_k.descriptor(keys_at + tile * k_step), v_from = fill_v.descriptor(values_at + tile * v_step);
        if (seen.holds_all(k0)) {
            fill_k.whole(k_from, tiles[part][0]);
            fill_v.whole(v_from, tiles[part][1]);
        } else {
            const auto holds = [&](int r) { return seen.holds(k0 + r); };
            fill_k.held(k_from, tiles[part][0], holds);
            fill_v.held(v_from, tiles[part][1], holds);
        }
    };
    // Nothing, in the place of a tile that is not there: the waits count on as many loads each time.
    const auto fill_none = [&](int part) __attribute__((always_inline)) {
        const auto holds = [](int) { return false; };
        fill_k.held(fill_k.descriptor(keys_at), tiles[part][0], holds);
        fill_v.held(fill_v.descriptor(values_at), tiles[part][1], holds);
    };

    if constexpr (BIAS) {
        bias.load(a, head);
        __syncthreads();
        by_distance.begin(bias, a.buckets);
        __syncthreads();
    }
    short8_t q[STEPS];
    const char *const query = a.q.of((int64_t)seq.q0 + (i < seq.nq ? i : seq.nq - 1), head);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) q[s] = __builtin_bit_cast(short8_t, piece_of_head(query, s * 16 + h * 8, a.hd, i < seq.nq));
    // Scores are in units of `unit` powers of two: as the products give them without a bias, natural ones with one.  Of a tile whose keys all have the last bucket's
    // bias (far) it is not added, but enters the largest score and the exponent as a whole.
    // Where a row's largest score is large in size (a table's lowest number, or large products), differences to it are formed before they are brought to powers of two: its multiple
    // by LOG2E is off by its size times 2^-24, a factor of more than fp16 holds from 10^7 on.
    const float unit = BIAS ? LOG2E : a.scale * LOG2E, grows = GROWS / unit, usual = BIAS ? USUAL : USUAL / a.scale;
    bool large = false;                    // of some row of the wave
    f32x16 out[HD / 32] = {}, scores[2];
    bool far[2] = {};
    float most = -INFINITY, used = -INFINITY, from = 0.0f, shift = SHIFT<DT>, sum = 0.0f;
    // What is left of a tile's scores: the bias, and -inf where a query does not see a key.
    const auto add_bias = [&](f32x16 &s, bool &is, int k0, int part) __attribute__((always_inline)) {
        if constexpr (BIAS) {
            is = is_far(k0);
            if (!is) {
                const float *const at = by_distance.values(bias, lowest(k0), part) + (place - first) + 4 - 4 * h;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], a.scale, at[27 - (8 * (e / 4) + e % 4)]);
            }
        }
    };
    const auto finish = [&](f32x16 &s, bool &is, int k0, int part) __attribute__((always_inline)) {
        add_bias(s, is, k0, part);
        const bool all = k0 + KEYS - 1 <= of_wave && (k0 > of_wave + 31 - a.window || k0 + KEYS <= a.sinks);
        if (!all) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (!sees(place, k0 + 8 * (e / 4) + 4 * h + e % 4, a.window, a.sinks)) s[e] = -INFINITY;
        }
    };
    // In step t the scores of tile t + 1 are formed beside the exponentials of tile t, and the products with its values follow.  Meanwhile tile t + 3 goes to the
    // part of the ring whose tile all waves have left.  Four steps a round, so that the parts of the ring are constants.
    // What this wave's queries see of a tile: nothing?
    const auto none = [&](int k0) { return k0 > of_wave + 31 || (k0 + KEYS <= of_wave - a.window + 1 && k0 >= a.sinks); };
    const auto products = [&](auto part_, bool sees_now, bool sees_next, auto &&between) __attribute__((always_inline)) {
        constexpr int part = part_, after = (part + 1) % RING;
        f32x16 &now = scores[part & 1], &next = scores[after & 1];
        const bool &is = far[part & 1];
        if (sees_now) {
            float largest = now[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) largest = fmaxf(largest, now[e]);
            if (BIAS && is) largest = __builtin_fmaf(largest, a.scale, by_distance.far);
            most = max_of_halves(fmaxf(most, largest));
            if (__any(most > used + grows)) {
                const bool some = most > -INFINITY;
                const float times = some ? exp2_((used - most) * unit) : 1.0f;          // 0 at first
                used = most;
                from = some ? most : 0.0f;
                large = __any(fabsf(from) > usual);
                shift = fabsf(from) > usual ? SHIFT<DT> : SHIFT<DT> - from * unit;
                sum *= times;
#pragma unroll
                for (int d = 0; d < HD / 32; ++d) out[d] *= times;
            }
            if (large) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float score = BIAS && is ? __builtin_fmaf(now[e], a.scale, by_distance.far) : now[e];
                    now[e] = fabsf(from) > usual ? score - from : score;
                }
            }
        }
        arrived<FILLS>();                   // tile t + 2 may be on its way
        between();
        const bool as_far = BIAS && is && !large;
        const float times = as_far ? a.scale * LOG2E : unit, plus = as_far ? __builtin_fmaf(by_distance.far - from, LOG2E, SHIFT<DT>) : shift;
        __builtin_amdgcn_s_setprio(1);
        if (sees_next) {                    // behind the last tile: of whatever the ring holds, and not looked at
            next = f32x16{};
#pragma unroll
            for (int c = 0; c < STEPS; ++c) next = mfma32<DT>(T::rows(tiles[after][0], 0, c, lane), q[c], next);
        }
        if (sees_now) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                now[e] = exp2_(__builtin_fmaf(now[e], times, plus));
                sum += now[e];
            }
            asm volatile("" : "+v"(sum));       // beside the products, not behind them
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const short8_t p = pack8<DT>(now, 8 * k);
#pragma unroll
                for (int d = 0; d < HD / 32; ++d) out[d] = mfma32<DT>(T::columns(tiles[part][1], k * 16, d, lane), p, out[d]);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    };
    const auto step = [&](auto part_, int t) __attribute__((always_inline)) {
        constexpr int part = part_, after = (part + 1) % RING, third = (part + 3) % RING;
        const bool sees_next = t + 1 < to_tile && !none(seen.tile(t + 1) * KEYS);
        products(part_, !none(seen.tile(t) * KEYS), sees_next, [&]() __attribute__((always_inline)) {
            if (t + 3 < to_tile) fill(t + 3, third);
            else fill_none(third);
        });
        if (sees_next) finish(scores[after & 1], far[after & 1], seen.tile(t + 1) * KEYS, after);
    };
    // Where every query sees the tiles t + 1 to t + 3 whole, nothing is asked; k0: the first key of tile t; k_at, v_at: tile t + 3.
    const auto plain_step = [&](auto part_, int k0, const char *&k_at, const char *&v_at) __attribute__((always_inline)) {
        constexpr int part = part_, after = (part + 1) % RING, third = (part + 3) % RING;
        products(part_, true, true, [&]() __attribute__((always_inline)) {
            fill_k.whole(fill_k.descriptor(k_at), tiles[third][0]);
            fill_v.whole(fill_v.descriptor(v_at), tiles[third][1]);
            if constexpr (BIAS) by_distance.look_up(bias, lowest(k0 + 3 * KEYS), third, a.buckets);
        });
        add_bias(scores[after & 1], far[after & 1], k0 + KEYS, after);
        k_at += k_step;
        v_at += v_step;
    };
    constexpr std::integral_constant<int, 0> p0{};
    constexpr std::integral_constant<int, 1> p1{};
    constexpr std::integral_constant<int, 2> p2{};
    constexpr std::integral_constant<int, 3> p3{};
    if (from_tile < to_tile) {
        int plain_from, plain_to;
        seen.plain(a, first, last, plain_from, plain_to);
        if (SHARED && plain_to > to_tile) plain_to = to_tile;
        for (int t = 0; t < 3; ++t) {
            if (from_tile + t < to_tile) fill(from_tile + t, t);
            else fill_none(t);
        }
        arrived<2 * FILLS>();
        scores[0] = f32x16{};
#pragma unroll
        for (int c = 0; c < STEPS; ++c) scores[0] = mfma32<DT>(T::rows(tiles[0][0], 0, c, lane), q[c], scores[0]);
        finish(scores[0], far[0], seen.tile(from_tile) * KEYS, 0);
        for (int t = from_tile;;) {
            if (t >= plain_from && t + 6 < plain_to) {
                int k0 = seen.tile(t) * KEYS;
                const char *k_at = keys_at + (seen.tile(t) + 3) * k_step, *v_at = values_at + (seen.tile(t) + 3) * v_step;
                for (; t + 6 < plain_to; t += 4, k0 += 4 * KEYS) {
                    plain_step(p0, k0, k_at, v_at);
                    plain_step(p1, k0 + KEYS, k_at, v_at);
                    plain_step(p2, k0 + 2 * KEYS, k_at, v_at);
                    plain_step(p3, k0 + 3 * KEYS, k_at, v_at);
                }
            }
            step(p0, t);
            if (++t == to_tile) break;
            step(p1, t);
            if (++t == to_tile) break;
            step(p2, t);
            if (++t == to_tile) break;
            step(p3, t);
            if (++t == to_tile) break;
        }
        arrived<0>();                       // nothing is on its way into the shared memory of the block that comes next
    }
    sum = sum_of_halves(sum);
    if constexpr (SHARED) {
        const float times = most > -INFINITY ? exp2_((used - most) * unit) : 1.0f;
        const int64_t row = (int64_t)blockIdx.x * QUERIES + w * 32 + (lane & 31);
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4 *>(f.sums + row * HD + d * 32 + 2 * e + 4 * h) = f32x4{out[d][e], out[d][e + 1], out[d][e + 2], out[d][e + 3]} * times;
        if (h == 0) {
            f.stats[row * 2] = most;
            f.stats[row * 2 + 1] = sum * times;
        }
        return;
    }
    const bool there = i < seq.nq;
    const float times = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;       // NaN stays
    char *const to = a.out.of((int64_t)seq.q0 + i, head);
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) store_row32<DT>(to, d * 32, a.hd, out[d], times, there);
    if (a.stats && there && h == 0) {
        float *const at = a.stats + (((int64_t)seq.q0 + i) * a.heads + head) * 2;
        const bool empty = most == -INFINITY;
        at[0] = BIAS ? most : empty ? most : most * a.scale;
        at[1] = empty ? 0.0f : (__builtin_amdgcn_logf(sum) - SHIFT<DT> + (used - most) * unit) * LN2;
    }
}

// ---------------------------------------------------------------- few queries
// Up to 16 queries a sequence: the keys and values are read once for all queries and heads that share them, and nothing else counts.  A block's waves take 32 keys
// at a time in turn: keys straight into registers as operands, values through shared memory of the wave's own, to be transposed.  The rows of
// the products are the heads of a group, query by query, ROWS in all.  Long sequences are shared out among blocks, whose sums k_attend_join adds.
constexpr int FEW = 16, FEW_KEYS = 32;
// Waves of a block: eight fill a compute unit's memory pipes without a second launch (four a block and twice the blocks, joined: 32 sequences with a window of 1024,
// 8 key heads of 128, 36 us); wide heads with 32 rows leave registers for four.
constexpr int few_waves(int hd, int nt) { return hd == 128 && nt == 2 ? 4 : 8; }

__device__ __forceinline__ float max_of_quads(float x) {
    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max_of_halves(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
}
__device__ __forceinline__ float sum_of_quads(float x) {
    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return sum_of_halves(__uint_as_float(both[0]) + __uint_as_float(both[1]));
}

// What is written of a finished row: largest score `most` (in units), sum of shares, the result's elements.
template <int DT, bool BIAS>
__device__ __forceinline__ void store_stats(const Attn &a, int64_t row, int head, float most, float sum) {
    float *const at = a.stats + (row * a.heads + head) * 2;
    const bool empty = most == -INFINITY;
    at[0] = BIAS || empty ? most : most * a.scale;
    at[1] = empty ? 0.0f : (__builtin_amdgcn_logf(sum) - SHIFT<DT>) * LN2;
}

// Four elements of a head's row.
template <int DT>
__device__ __forceinline__ void store4(char *row, int column, int hd, f32x4 v, float times) {
    const u32x2 packed{both<DT>(v[0] * times, v[1] * times), both<DT>(v[2] * times, v[3] * times)};
    if (column + 4 <= hd) {
        store_half_piece(row, column, packed);
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (column + e < hd) reinterpret_cast<unsigned short *>(row)[column + e] = (unsigned short)(packed[e / 2] >> (16 * (e & 1)));
}

template <int DT, int HD, bool BIAS, int NT>
__global__ __launch_bounds__((64 * few_waves(HD, NT))) void k_attend_few(Attn a, Few f) {
    using T = Tile<HD>;
    constexpr int ROWS = 16 * NT, STEPS = HD / 32, PASSES = FEW_KEYS * T::PIECES / 64, WAVES = few_waves(HD, NT);
    static_assert(FEW_KEYS * T::ROW == 16 * HD * 4, "a wave's sums of 16 rows take the place of its values");
    __shared__ __attribute__((aligned(1024))) char values[WAVES][FEW_KEYS * T::ROW];
    __shared__ float of_waves[WAVES][ROWS][2];
    __shared__ int first_of[MAX_BUCKETS];
    const int lane = threadIdx.x & 63, w = wave_of(), g = lane >> 4, of16 = lane & 15;
    const int share = blockIdx.x % f.shares, row_tile = blockIdx.x / f.shares % f.row_tiles;
    const int of_kv = blockIdx.x / f.shares / f.row_tiles, kv = of_kv % a.kv_heads, b = of_kv / a.kv_heads;
    const int group = a.heads / a.kv_heads, rows_before = row_tile * ROWS;
    const Sequence seq(a, b);
    const int off = seq.nk - seq.nq, rows = seq.nq * group;
    if (rows_before >= rows) return;
    const Seen<FEW_KEYS> seen(a, off, seq.nk - 1);
    const int from = (int)((int64_t)seen.tiles * share / f.shares), to = (int)((int64_t)seen.tiles * (share + 1) / f.shares);

    int place[NT], head[NT];
    bool there[NT];
    short8_t q[NT][STEPS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = rows_before + n * 16 + of16;
        there[n] = r < rows;
        place[n] = off + r / group;
        head[n] = kv * group + r % group;
        const char *const query = a.q.of((int64_t)seq.q0 + (there[n] ? r / group : 0), kv * group + (there[n] ? r % group : 0));
#pragma unroll
        for (int s = 0; s < STEPS; ++s) q[n][s] = __builtin_bit_cast(short8_t, piece_of_head(query, s * 32 + g * 8, a.hd, there[n]));
    }
    u32x4 from_k[2][STEPS], from_v[PASSES];
    const int piece = lane % T::PIECES, of_pass = lane / T::PIECES;
    constexpr int APART = 64 / T::PIECES;
    const char *const keys_at = a.k.of(seq.k0, kv), *const values_at = a.v.of(seq.k0, kv);
    const auto load = [&](int t) {
        const int k0 = seen.tile(t) * FEW_KEYS;
        const auto row = [&](const char *at, int64_t ld, int j) { return at + (int64_t)(j < seq.nk ? j : seq.nk - 1) * (ld * 2); };
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const char *const key = row(keys_at, a.k.ld, k0 + n * 16 + of16);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) from_k[n][s] = load_piece<DT>(key, column_of(s * 32 + g * 8, a.hd));
        }
#pragma unroll
        for (int n = 0; n < PASSES; ++n) from_v[n] = load_piece<DT>(row(values_at, a.v.ld, k0 + of_pass + n * APART), column_of(piece * 8, a.hd));
    };
    int far_from = 0;
    float far_bias[NT] = {};
    if (from + w < to) load(from + w);
    if constexpr (BIAS) {
        for (int i = threadIdx.x; i < a.buckets; i += 64 * WAVES) first_of[i] = a.first[i];
#pragma unroll
        for (int n = 0; n < NT; ++n)
            if (there[n]) far_bias[n] = table_value(a, a.buckets - 1, head[n]);
        __syncthreads();
        far_from = first_of[a.buckets - 1];
    }
    const float unit = BIAS ? LOG2E : a.scale * LOG2E;
    f32x4 out[NT][HD / 16] = {};
    float most[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        most[n] = -INFINITY;
        sum[n] = 0.0f;
    }
    char *const mine = values[w];
    for (int t = from + w; t < to; t += WAVES) {
        const int k0 = seen.tile(t) * FEW_KEYS;
        if (!seen.holds_all(k0) || a.hd != HD) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int s = 0; s < STEPS; ++s) from_k[n][s] = finished(from_k[n][s], s * 32 + g * 8, a.hd, seen.holds(k0 + n * 16 + of16));
#pragma unroll
            for (int n = 0; n < PASSES; ++n) from_v[n] = finished(from_v[n], piece * 8, a.hd, seen.holds(k0 + of_pass + n * APART));
        }
        short8_t keys[2][STEPS];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) keys[n][s] = __builtin_bit_cast(short8_t, from_k[n][s]);
        asm volatile("" ::: "memory");                  // the last tile's values have been read
#pragma unroll
        for (int n = 0; n < PASSES; ++n) *reinterpret_cast<u32x4 *>(mine + T::at(of_pass + n * APART, piece)) = from_v[n];
        asm volatile("" ::: "memory");                  // a wave's accesses of shared memory go in their order
        if (t + WAVES < to) load(t + WAVES);
        f32x4 s[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                s[n][k] = f32x4{};
#pragma unroll
                for (int c = 0; c < STEPS; ++c) s[n][k] = mfma16<DT>(keys[k][c], q[n][c], s[n][k]);
            }
        if constexpr (BIAS) {
            const bool far = off - (k0 + FEW_KEYS - 1) >= far_from;
            // distances off - (k0 + 31) + lane: up to 16 queries' places, 32 keys
            const int lowest = off - (k0 + FEW_KEYS - 1);
            int bucket = 0;
            if (!far) {
                const int d = lowest + lane < 0 ? 0 : lowest + lane;
                int some = a.buckets;
                while (some > 1) {
                    const int half = some >> 1;
                    const bool up = first_of[bucket + half] <= d;
                    bucket = up ? bucket + half : bucket;
                    some = up ? some - half : half;
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float value = far_bias[n];
                        if (!far) {
                            const int of = __shfl(bucket, (place[n] - (k0 + k * 16 + 4 * g + e) - lowest) & 63);
                            value = there[n] ? table_value(a, of, head[n]) : 0.0f;
                        }
                        s[n][k][e] = __builtin_fmaf(s[n][k][e], a.scale, value);
                    }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float now = most[n];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = k0 + k * 16 + 4 * g + e;
                    if (j >= seq.nk || !sees(place[n], j, a.window, a.sinks)) s[n][k][e] = -INFINITY;
                    now = fmaxf(now, s[n][k][e]);
                }
            now = max_of_quads(now);
            const float was = most[n], base = now == -INFINITY ? 0.0f : now;
            const float times = was == -INFINITY ? 0.0f : exp2_((was - base) * unit);
            most[n] = now;
            float added = 0.0f;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[n][k][e] = exp2_(__builtin_fmaf(s[n][k][e] - base, unit, SHIFT<DT>));
                    added += s[n][k][e];
                }
            sum[n] = sum[n] * times + added;
            u32x4 packed;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                packed[2 * k] = both<DT>(s[n][k][0], s[n][k][1]);
                packed[2 * k + 1] = both<DT>(s[n][k][2], s[n][k][3]);
            }
            const short8_t p = __builtin_bit_cast(short8_t, packed);
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) out[n][d] = mfma16<DT>(T::columns16(mine, d, lane), p, out[n][d] * times);
        }
    }
    // The waves' sums, relative to the block's largest score: 16 rows at a time, each thread adds four elements of a row, wave by wave.
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        sum[n] = sum_of_quads(sum[n]);
        if (g == 0) {
            of_waves[w][n * 16 + of16][0] = most[n];
            of_waves[w][n * 16 + of16][1] = sum[n];
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r16 = n * 16 + of16;
        float all_most = -INFINITY, all_sum = 0.0f;
        for (int v = 0; v < WAVES; ++v) all_most = fmaxf(all_most, of_waves[v][r16][0]);
        const float base = all_most == -INFINITY ? 0.0f : all_most;
        for (int v = 0; v < WAVES; ++v) all_sum += of_waves[v][r16][1] * exp2_((of_waves[v][r16][0] - base) * unit);
        const float times = exp2_((most[n] - base) * unit);              // 0 where this wave saw nothing
        float *const mine_out = reinterpret_cast<float *>(mine);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) *reinterpret_cast<f32x4 *>(mine_out + of16 * HD + d * 16 + 4 * g) = out[n][d] * times;
        if (w == 0 && g == 0) {
            if (f.shares > 1) {
                f.stats[((int64_t)blockIdx.x * ROWS + r16) * 2] = all_most;
                f.stats[((int64_t)blockIdx.x * ROWS + r16) * 2 + 1] = all_sum;
            } else if (a.stats && there[n]) {
                store_stats<DT, BIAS>(a, (int64_t)seq.q0 + (rows_before + r16) / group, head[n], all_most, all_sum);
            }
        }
        __syncthreads();
        for (int x = threadIdx.x; x < 16 * HD / 4; x += 64 * WAVES) {
            const int row = x / (HD / 4), c = x % (HD / 4) * 4, of_rows = rows_before + n * 16 + row;
            f32x4 all{};
#pragma unroll
            for (int v = 0; v < WAVES; ++v) all += *reinterpret_cast<const f32x4 *>(values[v] + x * 16);
            if (f.shares > 1) {
                *reinterpret_cast<f32x4 *>(f.sums + ((int64_t)blockIdx.x * ROWS + n * 16 + row) * HD + c) = all;
            } else if (of_rows < rows && c < a.hd) {
                float most_of = -INFINITY, sum_of = 0.0f;
                for (int v = 0; v < WAVES; ++v) most_of = fmaxf(most_of, of_waves[v][n * 16 + row][0]);
                const float base_of = most_of == -INFINITY ? 0.0f : most_of;
                for (int v = 0; v < WAVES; ++v) sum_of += of_waves[v][n * 16 + row][1] * exp2_((of_waves[v][n * 16 + row][0] - base_of) * unit);
                store4<DT>(a.out.of((int64_t)seq.q0 + of_rows / group, kv * group + of_rows % group), c, a.hd, all, sum_of > 0.0f ? 1.0f / sum_of : sum_of);
            }
        }
        __syncthreads();                    // the next 16 rows come to the same place
    }
}

// Adds the shares of a row, in order: a wave a row.  (4 tokens of 32 heads, 16 shares: 5 us, a launch and two loads behind each other.)
template <int DT, int HD, bool BIAS, int NT>
__global__ __launch_bounds__(256) void k_attend_join(Attn a, Few f) {
    constexpr int ROWS = 16 * NT, EACH = HD / 64;
    const int lane = threadIdx.x & 63;
    const int64_t work = (int64_t)blockIdx.x * 4 + wave_of();                // [sequence, key head][row tile][row]
    const int r = (int)(work % ROWS), row_tile = (int)(work / ROWS % f.row_tiles);
    const int64_t of_kv = work / ROWS / f.row_tiles;
    const int kv = (int)(of_kv % a.kv_heads), group = a.heads / a.kv_heads, of_rows = row_tile * ROWS + r;
    // k_attend's rows are a head's tokens, k_attend_few's a token's heads
    const int token = ROWS == QUERIES ? row_tile / group * QUERIES + r : of_rows / group, head = kv * group + (ROWS == QUERIES ? row_tile : of_rows) % group;
    if (of_kv / a.kv_heads >= a.batch) return;
    const Sequence seq(a, (int)(of_kv / a.kv_heads));
    if (token >= seq.nq) return;
    const float unit = BIAS ? LOG2E : a.scale * LOG2E;
    const int64_t block = (of_kv * f.row_tiles + row_tile) * f.shares;
    const float *const stats = f.stats + (block * ROWS + r) * 2, *const sums = f.sums + (block * ROWS + r) * HD + lane * EACH;
    // a lane has every 64th share's part in the sum
    float most = -INFINITY, sum = 0.0f, out[EACH] = {};
    for (int s = lane; s < f.shares; s += 64) most = fmaxf(most, stats[(int64_t)s * ROWS * 2]);
#pragma unroll
    for (int n = 1; n < 64; n *= 2) most = fmaxf(most, __shfl_xor(most, n));
    const float base = most == -INFINITY ? 0.0f : most;
    for (int s0 = 0; s0 < f.shares; s0 += 64) {
        const int mine = s0 + lane < f.shares ? s0 + lane : f.shares - 1, here = f.shares - s0 < 64 ? f.shares - s0 : 64;
        const float of_share = exp2_((stats[(int64_t)mine * ROWS * 2] - base) * unit), total = stats[(int64_t)mine * ROWS * 2 + 1];
        for (int s = 0; s < here; s += 8) {                 // eight shares in flight
            float part[8][EACH];
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int e = 0; e < EACH; ++e) part[u][e] = sums[(int64_t)(s0 + (s + u < here ? s + u : here - 1)) * ROWS * HD + e];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int of = s + u < here ? s + u : here - 1;
                const float times = s + u < here ? __shfl(of_share, of) : 0.0f;
                sum += __shfl(total, of) * times;
#pragma unroll
                for (int e = 0; e < EACH; ++e) out[e] += part[u][e] * times;
            }
        }
    }
    const float times = sum > 0.0f ? 1.0f / sum : sum;
    const int64_t row = (int64_t)seq.q0 + token;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
        if (lane * EACH + e < a.hd) store_one<DT>(a.out.of(row, head), lane * EACH + e, out[e] * times);
    if (a.stats && lane == 0) store_stats<DT, BIAS>(a, row, head, most, sum);
}

// ---------------------------------------------------------------- host
struct Plan {
    bool few;
    int tiles_of_rows, row_tiles, shares;            // few: 16-row tiles of a block; row tiles of a key head; shares of the keys
    int64_t blocks, sums, stats, bytes;
};

Plan plan_of(const paro_attn_t &d) {
    Plan p{};
    const int64_t group = d.heads / d.kv_heads;
    p.few = d.len_q <= FEW;
    if (!p.few) {
        p.blocks = ceil_div(d.len_q, QUERIES) * d.heads * d.batch;
        const auto copy = [&](int64_t ld, int64_t head) {
            if (!fills_take(ld ? ld : d.kv_heads * d.head_dim, head ? head : d.head_dim, d.head_dim)) p.bytes += copy_bytes(d, d.len_k, d.kv_heads);
        };
        copy(d.ld_k, d.head_k);
        copy(d.ld_v, d.head_v);
        // Shares of 1024 keys and more, for two blocks a compute unit; by eights, where there are as many.
        const int64_t span = d.window ? std::min<int64_t>(d.len_k, std::min<int64_t>(d.window, d.len_k) + QUERIES + std::min<int64_t>(d.sinks, d.len_k)) : d.len_k;
        p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / std::max<int64_t>(1, p.blocks), span / (32 * KEYS)), MOST_SHARES));
        if (p.shares > 8) p.shares = p.shares / 8 * 8;
        p.row_tiles = (int)(ceil_div(d.len_q, QUERIES) * group);
        p.blocks *= p.shares;
        if (p.shares > 1) {
            p.sums = p.bytes;
            p.stats = p.sums + p.blocks * QUERIES * (d.head_dim <= 64 ? 64 : 128) * 4;
            p.bytes = p.stats + p.blocks * QUERIES * 8;
        }
        return p;
    }
    const int64_t rows = std::max<int64_t>(1, d.len_q * group), head_dim = d.head_dim <= 64 ? 64 : 128;
    p.tiles_of_rows = rows <= 16 ? 1 : 2;
    p.row_tiles = (int)ceil_div(rows, 16 * p.tiles_of_rows);
    const int64_t whole = d.batch * d.kv_heads * p.row_tiles, waves = few_waves((int)head_dim, p.tiles_of_rows);
    const int64_t span = d.window ? std::min<int64_t>(d.len_k, std::min<int64_t>(d.window, d.len_k) + d.len_q + std::min<int64_t>(d.sinks, d.len_k)) : d.len_k;
    // Eight waves a compute unit, sixteen over long caches (4 of 50000 to 100000 keys, 8 key heads of 128: 272 us, so 259); each of eight has three tiles of keys at least, as a
    // second launch costs what three take, each of sixteen twelve (32 sequences with a window of 1024 in 512 blocks 38 us, in 256 27).
    const auto shares = [&](int64_t all, int64_t tiles) { return std::min<int64_t>(ceil_div(all / waves, whole), ceil_div(span, tiles * waves * FEW_KEYS)); };
    p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(std::max(shares(2048, 3), shares(4096, 12)), MOST_SHARES));
    p.blocks = whole * p.shares;
    if (p.shares > 1) {
        p.stats = p.blocks * 16 * p.tiles_of_rows * head_dim * 4;
        p.bytes = p.stats + p.blocks * 16 * p.tiles_of_rows * 8;
    }
    return p;
}

template <int DT, int HD, bool BIAS>
void launch(const Attn &a, const Plan &p, char *workspace, hipStream_t st) {
    const Few f{p.shares, p.row_tiles, reinterpret_cast<float *>(workspace + p.sums), reinterpret_cast<float *>(workspace + p.stats)};
    if (!p.few) {
        if (p.shares > 1) {
            hipLaunchKernelGGL((k_attend<DT, HD, BIAS, true>), dim3((unsigned)p.blocks), dim3(256), 0, st, a, f);
            hipLaunchKernelGGL((k_attend_join<DT, HD, BIAS, QUERIES / 16>), dim3((unsigned)(p.blocks / p.shares * (QUERIES / 4))), dim3(256), 0, st, a, f);
        } else {
            hipLaunchKernelGGL((k_attend<DT, HD, BIAS, false>), dim3((unsigned)p.blocks), dim3(256), 0, st, a, f);
        }
        return;
    }
    const unsigned joins = (unsigned)(p.blocks / p.shares * 4 * p.tiles_of_rows);
    if (p.tiles_of_rows == 1) {
        hipLaunchKernelGGL((k_attend_few<DT, HD, BIAS, 1>), dim3((unsigned)p.blocks), dim3(64 * few_waves(HD, 1)), 0, st, a, f);
        if (p.shares > 1) hipLaunchKernelGGL((k_attend_join<DT, HD, BIAS, 1>), dim3(joins), dim3(256), 0, st, a, f);
    } else {
        hipLaunchKernelGGL((k_attend_few<DT, HD, BIAS, 2>), dim3((unsigned)p.blocks), dim3(64 * few_waves(HD, 2)), 0, st, a, f);
        if (p.shares > 1) hipLaunchKernelGGL((k_attend_join<DT, HD, BIAS, 2>), dim3(joins), dim3(256), 0, st, a, f);
    }
}

}  // namespace

int64_t paro::attn_forward_workspace(const paro_attn_t &d) { return plan_of(d).bytes; }

extern "C" {

int paro_attn(const paro_attn_t *d, const void *q, const void *k, const void *v, const int32_t *q_starts, const int32_t *k_starts, const int32_t *k_lens,
              const void *table, const int32_t *first, void *out, float *stats, void *workspace, int64_t workspace_bytes, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_attn: ";
        int rc;
        if ((rc = check_attn(f, d)) || (rc = check_rows(f, *d, q_starts, k_starts)) || d->batch == 0 || d->len_q == 0) return rc;
        if ((rc = check_inputs(f, *d, q, k, v, q_starts, k_starts, k_lens, table, first)) || (rc = check_array(out, 2, f + "out"))) return rc;
        if (stats && (rc = check_array(stats, 4, f + "stats"))) return rc;
        const Plan p = plan_of(*d);
        const int threads = p.few ? 64 * few_waves(d->head_dim <= 64 ? 64 : 128, p.tiles_of_rows) : 256;
        if ((rc = check_room(f, p.bytes, workspace, workspace_bytes)) || (rc = check_launch(f, p.blocks, threads))) return rc;
        Attn a = attn_of(*d, q, k, v, q_starts, k_starts, k_lens, table, first);
        a.out.at = static_cast<char *>(out);
        a.stats = stats;
        a.tiles = (int)ceil_div(d->len_q, QUERIES);
        a.bunch = bunch_of(a.tiles * (d->heads / d->kv_heads));
        hipStream_t st = static_cast<hipStream_t>(stream);
        char *ws = static_cast<char *>(workspace);
        if (!p.few) {
            if ((rc = check_aligned(f, a.k, a.hd, "k")) || (rc = check_aligned(f, a.v, a.hd, "v"))) return rc;
            Copying copying(ws, 0);
            a.copied_k = copying.take(*d, a.keys, d->len_k, d->kv_heads, true);
            a.copied_v = copying.take(*d, a.values, d->len_k, d->kv_heads, true);
            if ((rc = check_launch(f, copying.blocks(a), 256))) return rc;
            copying.launch(a, st);
        }
#define PARO_FORWARD(DT, HD, BIAS) launch<DT, HD, BIAS>(a, p, ws, st)
        PARO_BY_FORM(PARO_FORWARD);
#undef PARO_FORWARD
        PARO_LAUNCHED("paro_attn");
        return PARO_OK;
    });
}

}  // extern "C"
