// Gradient of the attention with a sliding window, sinks and a relative position bias (gfx950).  With P = softmax(s), from dout and the stored out and
// statistics of the rows:
//
//   D_i = dout_i . out_i,  dP_ij = dout_i . v_j,  dS_ij = P_ij (dP_ij - D_i)
//   dv_j = sum_i P_ij dout_i,  dk_j = scale sum_i dS_ij q_i,  dq_i = scale sum_j dS_ij k_j,  dtable[b] = sum of dS_ij over bucket(p_i - j) = b
//
// Two passes over the pairs that see each other, each of which forms P and dP again: grad_kv goes over the queries and keeps dk and dv of 128 keys in registers,
// grad_q over the keys and keeps dq of 128 queries.  That is seven products where five would do, but every sum has one place and one order: no atomics on
// results, the same call gives the same bits.  P and dS are rounded to 16 bits for the products; as in the forward pass, a product's result is
// the next one's operand as it stands.  fp16: P is multiplied by 2^15; dS by a power of two that brings twice the largest |dout_i| |v_j| to at most 2^15, so that none
// overflows and the small ones keep their bits.
#include "attn.hpp"

namespace {

constexpr int BLOCK = 128;                   // keys of a grad_kv block, queries of a grad_q block: 32 a wave
constexpr int Q_STEP = 32;                   // queries of a tile
constexpr int MOST_SHARES = 64;
template <int DT>
constexpr float SHIFT = DT == PARO_F16 ? 15.0f : 0.0f;

struct Grad {
    Attn a;
    Rows dout, dq, dk, dv;
    Rows queries, douts;                     // q and dout as the fills take them: themselves, or copies, of sequence b from row b len_q on
    bool copied_q, copied_o;
    float *base, *dots;                      // [head][rows_q]: P = exp2(s * LOG2E - base), or, where the base is large in size, from the statistics (see peak_of); D
    int *large;                              // [4 heads][16 rows]: whether the base of one is
    float *largest;                          // of fp16: the largest |dout_i|^2 and |v_j|^2 of each block of k_dots, of rows that see each other
    float *times;                            // of fp16: what dS is multiplied by, and the inverse
    float *partial;                          // of shared key tiles: [slot][dk, dv][128][HD]
    float *of_table;                         // [head][sequence][tile of queries][bucket]
    char *dtable;
    int blocks_q, blocks_v, blocks_heads;    // of k_dots
    int key_tiles, sink_tiles, shares, sink_shares, slots, bunch_kv;      // of a sequence's key head; sink_tiles: the first ones, whose keys are sinks
};

// ---------------------------------------------------------------- statistics of the rows
constexpr int DOT_ROWS = 16, DOT_HEADS = 8, FLAG_HEADS = 64 / DOT_ROWS;      // heads of a wave, whose rows have one flag

template <int HD>
__device__ __forceinline__ float over_lanes(float x) {       // of HD / 8 lanes side by side
#pragma unroll
    for (int n = 1; n < HD / 8; n *= 2) x += __shfl_xor(x, n);
    return x;
}
// D, and what P is formed from, of 16 rows of 8 heads; blocks behind those of the queries: the values' largest row, of those that some query sees.  Reads dout and out once: 8192
// tokens of 32 heads of 128 30 us at best, 4.6 TB/s.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_dots(Grad g) {
    const Attn &a = g.a;
    constexpr int LANES = HD / 8, AT_ONCE = 256 / LANES, U = DOT_ROWS * DOT_HEADS / AT_ONCE;       // all of a block in flight
    __shared__ float dots[DOT_HEADS][DOT_ROWS + 1], squares[DT == PARO_F16 ? DOT_HEADS : 1][DOT_ROWS + 1];
    const bool of_values = (int)blockIdx.x >= g.blocks_q;
    const unsigned tiles = (of_values ? g.blocks_v : g.blocks_q) / a.batch, block = of_values ? blockIdx.x - g.blocks_q : blockIdx.x;
    const int b = block / tiles, row0 = block % tiles * DOT_ROWS, column = threadIdx.x % LANES * 8, head0 = blockIdx.y * DOT_HEADS;
    const Sequence seq(a, b);
    const int heads = of_values ? a.kv_heads : a.heads, n = !of_values ? seq.nq : seq.nq ? seq.nk : 0;
    const int rows = n - row0 < DOT_ROWS ? n - row0 : DOT_ROWS, items = rows > 0 && head0 < heads ? rows * DOT_HEADS : 0;
    for (int x0 = threadIdx.x / LANES; x0 < items; x0 += U * AT_ONCE) {
        u32x4 u_raw[U], o_raw[U];
        int r[U], head[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * AT_ONCE, at = x < items ? x : items - 1;
            r[u] = at / DOT_HEADS;
            head[u] = head0 + at % DOT_HEADS < heads ? head0 + at % DOT_HEADS : heads - 1;
            if (of_values) {
                u_raw[u] = o_raw[u] = piece_of_head(a.v.of((int64_t)seq.k0 + row0 + r[u], head[u]), column, a.hd, true);
            } else {
                u_raw[u] = piece_of_head(g.dout.of((int64_t)seq.q0 + row0 + r[u], head[u]), column, a.hd, true);
                o_raw[u] = piece_of_head(a.out.of((int64_t)seq.q0 + row0 + r[u], head[u]), column, a.hd, true);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[8], o[8], dot = 0.0f, square = 0.0f;
            unpack<DT>(u_raw[u], x);
            unpack<DT>(o_raw[u], o);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot += x[e] * o[e];
            if constexpr (DT == PARO_F16) {
#pragma unroll
                for (int e = 0; e < 8; ++e) square += x[e] * x[e];
                square = over_lanes<HD>(square);
                if (column == 0) squares[head[u] - head0][r[u]] = square;
            }
            dot = over_lanes<HD>(dot);
            if (column == 0) dots[head[u] - head0][r[u]] = dot;
        }
    }
    __syncthreads();
    const int r = threadIdx.x % DOT_ROWS, head = head0 + threadIdx.x / DOT_ROWS;
    float largest = 0.0f;
    bool large = false;
    if (threadIdx.x < DOT_ROWS * DOT_HEADS && r < rows && head < heads) {
        bool counts;                         // P is zero in rows that see no key, and for keys that no row sees
        if (of_values) {
            const int j = row0 + r;
            counts = j < a.sinks || j >= seq.nk - seq.nq - a.window + 1;
        } else {
            const float *const stats = a.stats + (((int64_t)seq.q0 + row0 + r) * a.heads + head) * 2;
            const float most = stats[0], log_sum = stats[1];
            const int64_t at = (int64_t)head * a.rows_q + seq.q0 + row0 + r;
            const bool empty = most == -INFINITY;
            g.dots[at] = dots[threadIdx.x / DOT_ROWS][r];
            g.base[at] = empty ? INFINITY : __builtin_fmaf(most, LOG2E, log_sum * LOG2E) - SHIFT<DT>;
            counts = !empty;
            large = counts && fabsf(most) > USUAL;
        }
        if constexpr (DT == PARO_F16) {
            const float square = squares[threadIdx.x / DOT_ROWS][r];
            if (counts && square < INFINITY) largest = square;          // a row that is not finite leaves the others' scale alone
        }
    }
    large = __any(large);
    if (!of_values && threadIdx.x < DOT_ROWS * DOT_HEADS && (threadIdx.x & 63) == 0)
        g.large[(int64_t)(head / FLAG_HEADS) * g.blocks_q + blockIdx.x] = large;
    if constexpr (DT == PARO_F16) {
        __shared__ float of_waves[4];
#pragma unroll
        for (int x = 1; x < 64; x *= 2) largest = fmaxf(largest, __shfl_xor(largest, x));
        if ((threadIdx.x & 63) == 0) of_waves[wave_of()] = largest;
        __syncthreads();
        if (threadIdx.x == 0) g.largest[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = fmaxf(fmaxf(of_waves[0], of_waves[1]), fmaxf(of_waves[2], of_waves[3]));
    }
}
// |dP - D| is at most twice the largest |dout_i| |v_j|, as out is a mean of values.  One block: 4 us, a launch and its latency.
__global__ __launch_bounds__(256) void k_times(Grad g) {
    __shared__ float of_waves[2][4];
    float most[2] = {0.0f, 0.0f};
    const int blocks = g.blocks_q + g.blocks_v;
    for (int y = 0; y < g.blocks_heads; ++y)
#pragma unroll 4
        for (int x = threadIdx.x; x < blocks; x += 256) {
            const float v = g.largest[(int64_t)y * blocks + x];
            if (x < g.blocks_q) most[0] = fmaxf(most[0], v);
            else most[1] = fmaxf(most[1], v);
        }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int x = 1; x < 64; x *= 2) most[k] = fmaxf(most[k], __shfl_xor(most[k], x));
        if ((threadIdx.x & 63) == 0) of_waves[k][wave_of()] = most[k];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) most[k] = fmaxf(fmaxf(of_waves[k][0], of_waves[k][1]), fmaxf(of_waves[k][2], of_waves[k][3]));
        const bool usual = most[0] > 0.0f && most[1] > 0.0f;       // of zeros nothing is scaled
        int power = 0;
        if (usual) {
            int e0, e1;
            frexpf(most[0], &e0);                    // most <= 2^e
            frexpf(most[1], &e1);
            power = 14 - (e0 + 1) / 2 - (e1 + 1) / 2 - 1;
            power = power < -100 ? -100 : power > 100 ? 100 : power;
        }
        g.times[0] = ldexpf(1.0f, power);
        g.times[1] = ldexpf(1.0f, -power);
    }
}

// Where scores are large in size (a table's lowest number, or large products), LOG2E times one says too little: P = exp2((s - peak) * LOG2E - log_sum), with s as the forward pass
// had it.  Of a row that sees no key the peak is infinity.
__device__ __forceinline__ float peak_of(float most) { return most == -INFINITY ? INFINITY : most; }
template <int DT>
__device__ __forceinline__ float log_sum_of(float log_sum) { return log_sum * LOG2E - SHIFT<DT>; }

// ---------------------------------------------------------------- dk and dv
struct Share {
    int tile, share, shares, slot;           // slot < 0: the block has the tile to itself
};
__device__ __forceinline__ Share share_of(const Grad &g, int block, int of_kv) {
    Share s;
    const int of_sinks = g.sink_tiles * g.sink_shares;
    if (block < of_sinks) {
        s.shares = g.sink_shares;
        s.tile = block / g.sink_shares;
        s.share = block % g.sink_shares;
    } else {
        s.shares = g.shares;
        s.tile = g.sink_tiles + (block - of_sinks) / g.shares;
        s.share = (block - of_sinks) % g.shares;
    }
    s.slot = s.shares > 1 ? of_kv * g.slots + block : -1;
    return s;
}

template <int HD, bool BIAS>
struct SharedKv {
    __attribute__((aligned(1024))) char tiles[2][2][Q_STEP * Tile<HD>::ROW];   // [buffer][queries, dout]
    __attribute__((aligned(1024))) char values[BLOCK * Tile<HD>::ROW];
    __attribute__((aligned(16))) float rows[2][4][Q_STEP];                     // [buffer][base, dots, of large ones peak, log_sum]
    std::conditional_t<BIAS, Bias, int> bias;
};
template <int DT, int HD, bool BIAS>
__device__ __forceinline__ void grad_kv(const Grad &g, unsigned block, SharedKv<HD, BIAS> &shared) {
    using T = Tile<HD>;
    const Attn &a = g.a;
    auto &tiles = shared.tiles;
    auto &values = shared.values;
    auto &rows = shared.rows;
    auto &bias = shared.bias;
    constexpr int STEPS = HD / 16;
    const int per_kv = g.sink_tiles * g.sink_shares + (g.key_tiles - g.sink_tiles) * g.shares;
    if (block >= (unsigned)(per_kv * a.batch * a.kv_heads)) return;
    const Work work(block, a.batch * a.kv_heads, per_kv, g.bunch_kv, 1);
    const int of_kv = work.unit, kv = of_kv % a.kv_heads, b = of_kv / a.kv_heads;
    const Share share = share_of(g, work.within, of_kv);
    const Sequence seq(a, b);
    const int k0 = share.tile * BLOCK;
    if (k0 >= seq.nk) return;
    const int lane = threadIdx.x & 63, w = wave_of(), h = lane >> 5, off = seq.nk - seq.nq, group = a.heads / a.kv_heads;
    const int of_wave = k0 + w * 32, j = of_wave + (lane & 31);                // the lane's key
    // The tiles of queries that see any of the keys, for each head of the group; and this share of them.
    const int last_key = k0 + BLOCK < seq.nk ? k0 + BLOCK - 1 : seq.nk - 1;
    const int64_t until = k0 < a.sinks ? seq.nq : (int64_t)last_key + a.window - off;
    const int lo = k0 - off > 0 ? k0 - off : 0, hi = until < seq.nq ? (int)until : seq.nq;
    const int tile0 = lo / Q_STEP, per_head = hi > lo ? (hi + Q_STEP - 1) / Q_STEP - tile0 : 0;
    const int64_t all = (int64_t)per_head * group;
    const int from = (int)(all * share.share / share.shares), to = (int)(all * (share.share + 1) / share.shares);

    bool large = false;                       // whether the base of some row is
    {
        const int tiles16 = g.blocks_q / a.batch, first16 = lo / DOT_ROWS, some = hi > lo ? (hi + DOT_ROWS - 1) / DOT_ROWS - first16 : 0;
        for (int y = kv * group / FLAG_HEADS; y <= (kv * group + group - 1) / FLAG_HEADS; ++y)
            for (int x = threadIdx.x; x < some; x += 256) large |= g.large[(int64_t)y * g.blocks_q + b * tiles16 + first16 + x] != 0;
        large = __syncthreads_or(large);
    }
    // The next step's head, and its first query.
    const int64_t row_q = g.copied_q ? (int64_t)b * a.len_q : seq.q0, row_o = g.copied_o ? (int64_t)b * a.len_q : seq.q0;
    const Filled<HD, Q_STEP> fill_q(g.queries.ld, a.hd), fill_o(g.douts.ld, a.hd);
    // What the next step takes: its head and tile of queries, where their rows are, and this thread's number of theirs.
    const int which = threadIdx.x / Q_STEP;
    const float *const of_rows = (which == 0 ? g.base : g.dots) + seq.q0 + threadIdx.x % Q_STEP;
    const int64_t q_step = g.queries.ld * (2 * Q_STEP), o_step = g.douts.ld * (2 * Q_STEP);
    const char *q_at = nullptr, *o_at = nullptr;
    const float *row_at = nullptr;
    float from_row = 0.0f;
    int next_head = 0, next_tile = 0, next_i0 = 0;
    const auto point = [&]() __attribute__((always_inline)) {
        const int head = kv * group + next_head;
        next_i0 = (tile0 + next_tile) * Q_STEP;
        q_at = g.queries.of(row_q + next_i0, head);
        o_at = g.douts.of(row_o + next_i0, head);
        row_at = of_rows + (int64_t)head * a.rows_q + next_i0;
    };
    const auto load = [&](auto buffer, auto large_) __attribute__((always_inline)) {
        const int left = seq.nq - 1 - next_i0 - (int)threadIdx.x % Q_STEP;               // rows behind this thread's
        if (which < 2) {
            const float x = row_at[left < 0 ? left : 0];
            from_row = left >= 0 ? x : which == 0 ? INFINITY : 0.0f;
        } else if (large_ && which < 4) {
            const int i = next_i0 + (int)threadIdx.x % Q_STEP;
            const float x = a.stats[(((int64_t)seq.q0 + (left < 0 ? i + left : i)) * a.heads + kv * group + next_head) * 2 + which - 2];
            from_row = which == 2 ? left >= 0 ? peak_of(x) : INFINITY : log_sum_of<DT>(x);
        }
        const u32x4 q_from = fill_q.descriptor(q_at), o_from = fill_o.descriptor(o_at);
        if (next_i0 + Q_STEP <= seq.nq && next_i0 >= -off) {
            fill_q.whole(q_from, tiles[buffer][0]);
            fill_o.whole(o_from, tiles[buffer][1]);
        } else {
            const auto holds = [&](int r) { return next_i0 + r < seq.nq && next_i0 + r >= -off; };       // what stands in front of the first key is of no account
            fill_q.held(q_from, tiles[buffer][0], holds);
            fill_o.held(o_from, tiles[buffer][1], holds);
        }
    };
    Distances by_distance{}, next_distance{};
    int of_head = -1;
    const auto lowest_of = [&](int i0) { return off + i0 - (k0 + BLOCK - 1); };
    const auto stage = [&](auto buffer, auto large_) __attribute__((always_inline)) {
        if (threadIdx.x < (large_ ? 4 : 2) * Q_STEP) rows[buffer][threadIdx.x / Q_STEP][threadIdx.x % Q_STEP] = from_row;
        if constexpr (BIAS) {
            const int head = kv * group + next_head;
            if (head != of_head) {
                __syncthreads();                                // the last head's tiles are done with its bias
                bias.load(a, head);
                __syncthreads();
                of_head = head;
                next_distance.begin(bias, a.buckets);           // read behind the next step's barrier
                __syncthreads();
            }
            next_distance.look_up(bias, lowest_of(next_i0), buffer, a.buckets);
        }
    };

    // The wave's keys stay in registers, its values (two blocks a compute unit leave no registers for them) in shared memory.
    short8_t keys[STEPS];
    {
        const int at = j < seq.nk ? j : seq.nk - 1;
        const char *const key = a.k.of((int64_t)seq.k0 + at, kv), *const value = a.v.of((int64_t)seq.k0 + at, kv);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            keys[s] = __builtin_bit_cast(short8_t, piece_of_head(key, s * 16 + h * 8, a.hd, j < seq.nk));
            *reinterpret_cast<u32x4 *>(values + w * 32 * T::ROW + T::at(lane & 31, 2 * s + h)) = piece_of_head(value, s * 16 + h * 8, a.hd, j < seq.nk);
        }
    }
    const float unit = a.scale * LOG2E, times = DT == PARO_F16 ? g.times[0] * 0x1p-15f : 1.0f;
    f32x16 dk[HD / 32] = {}, dv[HD / 32] = {};
    constexpr std::integral_constant<int, 0> b0{};
    constexpr std::integral_constant<int, 1> b1{};
    int left = to - from;
    const auto step = [&](auto buffer_, auto other, auto large_) __attribute__((always_inline)) {
        constexpr int buffer = buffer_;
        constexpr bool LARGE = large_;
        const int i0 = next_i0, first = off + i0;
        const bool more = --left > 0;
        by_distance = next_distance;
        next_i0 += Q_STEP;
        q_at += q_step;
        o_at += o_step;
        row_at += Q_STEP;
        if (++next_tile == per_head) {
            next_tile = 0;
            ++next_head;
            point();
        }
        arrived<0>();                        // this step's tiles; and all waves have left the last step's
        if (more) load(other, large_);
        const char *const queries = tiles[buffer][0], *const douts = tiles[buffer][1];
        const bool none = first + Q_STEP - 1 < of_wave || (first - (of_wave + 31) >= a.window && of_wave >= a.sinks);
        if (!none) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int c = 0; c < STEPS; ++c) s = mfma32<DT>(T::rows(queries, 0, c, lane), keys[c], s);
#pragma unroll
            for (int c = 0; c < STEPS; ++c) dp = mfma32<DT>(T::rows(douts, 0, c, lane), T::rows(values, w * 32, c, lane), dp);
            const bool every = first >= of_wave + 31 && (first + Q_STEP - 1 - of_wave < a.window || of_wave + 31 < a.sinks);
            const bool far = BIAS && by_distance.usual && by_distance.beyond(lowest_of(i0));
            if constexpr (BIAS) {
                if (!far) {
                    const float *const at = by_distance.values(bias, lowest_of(i0), buffer) + BLOCK - 1 - (w * 32 + (lane & 31)) + 4 * h;
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], a.scale, at[8 * (e / 4) + e % 4]);
                }
            }
            if (!every) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!sees(first + 8 * (e / 4) + 4 * h + e % 4, j, a.window, a.sinks)) s[e] = -INFINITY;
            }
            const float by = BIAS && !far ? LOG2E : unit, plus = BIAS && far ? by_distance.far * LOG2E : 0.0f;
            if constexpr (LARGE) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int r = 8 * (e / 4) + 4 * h + e % 4;
                    const float score = !BIAS ? s[e] * a.scale : far ? __builtin_fmaf(s[e], a.scale, by_distance.far) : s[e], peak = rows[buffer][2][r];
                    s[e] = peak < INFINITY ? exp2_(__builtin_fmaf(score - peak, LOG2E, -rows[buffer][3][r])) : 0.0f;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 base = *reinterpret_cast<const f32x4 *>(rows[buffer][0] + 2 * e + 4 * h);
#pragma unroll
                    for (int x = 0; x < 4; ++x) s[e + x] = exp2_(__builtin_fmaf(s[e + x], by, BIAS ? plus - base[x] : -base[x]));
                }
            }
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f32x4 dot = *reinterpret_cast<const f32x4 *>(rows[buffer][1] + 2 * e + 4 * h);
#pragma unroll
                for (int x = 0; x < 4; ++x) dp[e + x] = s[e + x] * (DT == PARO_F16 ? (dp[e + x] - dot[x]) * times : dp[e + x] - dot[x]);
            }
            if (!every) {                        // what a key that is not seen holds is of no account
#pragma unroll
                for (int e = 0; e < 16; ++e) dp[e] = s[e] == 0.0f ? 0.0f : dp[e];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const short8_t p = pack8<DT>(s, 8 * k), ds = pack8<DT>(dp, 8 * k);
#pragma unroll
                for (int d = 0; d < HD / 32; ++d) {
                    dv[d] = mfma32<DT>(T::columns(douts, k * 16, d, lane), p, dv[d]);
                    dk[d] = mfma32<DT>(T::columns(queries, k * 16, d, lane), ds, dk[d]);
                }
            }
        }
        if (more) stage(other, large_);
    };
    if (from < to) {
        next_head = from / per_head;
        next_tile = from % per_head;
        point();
        const auto steps = [&](auto large_) __attribute__((always_inline)) {
            load(b0, large_);
            stage(b0, large_);
            while (left > 0) {
                step(b0, b1, large_);
                if (left > 0) step(b1, b0, large_);
            }
        };
        if (large) steps(std::true_type{});
        else steps(std::false_type{});
    }
    if (share.slot >= 0) {
        float *const at = g.partial + ((int64_t)share.slot * 2 * BLOCK + w * 32 + (lane & 31)) * HD + 4 * h;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                *reinterpret_cast<f32x4 *>(at + d * 32 + 2 * e) = f32x4{dk[d][e], dk[d][e + 1], dk[d][e + 2], dk[d][e + 3]};
                *reinterpret_cast<f32x4 *>(at + BLOCK * HD + d * 32 + 2 * e) = f32x4{dv[d][e], dv[d][e + 1], dv[d][e + 2], dv[d][e + 3]};
            }
        return;
    }
    const float of_dk = DT == PARO_F16 ? a.scale * g.times[1] : a.scale, of_dv = DT == PARO_F16 ? 0x1p-15f : 1.0f;
    char *const to_k = g.dk.of((int64_t)seq.k0 + j, kv), *const to_v = g.dv.of((int64_t)seq.k0 + j, kv);
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) {
        store_row32<DT>(to_k, d * 32, a.hd, dk[d], of_dk, j < seq.nk);
        store_row32<DT>(to_v, d * 32, a.hd, dv[d], of_dv, j < seq.nk);
    }
}

// Adds the shares of a tile of keys, in order: eight rows of dk or dv a block.  Memory: 16 MiB 7 us.
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_grad_join(Grad g) {
    const Attn &a = g.a;
    constexpr int ROWS = 256 / (HD / 4);
    const int joined = g.shares > 1 ? g.key_tiles : g.sink_tiles;
    const int of_kv = blockIdx.x / joined, tile = blockIdx.x % joined, kv = of_kv % a.kv_heads, b = of_kv / a.kv_heads;
    const Sequence seq(a, b);
    const int r = blockIdx.y * ROWS + threadIdx.x / (HD / 4), c = threadIdx.x % (HD / 4) * 4, j = tile * BLOCK + r;
    const bool of_v = blockIdx.z;
    if (j >= seq.nk) return;
    const bool sinks = tile < g.sink_tiles;
    const int shares = sinks ? g.sink_shares : g.shares;
    const int64_t slot = (int64_t)of_kv * g.slots + (sinks ? tile * g.sink_shares : g.sink_tiles * g.sink_shares + (tile - g.sink_tiles) * g.shares);
    const float *at = g.partial + ((slot * 2 + of_v) * BLOCK + r) * HD + c;
    f32x4 sum = {};
#pragma unroll 8
    for (int s = 0; s < shares; ++s) sum += *reinterpret_cast<const f32x4 *>(at + (int64_t)s * (2 * BLOCK * HD));
    sum *= of_v ? (DT == PARO_F16 ? 0x1p-15f : 1.0f) : DT == PARO_F16 ? a.scale * g.times[1] : a.scale;
    char *const to = (of_v ? g.dv : g.dk).of((int64_t)seq.k0 + j, kv);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < a.hd) store_one<DT>(to, c + e, sum[e]);
}

// ---------------------------------------------------------------- dq, and the table's gradient
template <int HD, bool BIAS>
struct SharedQ {
    static constexpr int KEYS = 32, RING = !BIAS ? 4 : HD == 128 ? 3 : 2;       // so that two blocks (of short heads three) go into the shared memory
    static constexpr int DISTANCES = 32 + KEYS, SQUARE = 36;
    static_assert(NEAR + EDGE >= 4 * MAX_BUCKETS, "the waves' buckets take the place of the distances");
    __attribute__((aligned(1024))) char tiles[RING][2][KEYS * Tile<HD>::ROW];   // [part of the ring][keys, values]
    __attribute__((aligned(16))) float squares[BIAS ? 4 : 1][BIAS ? 32 * SQUARE : 4];      // [wave]: 32 x 32 of dS
    float diagonals[BIAS ? 4 : 1][DISTANCES];                                   // [wave]: sums of dS along a distance, of one tile
    float sums[BIAS ? NEAR + EDGE : 1], far_sums[4];                            // of the block: by distance; where the bias is not there for every one, [wave][bucket]
    std::conditional_t<BIAS, Bias, int> bias;
};
template <int DT, int HD, bool BIAS>
__device__ __forceinline__ void grad_q(const Grad &g, unsigned block, SharedQ<HD, BIAS> &shared) {
    using T = Tile<HD>;
    using S = SharedQ<HD, BIAS>;
    const Attn &a = g.a;
    constexpr int KEYS = S::KEYS, RING = S::RING, STEPS = HD / 16, DISTANCES = S::DISTANCES, SQUARE = S::SQUARE;
    auto &tiles = shared.tiles;
    auto &squares = shared.squares;
    auto &diagonals = shared.diagonals;
    auto &sums = shared.sums;
    auto &far_sums = shared.far_sums;
    auto &bias = shared.bias;
    const int group = a.heads / a.kv_heads;
    const Work work(block, a.batch * a.kv_heads, a.tiles * group, a.bunch, group);
    const int kv = work.unit % a.kv_heads, b = work.unit / a.kv_heads, head = kv * group + work.within % group;
    const int tile = a.tiles - 1 - work.within / group, i0 = tile * BLOCK;             // the longest first
    const bool want = BIAS && g.dtable;
    float *const of_table = g.of_table + (((int64_t)head * a.batch + b) * a.tiles + tile) * a.buckets;
    const Sequence seq(a, b);
    if (i0 >= seq.nq) {
        if (want)
            for (int x = threadIdx.x; x < a.buckets; x += 256) of_table[x] = 0.0f;
        return;
    }
    const int lane = threadIdx.x & 63, w = wave_of(), h = lane >> 5;
    const int off = seq.nk - seq.nq, first = i0 + off, last = (i0 + BLOCK < seq.nq ? i0 + BLOCK : seq.nq) - 1 + off;
    const Seen<KEYS> seen(a, first, last);
    const int of_wave = first + w * 32, place = of_wave + (lane & 31), i = i0 + w * 32 + (lane & 31);
    const int64_t row_k = a.copied_k ? (int64_t)b * a.len_k : seq.k0, row_v = a.copied_v ? (int64_t)b * a.len_k : seq.k0;
    const char *const keys_at = a.keys.of(row_k, kv), *const values_at = a.values.of(row_v, kv);
    const int64_t k_step = a.keys.ld * (2 * KEYS), v_step = a.values.ld * (2 * KEYS);
    const Filled<HD, KEYS> fill_k(a.keys.ld, a.hd), fill_v(a.values.ld, a.hd);
    constexpr int FILLS = 2 * Filled<HD, KEYS>::FILLS;
    Distances by_distance{};
    float far_sum = 0.0f;
    const auto lowest_of = [&](int k0) { return first - (k0 + KEYS - 1); };
    const auto fill = [&](int t, int part) __attribute__((always_inline)) {
        const int tile = seen.tile(t), k0 = tile * KEYS;
        if constexpr (BIAS) by_distance.look_up(bias, lowest_of(k0), part, a.buckets);
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
        for (int x = threadIdx.x; x < NEAR + EDGE; x += 256) sums[x] = 0.0f;
        __syncthreads();
        by_distance.begin(bias, a.buckets);
        __syncthreads();
    }
    short8_t q[STEPS], dout[STEPS];
    const int64_t row = (int64_t)seq.q0 + (i < seq.nq ? i : seq.nq - 1), of_row = (int64_t)head * a.rows_q + row;
    const float base = i < seq.nq ? g.base[of_row] : INFINITY, dot = i < seq.nq ? g.dots[of_row] : 0.0f;
    bool large = false;                       // whether the base of some row is
    {
        const int tiles16 = g.blocks_q / a.batch, x = i0 / DOT_ROWS + threadIdx.x;
        if (threadIdx.x < BLOCK / DOT_ROWS && x < tiles16) large = g.large[(int64_t)(head / FLAG_HEADS) * g.blocks_q + b * tiles16 + x] != 0;
        large = __syncthreads_or(large);
    }
    {
        const int at = i < seq.nq ? i : seq.nq - 1;
        const char *const query = a.q.of((int64_t)seq.q0 + at, head), *const grad = g.dout.of((int64_t)seq.q0 + at, head);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            q[s] = __builtin_bit_cast(short8_t, piece_of_head(query, s * 16 + h * 8, a.hd, i < seq.nq));
            dout[s] = __builtin_bit_cast(short8_t, piece_of_head(grad, s * 16 + h * 8, a.hd, i < seq.nq));
        }
    }
    const float unit = a.scale * LOG2E, times = DT == PARO_F16 ? g.times[0] * 0x1p-15f : 1.0f;
    f32x16 dq[HD / 32] = {};
    const float far_plus = by_distance.far * LOG2E - base;
    // In step t tile t + RING - 1 goes to the part of the ring whose tile all waves have left.  As many steps a round as the ring has parts, so
    // that these are constants.  PLAIN: every query sees the tile whole, and the tile that is brought is there whole.
    const auto step = [&](auto part_, auto plain_, auto large_, int t, int k0, const char *k_at, const char *v_at) __attribute__((always_inline)) {
        constexpr bool LARGE = large_;
        constexpr int part = part_, PLAIN = plain_, coming = (part + RING - 1) % RING;
        arrived<(RING - 2) * FILLS>();
        if constexpr (PLAIN) {
            fill_k.whole(fill_k.descriptor(k_at), tiles[coming][0]);
            fill_v.whole(fill_v.descriptor(v_at), tiles[coming][1]);
            if constexpr (BIAS) by_distance.look_up(bias, lowest_of(k0 + (RING - 1) * KEYS), coming, a.buckets);
        } else {
            if (t + RING - 1 < seen.tiles) fill(t + RING - 1, coming);
            else fill_none(coming);
        }
        const char *const keys = tiles[part][0], *const values = tiles[part][1];
        const bool none = !PLAIN && (k0 > of_wave + 31 || (k0 + KEYS <= of_wave - a.window + 1 && k0 >= a.sinks));
        const bool beyond = BIAS && by_distance.beyond(lowest_of(k0)), far = beyond && by_distance.usual;
        if (want && !beyond)
            for (int x = lane; x < DISTANCES; x += 64) diagonals[BIAS ? w : 0][x] = 0.0f;
        if (!none) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int c = 0; c < STEPS; ++c) s = mfma32<DT>(T::rows(keys, 0, c, lane), q[c], s);
#pragma unroll
            for (int c = 0; c < STEPS; ++c) dp = mfma32<DT>(T::rows(values, 0, c, lane), dout[c], dp);
            if constexpr (BIAS) {
                if (!far) {
                    const float *const at = by_distance.values(bias, lowest_of(k0), part) + (place - first) + 4 - 4 * h;
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = __builtin_fmaf(s[e], a.scale, at[27 - (8 * (e / 4) + e % 4)]);
                }
            }
            const bool every = PLAIN || (k0 + KEYS - 1 <= of_wave && (k0 > of_wave + 31 - a.window || k0 + KEYS <= a.sinks));
            if (!every) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!sees(place, k0 + 8 * (e / 4) + 4 * h + e % 4, a.window, a.sinks)) s[e] = -INFINITY;
            }
            if constexpr (LARGE) {               // the row's numbers are read again in each step, as registers are few
                const float *const stats = a.stats + (row * a.heads + head) * 2;
                const float peak = i < seq.nq ? peak_of(stats[0]) : INFINITY, log_sum = log_sum_of<DT>(stats[1]);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float score = !BIAS ? s[e] * a.scale : far ? __builtin_fmaf(s[e], a.scale, by_distance.far) : s[e];
                    s[e] = peak < INFINITY ? exp2_(__builtin_fmaf(score - peak, LOG2E, -log_sum)) : 0.0f;
                }
            } else {
                const float by = BIAS && !far ? LOG2E : unit, plus = BIAS && far ? far_plus : -base;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = exp2_(__builtin_fmaf(s[e], by, plus));
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) dp[e] = s[e] * (DT == PARO_F16 ? (dp[e] - dot) * times : dp[e] - dot);
            if (!every) {                        // what a key that is not seen holds is of no account
#pragma unroll
                for (int e = 0; e < 16; ++e) dp[e] = s[e] == 0.0f ? 0.0f : dp[e];
            }
            if constexpr (BIAS) {
                if (want && beyond) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) far_sum += dp[e];
                } else if (want) {
                // Through shared memory (the wave's own, whose accesses go in their order): lane r of a half has of each of its 16 rows the key r in front of
                // the row, modulo 32, which are two distances.  (LDS atomics instead: 8 x 1024 tokens of 12 heads of 64 this kernel 214 us, so 96.)
                float *const square = squares[w];
                asm volatile("" ::: "memory");
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *reinterpret_cast<f32x4 *>(square + (lane & 31) * SQUARE + 2 * e + 4 * h) = f32x4{dp[e], dp[e + 1], dp[e + 2], dp[e + 3]};
                asm volatile("" ::: "memory");
                float near = 0.0f, behind = 0.0f;                       // distances r, and r - 32, from the square's first row and key
                const int r = lane & 31;
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                    const int row = h * 16 + y;
                    const float x = square[row * SQUARE + ((row - r) & 31)];
                    near += row >= r ? x : 0.0f;
                    behind += row >= r ? 0.0f : x;
                }
                near = sum_of_halves(near);
                behind = sum_of_halves(behind);
                // place KEYS - 1 + distance; behind: of r = 0 there is none
                const int place_of = KEYS - 1 + (h ? r - 32 : r);
                asm volatile("" ::: "memory");
                if (!h || r) diagonals[w][place_of] += h ? behind : near;
                asm volatile("" ::: "memory");
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const short8_t ds = pack8<DT>(dp, 8 * k);
#pragma unroll
                for (int d = 0; d < HD / 32; ++d) dq[d] = mfma32<DT>(T::columns(keys, k * 16, d, lane), ds, dq[d]);
            }
        }
        if constexpr (BIAS) {
            if (want && !beyond) {
                __syncthreads();
                // thread x has the distance lowest + x of the tile
                const int x = threadIdx.x, d = lowest_of(k0) + x;
                float sum = 0.0f;
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (x >= v * 32 && x < v * 32 + DISTANCES) sum += diagonals[v][x - v * 32];
                if (by_distance.whole) {
                    if (d >= 0 && x < EDGE) sums[d] += sum;
                } else {
                    // buckets are runs of distances, whose sums the last lane of a run adds
                    const int bucket = d < 0 || x >= EDGE ? -1 : bias.bucket(d, a.buckets);
#pragma unroll
                    for (int n = 1; n < 64; n *= 2) {
                        const float before = __shfl_up(sum, n);
                        const int of = __shfl_up(bucket, n);
                        if (lane >= n && of == bucket) sum += before;
                    }
                    const int next = __shfl_down(bucket, 1);
                    if (bucket >= 0 && (lane == 63 || next != bucket)) sums[w * MAX_BUCKETS + bucket] += sum;
                }
            }
        }
    };
    if (seen.tiles) {
        int plain_from, plain_to;
        seen.plain(a, first, last, plain_from, plain_to);
        for (int t = 0; t < RING - 1; ++t) {
            if (t < seen.tiles) fill(t, t);
            else fill_none(t);
        }
        const auto steps = [&](auto large_) __attribute__((always_inline)) {
            for (int t = 0; t < seen.tiles;) {
                if (t >= plain_from && t + 2 * RING - 2 < plain_to) {
                    int k0 = seen.tile(t) * KEYS;
                    const char *k_at = keys_at + (seen.tile(t) + RING - 1) * k_step, *v_at = values_at + (seen.tile(t) + RING - 1) * v_step;
                    for (; t + 2 * RING - 2 < plain_to; t += RING)
                        static_for<0, RING>([&](auto part) __attribute__((always_inline)) {
                            step(part, std::integral_constant<int, 1>{}, large_, 0, k0, k_at, v_at);
                            k0 += KEYS;
                            k_at += k_step;
                            v_at += v_step;
                        });
                }
                static_for<0, RING>([&](auto part) __attribute__((always_inline)) {
                    if (t < seen.tiles) step(part, std::integral_constant<int, 0>{}, large_, t, seen.tile(t) * KEYS, nullptr, nullptr);
                    ++t;
                });
            }
        };
        if (large) steps(std::true_type{});
        else steps(std::false_type{});
        arrived<0>();                                           // nothing is on its way into the shared memory of the block that comes next
    }
    const float of_dq = DT == PARO_F16 ? a.scale * g.times[1] : a.scale;
    char *const to = g.dq.of((int64_t)seq.q0 + i, head);
#pragma unroll
    for (int d = 0; d < HD / 32; ++d) store_row32<DT>(to, d * 32, a.hd, dq[d], of_dq, i < seq.nq);
    if constexpr (BIAS) {
        if (want) {
#pragma unroll
            for (int x = 1; x < 64; x *= 2) far_sum += __shfl_xor(far_sum, x);
            if (lane == 0) far_sums[w] = far_sum;
            __syncthreads();
            const float back = DT == PARO_F16 ? g.times[1] : 1.0f;
            if (by_distance.whole) {                            // a wave a bucket; the last has what lies beyond too
                for (int x = w; x < a.buckets; x += 4) {
                    const int all = by_distance.far_from + EDGE, from = bias.first[x], until = x + 1 < a.buckets ? bias.first[x + 1] : all;
                    float sum = 0.0f;
                    for (int d = (from > 0 ? from : 0) + lane; d < until && d < all; d += 64) sum += sums[d];
#pragma unroll
                    for (int n = 1; n < 64; n *= 2) sum += __shfl_xor(sum, n);
                    if (x == a.buckets - 1) sum += far_sums[0] + far_sums[1] + far_sums[2] + far_sums[3];
                    if (lane == 0) of_table[x] = sum * back;
                }
            } else {
                for (int x = threadIdx.x; x < a.buckets; x += 256) {
                    float sum = 0.0f;
#pragma unroll
                    for (int v = 0; v < 4; ++v) sum += sums[v * MAX_BUCKETS + x] + (x == a.buckets - 1 ? far_sums[v] : 0.0f);
                    of_table[x] = sum * back;
                }
            }
        }
    }
}

// Both passes in one launch, as neither fills the chip to its end: the first of_kv blocks (a multiple of eight, so that what is one XCD's stays there) have keys,
// the others queries.  (In launches of their own: 1999 tokens of 10 heads of 77 88 + 59 us, so 114.)  8192 tokens of 32 heads of 128, all seen: 1777 us, 1080 TF of the seven
// products; matrix cores busy 56 % of the cycles at 1.77 GHz, shared memory 36 %.  8 x 1024 of 12 heads of 64 with bias 96 us: waves wait half of their cycles, three a SIMD.
// Steps for large scores (see peak_of) are loops of their own, as a question in each step costs registers: 8192 tokens 1862 us the call, so 1801, packed sequences 676, so 634.
template <int DT, int HD, bool BIAS>
__global__ __launch_bounds__(256, HD == 64 ? 3 : 2) void k_grads(Grad g, unsigned of_kv) {
    __shared__ union {
        SharedKv<HD, BIAS> kv;
        SharedQ<HD, BIAS> q;
    } shared;
    if (blockIdx.x < of_kv) grad_kv<DT, HD, BIAS>(g, blockIdx.x, shared.kv);
    else grad_q<DT, HD, BIAS>(g, blockIdx.x - of_kv, shared.q);
}

// Adds the blocks' sums of a head, in order: a thread has every `parts`-th of a bucket.  (64 blocks a head: 4 us, latency.)
template <int DT>
__global__ __launch_bounds__(256) void k_table_grad(Grad g) {
    const Attn &a = g.a;
    __shared__ float sums[256];
    const int head = blockIdx.x, parts = 256 / a.buckets, bucket = threadIdx.x % a.buckets, part = threadIdx.x / a.buckets;
    const int64_t blocks = (int64_t)a.batch * a.tiles;
    const float *const at = g.of_table + (int64_t)head * blocks * a.buckets + bucket;
    float sum = 0.0f;
    if (part < parts) {
#pragma unroll 8
        for (int64_t x = part; x < blocks; x += parts) sum += at[x * a.buckets];
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (part) return;
    for (int x = 1; x < parts; ++x) sum += sums[x * a.buckets + bucket];
    const int64_t to = (int64_t)bucket * a.heads + head;
    if (a.table_dtype == PARO_F32) reinterpret_cast<float *>(g.dtable)[to] = sum;
    else store_one<DT>(g.dtable, to, sum);
}

// ---------------------------------------------------------------- host
struct Plan {
    int blocks_q, blocks_v, blocks_heads, tiles, key_tiles, sink_tiles, shares, sink_shares, slots;
    int64_t kv_blocks, copies, dots, large, largest, times, partial, of_table, bytes;
};

Plan plan_of(const paro_attn_t &d) {
    Plan p{};
    const int64_t group = d.heads / d.kv_heads, hd = d.head_dim <= 64 ? 64 : 128, rows_q = d.rows_q ? d.rows_q : d.batch * d.len_q;
    const int64_t window = d.window && d.window < d.len_k ? d.window : d.len_k;
    p.blocks_q = (int)(ceil_div(d.len_q, DOT_ROWS) * d.batch);
    p.blocks_v = d.dtype == PARO_F16 ? (int)(ceil_div(d.len_k, DOT_ROWS) * d.batch) : 0;
    p.blocks_heads = (int)ceil_div(d.heads, DOT_HEADS);
    p.tiles = (int)ceil_div(d.len_q, BLOCK);
    p.key_tiles = (int)ceil_div(d.len_k, BLOCK);
    // Tiles of keys are shared out where there are few of them, by a reckoning of the time (us): a step of 32 queries takes 1.5 with one block on a compute unit, 2.3 with
    // two, each share four more at its beginning and end; its sums are written and read again.  Those with sinks, which every later query sees, by how many more
    // see them than see others.
    const int64_t whole = std::max<int64_t>(1, (int64_t)p.key_tiles * d.kv_heads * d.batch);
    const int64_t others = std::min<int64_t>(d.len_q, window + BLOCK);
    const double longest = std::max<double>(1.0, (double)ceil_div(others, Q_STEP) * group), usual = d.window ? longest : longest / 2;       // steps
    double least = 0.0;
    for (int shares = 1; shares <= MOST_SHARES; ++shares) {
        const double blocks = (double)whole * shares, rounds = std::ceil(blocks / 512);
        const double steps = rounds > 1 ? usual : longest;
        const double time = rounds * (steps / shares + 4) * (blocks > 256 ? 2.3 : 1.5) + (shares > 1 ? 5 + blocks * hd / 128 * 0.055 : 0.0);
        if (shares == 1 || time < least) {
            p.shares = shares;
            least = time;
        }
    }
    p.sink_tiles = window < d.len_k ? (int)std::min<int64_t>(ceil_div(std::min<int64_t>(d.sinks, d.len_k), BLOCK), p.key_tiles) : 0;
    // (a share's sums take 128 KiB of the workspace)
    p.sink_shares = p.shares;
    if (p.sink_tiles) {
        const int64_t most = std::min<int64_t>(MOST_SHARES, std::max<int64_t>(p.shares, 1024 / (p.sink_tiles * d.kv_heads * d.batch)));
        // (no query, one share: a tile's block writes its zeros)
        p.sink_shares = (int)std::min<int64_t>(p.shares * std::max<int64_t>(1, ceil_div(d.len_q, std::max<int64_t>(1, others))), most);
    }
    const int64_t per_kv = (int64_t)p.sink_tiles * p.sink_shares + (int64_t)(p.key_tiles - p.sink_tiles) * p.shares;
    p.slots = p.shares > 1 ? (int)per_kv : p.sink_shares > 1 ? p.sink_tiles * p.sink_shares : 0;
    p.kv_blocks = per_kv * d.kv_heads * d.batch;
    int64_t at = 0;
    const auto room = [&](int64_t floats) {
        const int64_t was = at;
        at += ceil_div(floats * 4, 256) * 256;
        return was;
    };
    room(rows_q * d.heads);                                                     // base
    p.dots = room(rows_q * d.heads);
    p.large = room((int64_t)p.blocks_q * p.blocks_heads * (DOT_HEADS / FLAG_HEADS));
    p.largest = room(d.dtype == PARO_F16 ? ((int64_t)p.blocks_q + p.blocks_v) * p.blocks_heads : 0);
    p.times = room(2);
    p.partial = room((int64_t)p.slots * d.kv_heads * d.batch * 2 * BLOCK * hd);
    p.of_table = room((int64_t)d.heads * d.batch * p.tiles * d.buckets);
    p.copies = at;
    const auto copy = [&](int64_t ld, int64_t head, int64_t len, int64_t heads) {
        if (!fills_take(ld ? ld : heads * d.head_dim, head ? head : d.head_dim, d.head_dim)) at += copy_bytes(d, len, heads);
    };
    copy(d.ld_q, d.head_q, d.len_q, d.heads);
    copy(d.ld_out, d.head_out, d.len_q, d.heads);
    copy(d.ld_k, d.head_k, d.len_k, d.kv_heads);
    copy(d.ld_v, d.head_v, d.len_k, d.kv_heads);
    p.bytes = at;
    return p;
}

void launch_table_grad(const Grad &g, int dtype, hipStream_t st) {
    if (dtype == PARO_F16) hipLaunchKernelGGL((k_table_grad<PARO_F16>), dim3((unsigned)g.a.heads), dim3(256), 0, st, g);
    else hipLaunchKernelGGL((k_table_grad<PARO_BF16>), dim3((unsigned)g.a.heads), dim3(256), 0, st, g);
}

template <int DT, int HD, bool BIAS>
void launch(const Grad &g, const Plan &p, hipStream_t st) {
    if (p.blocks_q + p.blocks_v) hipLaunchKernelGGL((k_dots<DT, HD>), dim3((unsigned)(p.blocks_q + p.blocks_v), (unsigned)p.blocks_heads), dim3(256), 0, st, g);
    if constexpr (DT == PARO_F16) hipLaunchKernelGGL(k_times, dim3(1), dim3(256), 0, st, g);
    const int64_t of_kv = ceil_div(p.kv_blocks, 8) * 8, of_q = (int64_t)p.tiles * g.a.heads * g.a.batch;
    if (of_kv + of_q) hipLaunchKernelGGL((k_grads<DT, HD, BIAS>), dim3((unsigned)(of_kv + of_q)), dim3(256), 0, st, g, (unsigned)of_kv);
    const int joined = p.shares > 1 ? p.key_tiles : p.sink_shares > 1 ? p.sink_tiles : 0;
    if (joined) hipLaunchKernelGGL((k_grad_join<DT, HD>), dim3((unsigned)(joined * g.a.kv_heads * g.a.batch), BLOCK / (1024 / HD), 2), dim3(256), 0, st, g);
    if (BIAS && g.dtable) launch_table_grad(g, DT, st);
}

}  // namespace

extern "C" {

int64_t paro_attn_workspace(const paro_attn_t *d, int grad) {
    int64_t bytes = 0;
    const int rc = guarded([&]() -> int {
        const int bad = check_attn("paro_attn_workspace: ", d);
        if (!bad) bytes = d->batch == 0 ? 0 : grad ? plan_of(*d).bytes : paro::attn_forward_workspace(*d);
        return bad;
    });
    return rc ? rc : bytes;
}

int paro_attn_grad(const paro_attn_t *d, const void *dout, const void *q, const void *k, const void *v, const void *out, const float *stats,
                   const int32_t *q_starts, const int32_t *k_starts, const int32_t *k_lens, const void *table, const int32_t *first, void *dq, void *dk, void *dv,
                   void *dtable, void *workspace, int64_t workspace_bytes, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_attn_grad: ";
        int rc;
        if ((rc = check_attn(f, d)) || (rc = check_rows(f, *d, q_starts, k_starts))) return rc;
        if (d->batch == 0 && !(d->buckets && dtable)) return PARO_OK;
        if (d->batch && d->len_q &&
            ((rc = check_array(dout, 2, f + "dout")) || (rc = check_array(out, 2, f + "out")) || (rc = check_array(stats, 4, f + "stats")) || (rc = check_array(dq, 2, f + "dq"))))
            return rc;
        if (d->batch && (rc = check_inputs(f, *d, q, k, v, q_starts, k_starts, k_lens, table, first))) return rc;
        if (d->batch && d->len_k && ((rc = check_array(dk, 2, f + "dk")) || (rc = check_array(dv, 2, f + "dv")))) return rc;
        if (d->buckets && dtable && (rc = check_array(dtable, size_of(d->table_dtype), f + "dtable"))) return rc;
        hipStream_t st = static_cast<hipStream_t>(stream);
        if (d->batch == 0) {                     // of a table that nothing has looked at: zeros
            Grad none{};
            none.a = attn_of(*d, q, k, v, q_starts, k_starts, k_lens, table, first);
            none.dtable = static_cast<char *>(dtable);
            launch_table_grad(none, d->dtype, st);
            PARO_LAUNCHED("paro_attn_grad");
            return PARO_OK;
        }
        const Plan p = plan_of(*d);
        if ((rc = check_room(f, p.bytes, workspace, workspace_bytes))) return rc;
        char *ws = static_cast<char *>(workspace);
        const auto floats = [&](int64_t at) { return reinterpret_cast<float *>(ws + at); };
        Grad g{};
        g.a = attn_of(*d, q, k, v, q_starts, k_starts, k_lens, table, first);
        g.a.out.at = static_cast<char *>(const_cast<void *>(out));
        g.a.stats = const_cast<float *>(stats);
        g.a.tiles = p.tiles;
        g.a.bunch = bunch_of(p.tiles * (d->heads / d->kv_heads));
        g.bunch_kv = bunch_of(ceil_div(p.kv_blocks, d->kv_heads * d->batch));
        const auto as = [](Rows like, const void *at) {
            like.at = static_cast<char *>(const_cast<void *>(at));
            return like;
        };
        g.dout = as(g.a.out, dout);
        g.dq = as(g.a.q, dq);
        g.dk = as(g.a.k, dk);
        g.dv = as(g.a.v, dv);
        g.base = floats(0);
        g.dots = floats(p.dots);
        g.large = reinterpret_cast<int *>(ws + p.large);
        g.largest = floats(p.largest);
        g.times = floats(p.times);
        g.partial = floats(p.partial);
        g.of_table = floats(p.of_table);
        g.dtable = static_cast<char *>(dtable);
        g.blocks_q = p.blocks_q;
        g.blocks_v = p.blocks_v;
        g.blocks_heads = p.blocks_heads;
        g.key_tiles = p.key_tiles;
        g.sink_tiles = p.sink_tiles;
        g.shares = p.shares;
        g.sink_shares = p.sink_shares;
        g.slots = p.slots;
        if ((rc = check_aligned(f, g.a.q, g.a.hd, "q")) || (rc = check_aligned(f, g.dout, g.a.hd, "dout")) || (rc = check_aligned(f, g.a.k, g.a.hd, "k")) ||
            (rc = check_aligned(f, g.a.v, g.a.hd, "v")))
            return rc;
        g.queries = g.a.q;
        g.douts = g.dout;
        Copying copying(ws, p.copies);
        g.copied_q = copying.take(*d, g.queries, d->len_q, d->heads, false);
        g.copied_o = copying.take(*d, g.douts, d->len_q, d->heads, false);
        g.a.copied_k = copying.take(*d, g.a.keys, d->len_k, d->kv_heads, true);
        g.a.copied_v = copying.take(*d, g.a.values, d->len_k, d->kv_heads, true);
        if ((rc = check_launch(f, copying.blocks(g.a), 256)) || (rc = check_launch(f, (int64_t)p.blocks_q + p.blocks_v, 256)) ||
            (rc = check_launch(f, p.kv_blocks + 8 + (int64_t)p.tiles * d->heads * d->batch, 256)))
            return rc;
        copying.launch(g.a, st);
#define PARO_BACKWARD(DT, HD, BIAS) launch<DT, HD, BIAS>(g, p, st)
        PARO_BY_FORM(PARO_BACKWARD);
#undef PARO_BACKWARD
        PARO_LAUNCHED("paro_attn_grad");
        return PARO_OK;
    });
}

int paro_rel_buckets(int buckets, int64_t max_distance, int32_t *first) {
    return guarded([&]() -> int {
        const std::string f = "paro_rel_buckets: ";
        if (buckets < 1 || buckets > MAX_BUCKETS) return fail(PARO_EINVAL, f + "buckets must be in [1, 256]");
        const int single = (buckets + 1) / 2, more = buckets - single;
        if (max_distance < single || max_distance >= FAR_AWAY) return fail(PARO_EINVAL, f + "max_distance must be in [(buckets + 1) / 2, 2^30)");
        if (!first) return fail(PARO_EINVAL, f + "first is NULL");
        for (int b = 0; b < single; ++b) first[b] = b;
        // h (D / h)^(k / m), rounded up; where it is a whole number the power in 64 bits may lie to either side of it
        for (int k = 0; k < more; ++k) {
            const long double x = single * std::pow((long double)max_distance / single, (long double)k / more), whole = std::nearbyint(x);
            first[single + k] = (int32_t)(std::fabs(x - whole) < 1e-12L * x ? whole : std::ceil(x));
        }
        return PARO_OK;
    });
}

}  // extern "C"
