// What the attention's forward and backward kernels share (attn.hip, attn_grad.hip): where a sequence lies, which keys a tile of queries sees, tiles
// of rows in shared memory and how the matrix instructions read them, the relative position bias.
//
// With off = keys - queries of a sequence, query i stands at place p = off + i and sees key j where 0 <= j <= p and (p - j < window or j < sinks).
#pragma once

#include <cmath>

#include "operators.hpp"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr int MAX_BUCKETS = 256, MIN_HEAD = 8, MAX_HEAD = 128;
constexpr float USUAL = 1e5f;            // a score in size, up to which LOG2E times it says enough of it
constexpr int FAR_AWAY = 1 << 30;        // a window that holds every key: lengths are at most this

template <int DT>
__device__ __forceinline__ f32x16 mfma32(short8_t a, short8_t b, f32x16 c) {
    if constexpr (DT == PARO_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
template <int DT>
__device__ __forceinline__ f32x4 mfma16(short8_t a, short8_t b, f32x4 c) {
    if constexpr (DT == PARO_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// A value of the lane 32 on (modulo 64) joined with a lane's own: both halves of a wave then have the same.
__device__ __forceinline__ float max_of_halves(float x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}
__device__ __forceinline__ float sum_of_halves(float x) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(both[0]) + __uint_as_float(both[1]);
}

// Blocks go to the eight XCDs in turn.  A unit is the work of a sequence's key head, which reads the same keys and values over and over: it stays on one XCD, to meet
// in its L2, and units go to the XCDs in turn, so that sequences of different lengths even out (runs of a sequence each: packed sequences of 1024 to 2048 tokens
// forward 295 us, so 220); what is left over in the end is shared by all.  An XCD takes its units a bunch at a time, the longest blocks of all of them first, `together`
// (the heads that read a key head) side by side.  (Unit by unit: 8 x 1024 tokens of 12 heads of 64 forward 44 us, so 36, backward 137, so 108; 8192 of 32 heads of 128
// 446 and 1820, so 430 and 1755.  All units at once: 32 x 2048 tokens of 32 heads with a window of 512 forward 1283, as their keys do not fit the
// L2, so 890.  Heads apart: packed sequences 235, so 213.)
struct Work {
    int unit, within;
    __device__ __forceinline__ Work(unsigned block, unsigned units, unsigned of_unit, unsigned bunch, unsigned together) {
        const unsigned whole = units / 8 * 8 * of_unit;
        if (block < whole) {
            const unsigned k = block / 8, g = k / (of_unit * bunch), left = units / 8 - g * bunch, n = (left < bunch ? left : bunch) * together;
            const unsigned r = k - g * (of_unit * bunch), x = r % n;
            unit = (int)((g * bunch + x / together) * 8 + block % 8);
            within = (int)(r / n * together + x % together);
        } else {
            const unsigned rest = block - whole, all = (units % 8) * of_unit, each = all / 8, more = all % 8, xcd = rest % 8;
            const unsigned at = xcd * each + (xcd < more ? xcd : more) + rest / 8;
            unit = (int)(units / 8 * 8 + at / of_unit);
            within = (int)(at % of_unit);
        }
    }
};
// Units of a bunch: two rounds of blocks of an XCD's 32 compute units, four units at least.
inline int bunch_of(int64_t of_unit) { return (int)std::max<int64_t>(4, 128 / std::max<int64_t>(1, of_unit)); }

// Rows of an array of heads: elements from token to token, and from head to head.
struct Rows {
    char *at;
    int64_t ld, head;
    __device__ __forceinline__ char *of(int64_t row, int h) const { return at + (row * ld + h * head) * 2; }
};

struct Attn {
    Rows q, k, v, out;
    Rows keys, values;                 // k and v as the fills take them: themselves, or copies, of sequence b from row b len_k on
    bool copied_k, copied_v;
    const int32_t *q_starts, *k_starts, *k_lens;
    float *stats;
    const void *table;
    const int32_t *first;
    int batch, heads, kv_heads, hd, len_q, len_k, rows_q, rows_k, window, sinks, buckets, table_dtype, tiles, bunch;
    float scale;
};

// Where a sequence's rows lie.  Whatever the arrays on the device hold, its rows are those inside [0, rows_q) and [0, rows_k), and of these the first len_q and len_k.
struct Sequence {
    int q0, nq, k0, nk;
    __device__ __forceinline__ Sequence(const Attn &a, int b) {
        const auto inside = [](int64_t x, int64_t most) { return (int)(x < 0 ? 0 : x > most ? most : x); };
        const int64_t qs = a.q_starts ? a.q_starts[b] : (int64_t)b * a.len_q, ks = a.k_starts ? a.k_starts[b] : (int64_t)b * a.len_k;
        q0 = inside(qs, a.rows_q);
        k0 = inside(ks, a.rows_k);
        const int64_t q_end = a.q_starts ? a.q_starts[b + 1] : qs + a.len_q;
        const int64_t k_end = a.k_lens ? ks + a.k_lens[b] : a.k_starts ? a.k_starts[b + 1] : ks + a.len_k;
        nq = inside((int64_t)inside(q_end, a.rows_q) - q0, a.len_q);
        nk = inside((int64_t)inside(k_end, a.rows_k) - k0, a.len_k);
    }
};

// The tiles of KEYS keys that queries at the places [first, last] see: those with sinks, then those of the windows.  Keys that none of the queries sees are
// not read (others': behind the end, between the sinks and the first window).
template <int KEYS>
struct Seen {
    int end, low, sinks;              // keys [0, sinks) and [low, end)
    int sink_tiles, first_tile, tiles;
    __device__ __forceinline__ Seen(const Attn &a, int first, int last) {
        end = last + 1 > 0 ? last + 1 : 0;
        low = first - a.window + 1 > 0 ? first - a.window + 1 : 0;
        if (low > end) low = end;
        sinks = a.sinks < end ? a.sinks : end;
        first_tile = low / KEYS;
        const int of_sinks = (sinks + KEYS - 1) / KEYS;
        sink_tiles = of_sinks < first_tile ? of_sinks : first_tile;
        tiles = sink_tiles + (end + KEYS - 1) / KEYS - first_tile;
        if (end == 0) tiles = 0;
    }
    // The tiles [from, to) of which every query sees every key.
    __device__ __forceinline__ void plain(const Attn &a, int first, int last, int &from, int &to) const {
        const int cut = last - a.window >= 0 ? (last - a.window) / KEYS + 1 : 0;        // the first tile in all windows
        from = sink_tiles + (cut > first_tile ? cut - first_tile : 0);
        to = first + 1 > 0 ? sink_tiles + (first + 1) / KEYS - first_tile : 0;
    }
    __device__ __forceinline__ int tile(int t) const { return t < sink_tiles ? t : first_tile + t - sink_tiles; }
    __device__ __forceinline__ bool holds_all(int k0) const { return k0 + KEYS <= end && (k0 >= low || k0 + KEYS <= sinks); }
    __device__ __forceinline__ bool holds(int j) const { return j < end && (j >= low || j < sinks); }
};
__device__ __forceinline__ bool sees(int p, int j, int window, int sinks) {
    const int reach = j < sinks ? INT32_MAX : window;
    return (unsigned)(p - j) < (unsigned)reach;
}

// ---------------------------------------------------------------- tiles of rows in shared memory
// HD (64 or 128) elements of 16 bits a row, whatever lies behind the head's own as zeros, in pieces of eight.  The pieces of a row are exchanged by its number such
// that the lanes that read at a time meet all banks, both where they read the same piece of 16 rows and where they read 64 bytes of 4 rows (transposed).
template <int HD>
struct Tile {
    static constexpr int ROW = HD * 2, PIECES = HD / 8;
    static __device__ __forceinline__ int key(int row) {
        if constexpr (HD == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
        else return ((row & 2) << 1) | ((row >> 2) & 3);
    }
    static __device__ __forceinline__ int at(int row, int piece) { return row * ROW + ((piece ^ key(row)) << 4); }

    // Operand with 32 rows of the tile as its rows (or columns), step s of 16 elements: a lane has row lane % 32, elements 8 * (lane / 32) on.
    static __device__ __forceinline__ short8_t rows(const char *tile, int row0, int s, int lane) {
        return *reinterpret_cast<const short8_t *>(tile + row0 * ROW + at(lane & 31, 2 * s + (lane >> 5)));
    }
    // Operand with the elements [32 * d, 32 * d + 32) as its rows and 16 rows of the tile, row0 on, as its steps: lane / 32 = h has of these the rows
    // 4h .. 4h + 3 and 8 + 4h .. 8 + 4h + 3, which is the order in which the result of a product has them.
    static __device__ __forceinline__ short8_t columns(const char *tile, int row0, int d, int lane) {
        const int h = lane >> 5, of16 = lane & 15, row = 4 * h + (of16 >> 2), piece = d * 4 + ((lane >> 4) & 1) * 2 + ((of16 & 3) >> 1);
        const char *lo = tile + row0 * ROW + at(row, piece) + (of16 & 1) * 8, *hi = tile + row0 * ROW + at(row + 8, piece) + (of16 & 1) * 8;
        return joined(lo, hi);
    }
    // The same for elements [16 * d, 16 * d + 16) and 32 rows of the tile: lane / 16 = g has the rows 4g .. 4g + 3 and 16 + 4g .. 16 + 4g + 3.
    static __device__ __forceinline__ short8_t columns16(const char *tile, int d, int lane) {
        const int g = lane >> 4, of16 = lane & 15, row = 4 * g + (of16 >> 2), piece = d * 2 + ((of16 & 3) >> 1);
        const char *lo = tile + at(row, piece) + (of16 & 1) * 8;
        return joined(lo, lo + 16 * ROW);               // rows 16 apart have the same key
    }
    static __device__ __forceinline__ short8_t joined(const char *lo, const char *hi) {
        const short4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)lo);
        const short4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)hi);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Eight elements of a head's row, from `column` on; what lies behind the head: zeros.  One load without a branch: a piece that reaches past the head's end is read
// from eight elements in front of that, and shifted.  (With branches for each element 1999 tokens of 10 heads of 77 took 78 us forward, so 44.)
// The row has to exist also where the piece is not wanted.
__device__ __forceinline__ int column_of(int column, int hd) { return column < hd - 8 ? column : hd - 8; }
__device__ __forceinline__ u32x4 shifted(u32x4 v, int elements) {          // towards the first, by 0 to 7
    if (elements & 4) v = u32x4{v[2], v[3], 0, 0};
    if (elements & 2) v = u32x4{v[1], v[2], v[3], 0};
    if (elements & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbit(i < 3 ? v[i + 1] : 0, v[i], 16);
    }
    return v;
}
__device__ __forceinline__ u32x4 finished(u32x4 v, int column, int hd, bool there) {       // of what was loaded from column_of
    if (hd & 7) v = shifted(v, (column - column_of(column, hd)) & 7);
    there = there && column < hd;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = there ? v[i] : 0;
    return v;
}
__device__ __forceinline__ u32x4 piece_of_head(const char *row, int column, int hd, bool there) {
    return finished(load_piece<PARO_BF16>(row, column_of(column, hd)), column, hd, there);
}
__device__ __forceinline__ void store_piece_of_head(char *row, int column, int hd, u32x4 v) {
    if (column + 8 <= hd) {
        store_piece<PARO_BF16>(row, column, v);
        return;
    }
    uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
#pragma unroll 1
    for (int e = column; e < hd; ++e) {
        reinterpret_cast<unsigned short *>(row)[e] = (unsigned short)lo;
        lo = lo >> 16 | hi << 48;
        hi >>= 16;
    }
}

// Two floats rounded to nearest even by one instruction.
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
template <int DT>
__device__ __forceinline__ unsigned both(float a, float b) {
    if constexpr (DT == PARO_F16) return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, f16x2_t));
    else return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{a, b}, bf16x2_t));
}

// A tile of rows on its way from memory to shared memory: 16 bytes a lane to `to` + 16 * lane, past the registers; lanes without a piece are sent NOWHERE, where the
// hardware reads zeros.  Rows have to lie on 16 bytes.  (Through registers, when it came in: 8192 tokens of 32 heads of 128 forward 520 us, so 457.)  In assembly because the
// compiler, which cannot tell the tiles apart, would wait for it before every read of shared memory; arrived() waits.  It writes no register; m0, which holds the place in
// shared memory, is an operand.  Five wait states have to stand between a vector instruction that writes a scalar register (v_readlane, where the compiler has kept
// the descriptor in a lane) and its use by a load, one between a write of m0 and its use; inside the assembly the compiler does not see to it.
typedef __attribute__((address_space(3))) char lds_char;
template <int AT>
__device__ __forceinline__ void fill(u32x4 from, unsigned offset, unsigned to) {
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to + AT), "v"(offset), "s"(from) : "memory");
}
// All but the wave's last `IN_FLIGHT` loads have arrived, all its accesses of shared memory are done; then those of all waves.
template <int IN_FLIGHT>
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(IN_FLIGHT) : "memory"); }
constexpr unsigned NOWHERE = 0x80000000u;

template <int HD, int ROWS>
struct Filled {
    using T = Tile<HD>;
    static constexpr int AT_ONCE = 64 / T::PIECES, FILLS = ROWS / AT_ONCE / 4;       // rows of an instruction; instructions of a wave of four
    static_assert(FILLS >= 1 && ROWS % (AT_ONCE * 4) == 0, "every wave fills a part");
    unsigned at[FILLS];              // of the lane's pieces, from the tile's first row

    static __device__ __forceinline__ int row(int n) { return (wave_of() * FILLS + n) * AT_ONCE + (int)(threadIdx.x & 63) / T::PIECES; }
    __device__ __forceinline__ Filled(int64_t ld, int hd) {
#pragma unroll
        for (int n = 0; n < FILLS; ++n) {
            const int piece = (int)(threadIdx.x % T::PIECES) ^ T::key(row(n));
            at[n] = piece * 8 < hd ? (unsigned)row(n) * (unsigned)(ld * 2) + piece * 16 : NOWHERE;
        }
    }
    static __device__ __forceinline__ u32x4 descriptor(const char *tile) {
        const uint64_t at = (uint64_t)(uintptr_t)tile;
        return u32x4{(unsigned)at, (unsigned)(at >> 32) & 0xFFFFu, 0x7FFFFFF0u, 0x00020000u};
    }
    static __device__ __forceinline__ unsigned place(const char *tile) { return (unsigned)(uintptr_t)(const lds_char *)tile + wave_of() * FILLS * 1024; }
    __device__ __forceinline__ void whole(u32x4 from, const char *tile) const {
        static_for<0, FILLS>([&](auto n) { fill<n * 1024>(from, at[n], place(tile)); });
    }
    template <class F>
    __device__ __forceinline__ void held(u32x4 from, const char *tile, F &&holds) const {
        static_for<0, FILLS>([&](auto n) { fill<n * 1024>(from, holds(row(n)) ? at[n] : NOWHERE, place(tile)); });
    }
};

// A row of 32 of the result of 32 x 32 products: a lane has of its row (lane % 32) the elements 8 * (i / 4) + 4 * (lane / 32) + i % 4.  Both halves of a
// wave exchange, so that each stores eight in a row.
template <int DT>
__device__ __forceinline__ void store_row32(char *row, int column, int hd, const f32x16 &x, float times, bool there) {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int i = 0; i < 16; i += 8) {
        const unsigned a0 = both<DT>(x[i] * times, x[i + 1] * times), a1 = both<DT>(x[i + 2] * times, x[i + 3] * times);
        const unsigned b0 = both<DT>(x[i + 4] * times, x[i + 5] * times), b1 = both<DT>(x[i + 6] * times, x[i + 7] * times);
        const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
        if (there) store_piece_of_head(row, column + 2 * i + 8 * h, hd, u32x4{s0[0], s1[0], s0[1], s1[1]});
    }
}
template <int DT>
__device__ __forceinline__ short8_t pack8(const f32x16 &x, int from) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = both<DT>(x[from + 2 * i], x[from + 2 * i + 1]);
    return __builtin_bit_cast(short8_t, v);
}

// ---------------------------------------------------------------- the bias
__device__ __forceinline__ float table_value(const Attn &a, int bucket, int head) {
    const int64_t at = (int64_t)bucket * a.heads + head;
    return a.table_dtype == PARO_F32 ? static_cast<const float *>(a.table)[at] : bits16_to_f32(a.table_dtype, static_cast<const unsigned short *>(a.table)[at]);
}
// A head's bias in shared memory.  Where the last bucket begins within NEAR (far_from), its values are there for every distance from -EDGE to far_from + EDGE, so that a
// tile reads them wherever it lies; otherwise each tile has a window of EDGE distances of its own looked up.  (Windows always, each a search of five steps: 8 x 1024
// tokens of 12 heads of 64 forward 46 us, so 40.)
constexpr int NEAR = 1024, EDGE = 160;
struct Bias {
    int first[MAX_BUCKETS];
    float column[MAX_BUCKETS];
    float by[EDGE + NEAR + EDGE];

    __device__ __forceinline__ void load(const Attn &a, int head) {         // then a barrier
        for (int b = threadIdx.x; b < a.buckets; b += 256) {
            first[b] = a.first[b];
            column[b] = table_value(a, b, head);
        }
    }
    // The last bucket that begins at `far` or before; the first where none does.
    __device__ __forceinline__ int bucket(int far, int buckets) const {
        int lo = 0, n = buckets;
        while (n > 1) {                                                     // the answer lies in [lo, lo + n)
            const int half = n >> 1;
            const bool up = first[lo + half] <= far;
            lo = up ? lo + half : lo;
            n = up ? n - half : half;
        }
        return lo;
    }
    __device__ __forceinline__ float of(int far, int buckets) const { return column[bucket(far < 0 ? 0 : far, buckets)]; }
};
struct Distances {                      // what a thread holds of it
    int far_from;                       // distances from here on have the last bucket's bias
    float far;
    bool whole, usual;                  // whole: of every distance;  usual: LOG2E times the far bias says enough of it

    // after load() and a barrier; then another
    __device__ __forceinline__ void begin(Bias &bias, int buckets) {
        far_from = __builtin_amdgcn_readfirstlane(bias.first[buckets - 1]);
        if (far_from < 0) far_from = 0;
        far = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(bias.column[buckets - 1])));
        usual = fabsf(far) < USUAL;
        whole = far_from <= NEAR;
        if (whole)
            for (int x = threadIdx.x; x < far_from + 2 * EDGE; x += 256) bias.by[x] = bias.of(x - EDGE, buckets);
    }
    __device__ __forceinline__ bool beyond(int lowest) const { return lowest >= far_from; }      // all of a tile, whose lowest distance this is
    // the window of a tile, for its part of the ring; then a barrier
    __device__ __forceinline__ void look_up(Bias &bias, int lowest, int part, int buckets) const {
        if (!whole && !(usual && beyond(lowest)) && threadIdx.x < EDGE) bias.by[part * EDGE + threadIdx.x] = bias.of(lowest + (int)threadIdx.x, buckets);
    }
    // values by distance from `lowest` on
    __device__ __forceinline__ const float *values(const Bias &bias, int lowest, int part) const {
        return whole ? bias.by + EDGE + (lowest < far_from ? lowest : far_from) : bias.by + part * EDGE;
    }
};

// ---------------------------------------------------------------- rows off 16 bytes
// Copies of the sequences' rows, heads side by side, each in whole pieces (zeros behind its end): sequence b from row b len on.  (3 x 1999 tokens, 10 heads of 77 over 5: 12 us
// for 43 MiB of four arrays.  Each block through its registers, when it came in: 340 us backward, so 240.)
constexpr int ALIGN_ROWS = 8;
struct Copies {
    Rows from[4];
    char *to[4];
    int heads[4];
    bool keys[4];                       // rows of keys, or of queries
};
__global__ __launch_bounds__(256) void k_align(Attn a, Copies c) {
    const int which = blockIdx.y, tiles = gridDim.x / a.batch, b = blockIdx.x / tiles, row0 = blockIdx.x % tiles * ALIGN_ROWS;
    const Sequence seq(a, b);
    const bool keys = c.keys[which];
    const int n = keys ? seq.nk : seq.nq, rows = n - row0 < ALIGN_ROWS ? n - row0 : ALIGN_ROWS, pieces = (a.hd + 7) / 8, of_row = c.heads[which] * pieces;
    const int64_t to0 = (int64_t)b * (keys ? a.len_k : a.len_q) + row0, from0 = (int64_t)(keys ? seq.k0 : seq.q0) + row0;
    const Rows from = c.from[which];
    u32x4 *const to = reinterpret_cast<u32x4 *>(c.to[which]) + to0 * of_row;
    const int all = rows > 0 ? rows * of_row : 0;
    for (int x0 = threadIdx.x; x0 < all; x0 += 4 * 256) {                    // four pieces in flight
        u32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int x = x0 + u * 256 < all ? x0 + u * 256 : all - 1, r = x / of_row, in = x % of_row;
            v[u] = piece_of_head(from.of(from0 + r, in / pieces), in % pieces * 8, a.hd, true);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (x0 + u * 256 < all) to[x0 + u * 256] = v[u];
    }
}

// ---------------------------------------------------------------- host
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int check_attn(const std::string &f, const paro_attn_t *d) {
    if (!d) return fail(PARO_EINVAL, f + "d is NULL");
    const auto bad = [&](const char *text) { return fail(PARO_EINVAL, f + text); };
    if (d->dtype != PARO_BF16 && d->dtype != PARO_F16) return bad("dtype must be PARO_BF16 or PARO_F16");
    if (d->batch < 0 || d->batch > (1 << 20)) return bad("batch must be in [0, 2^20]");
    if (d->heads < 1 || d->heads > 1024 || d->kv_heads < 1 || d->heads % d->kv_heads) return bad("heads must be in [1, 1024] and a multiple of kv_heads");
    if (d->head_dim < MIN_HEAD || d->head_dim > MAX_HEAD) return bad("head_dim must be in [8, 128]");
    if (d->len_q < 0 || d->len_q > FAR_AWAY || d->len_k < 0 || d->len_k > FAR_AWAY) return bad("len_q and len_k must be in [0, 2^30]");
    if (d->rows_q < 0 || d->rows_q > INT32_MAX || d->rows_k < 0 || d->rows_k > INT32_MAX) return bad("rows_q and rows_k must be in [0, 2^31)");
    if (d->batch * d->len_q > INT32_MAX && !d->rows_q) return bad("more than 2^31 - 1 rows of queries");
    if (d->batch * d->len_k > INT32_MAX && !d->rows_k) return bad("more than 2^31 - 1 rows of keys");
    if (d->window < 0 || d->sinks < 0) return bad("window and sinks must not be negative");
    if (!(d->scale >= 1e-18f) || !(d->scale <= 1e18f)) return bad("scale must be in [1e-18, 1e18]");
    if (d->buckets < 0 || d->buckets > MAX_BUCKETS) return bad("buckets must be in [0, 256]");
    if (d->buckets && d->table_dtype != PARO_F32 && d->table_dtype != d->dtype) return bad("table_dtype must be PARO_F32 or dtype");
    // a head's distance is that between neighbours in a row, or that between whole planes: each row of each head ends before the next one's begins
    const int64_t hd = d->head_dim, kv = d->kv_heads;
    const int64_t lds[4] = {d->ld_q, d->ld_k, d->ld_v, d->ld_out}, heads[4] = {d->head_q, d->head_k, d->head_v, d->head_out};
    for (int i = 0; i < 4; ++i) {
        const int64_t count = i == 0 || i == 3 ? d->heads : kv;
        const int64_t head = heads[i] ? heads[i] : hd, ld = lds[i] ? lds[i] : count * hd;
        if (head < hd || ld < hd) return bad("a head is longer than its distance to the next");
        if (head < ld && ld < (count - 1) * head + hd) return bad("a row is longer than its distance to the next");
        if (ld > ((int64_t)1 << 24) || head > ((int64_t)1 << 50)) return bad("distances between rows are at most 2^24, between heads 2^50");
    }
    if (ceil_div(std::max(d->len_q, d->len_k), 8) * d->heads > INT32_MAX / std::max<int64_t>(1, d->batch))
        return bad("batch * heads * length is at most 2^34");
    return PARO_OK;
}
// Without arrays that say where sequences lie, they lie one behind the other.
inline int check_rows(const std::string &f, const paro_attn_t &d, const void *q_starts, const void *k_starts) {
    if (!q_starts && d.rows_q && d.rows_q < d.batch * d.len_q) return fail(PARO_EINVAL, f + "rows_q holds fewer than batch * len_q rows");
    if (!k_starts && d.rows_k && d.rows_k < d.batch * d.len_k) return fail(PARO_EINVAL, f + "rows_k holds fewer than batch * len_k rows");
    return PARO_OK;
}
inline int check_inputs(const std::string &f, const paro_attn_t &d, const void *q, const void *k, const void *v, const int32_t *q_starts, const int32_t *k_starts,
                        const int32_t *k_lens, const void *table, const int32_t *first) {
    int rc = d.len_q ? check_array(q, 2, f + "q") : PARO_OK;
    if (!rc && d.len_k) rc = check_array(k, 2, f + "k");
    if (!rc && d.len_k) rc = check_array(v, 2, f + "v");
    if (!rc && q_starts) rc = check_array(q_starts, 4, f + "q_starts");
    if (!rc && k_starts) rc = check_array(k_starts, 4, f + "k_starts");
    if (!rc && k_lens) rc = check_array(k_lens, 4, f + "k_lens");
    if (!rc && d.buckets) rc = check_array(table, size_of(d.table_dtype), f + "table");
    if (!rc && d.buckets) rc = check_array(first, 4, f + "first");
    return rc;
}
inline int check_room(const std::string &f, int64_t needed, const void *workspace, int64_t bytes) {
    if (!needed) return PARO_OK;
    const int rc = check_array(workspace, 16, f + "workspace");
    if (rc) return rc;
    return bytes < needed ? fail(PARO_ERANGE, f + "the workspace is smaller than paro_attn_workspace says") : PARO_OK;
}
// A launch counts its threads in 32 bits.
inline int check_launch(const std::string &f, int64_t blocks, int64_t threads) {
    return blocks * threads > UINT32_MAX ? fail(PARO_ERANGE, f + "more sequences, heads and tokens than a launch takes") : PARO_OK;
}
// Rows that lie on 16 bytes and heads of whole pieces: what goes past the registers.
inline bool fills_take(int64_t ld, int64_t head, int64_t hd) { return hd % 8 == 0 && ld % 8 == 0 && head % 8 == 0; }
inline int64_t copy_bytes(const paro_attn_t &d, int64_t len, int64_t heads) { return ceil_div(d.batch * len * heads * ceil_div(d.head_dim, 8) * 16, 256) * 256; }
inline int check_aligned(const std::string &f, const Rows &r, int hd, const char *name) {
    return fills_take(r.ld, r.head, hd) && (reinterpret_cast<uintptr_t>(r.at) & 15) ? fail(PARO_EALIGN, f + name + " is not 16-byte aligned, as its rows are") : PARO_OK;
}
// Rows that the fills do not take are copied into the workspace.
struct Copying {
    Copies c{};
    int arrays = 0;
    int64_t most = 0;
    char *ws;
    int64_t at;
    Copying(char *workspace, int64_t offset) : ws(workspace), at(offset) {}
    bool take(const paro_attn_t &d, Rows &rows, int64_t len, int64_t heads, bool keys) {
        if (fills_take(rows.ld, rows.head, d.head_dim)) return false;
        const int64_t width = ceil_div(d.head_dim, 8) * 8;
        c.from[arrays] = rows;
        c.heads[arrays] = (int)heads;
        c.keys[arrays] = keys;
        rows = Rows{ws + at, heads * width, width};
        c.to[arrays++] = rows.at;
        at += copy_bytes(d, len, heads);
        most = std::max(most, len);
        return true;
    }
    int64_t blocks(const Attn &a) const { return ceil_div(most, ALIGN_ROWS) * a.batch; }
    void launch(const Attn &a, hipStream_t st) const {
        if (arrays && most && a.batch)
            hipLaunchKernelGGL(k_align, dim3((unsigned)blocks(a), (unsigned)arrays), dim3(256), 0, st, a, c);
    }
};
inline Attn attn_of(const paro_attn_t &d, const void *q, const void *k, const void *v, const int32_t *q_starts, const int32_t *k_starts, const int32_t *k_lens,
                    const void *table, const int32_t *first) {
    const auto rows = [&](const void *at, int64_t heads, int64_t ld, int64_t head) {
        return Rows{static_cast<char *>(const_cast<void *>(at)), ld ? ld : heads * d.head_dim, head ? head : d.head_dim};
    };
    Attn a{};
    a.q = rows(q, d.heads, d.ld_q, d.head_q);
    a.k = rows(k, d.kv_heads, d.ld_k, d.head_k);
    a.v = rows(v, d.kv_heads, d.ld_v, d.head_v);
    a.out = rows(nullptr, d.heads, d.ld_out, d.head_out);
    a.keys = a.k;
    a.values = a.v;
    a.q_starts = q_starts;
    a.k_starts = k_starts;
    a.k_lens = k_lens;
    a.table = table;
    a.first = first;
    a.batch = (int)d.batch;
    a.heads = (int)d.heads;
    a.kv_heads = (int)d.kv_heads;
    a.hd = (int)d.head_dim;
    a.len_q = (int)d.len_q;
    a.len_k = (int)d.len_k;
    a.rows_q = (int)(d.rows_q ? d.rows_q : d.batch * d.len_q);
    a.rows_k = (int)(d.rows_k ? d.rows_k : d.batch * d.len_k);
    a.window = d.window && d.window < FAR_AWAY ? (int)d.window : FAR_AWAY;
    a.sinks = (int)std::min<int64_t>(d.sinks, FAR_AWAY);
    a.buckets = d.buckets;
    a.table_dtype = d.table_dtype;
    a.scale = d.scale;
    return a;
}

#define PARO_BY_FORM(CALL)                                                                                                            \
    (d->dtype == PARO_BF16 ? d->head_dim <= 64 ? d->buckets ? CALL(PARO_BF16, 64, true) : CALL(PARO_BF16, 64, false)                    \
                                               : d->buckets ? CALL(PARO_BF16, 128, true) : CALL(PARO_BF16, 128, false)                  \
                           : d->head_dim <= 64 ? d->buckets ? CALL(PARO_F16, 64, true) : CALL(PARO_F16, 64, false)                      \
                                               : d->buckets ? CALL(PARO_F16, 128, true) : CALL(PARO_F16, 128, false))

}  // namespace

namespace paro {
int64_t attn_forward_workspace(const paro_attn_t &d);
}
