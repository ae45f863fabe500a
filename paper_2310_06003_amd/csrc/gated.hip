// The gated projections of a feed-forward block and their gradient (gfx950):
//
//   g = x Wg',  u = x Wu',  h = act(g) * u
//   dg = dh u act'(g),  du = dh act(g);   dx = dg Wg + du Wu,  dWg = dg' x,  dWu = du' x
//
// Bound by the matrix cores for many tokens, by reading the weights for few.  Three products of one kernel: a block computes
// a tile of the result with 16x16x32 matrix instructions in fp32, its waves side by side on it, from a ring of five parts of shared memory,
// each 64 steps of the inner dimension of one operand, that are filled past the registers.  Forward, a tile holds the gate's and the up projection's columns of
// the same hidden elements, so that one wave has both and the activation and the product happen in its registers.
// An operand whose inner dimension lies along memory (x, W forward; dg | du of dx) is read from shared memory in pieces of eight steps; one
// whose inner dimension goes from row to row (W of dx; both of dW) is staged as it lies and transposed by the reading instruction.
#include <type_traits>

#include "operators.hpp"

namespace {

constexpr int STEPS = 64;                // of the inner dimension, a stage: a part of the ring for each operand
constexpr int ROW_BYTES = STEPS * 2;     // of an operand that lies along it
enum { FORWARD = 0, INPUT_GRAD = 1, WEIGHT_GRAD = 2 };

typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char;

template <int DT>
__device__ __forceinline__ f32x4 mfma(short8_t a, short8_t b, f32x4 c) {
    if constexpr (DT == PARO_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// The activation and its derivative.
template <int ACT>
__device__ __forceinline__ float act(float g) {
    if constexpr (ACT == PARO_SILU) return g / (1.0f + __expf(-g));
    else return 0.5f * g * (1.0f + erff(g * 0.70710678118654752440f));
}
template <int ACT>
__device__ __forceinline__ void act_and_slope(float g, float &a, float &da) {
    if constexpr (ACT == PARO_SILU) {
        const float y = 1.0f / (1.0f + __expf(-g));
        a = g * y;
        da = y * (1.0f + g * (1.0f - y));
    } else {
        const float y = 0.5f * (1.0f + erff(g * 0.70710678118654752440f));
        a = g * y;
        da = y + g * __expf(-0.5f * g * g) * 0.39894228040143267794f;
    }
}

__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// 16 bytes a lane from memory to shared memory at `to` + 16 * lane, past the registers; out of range: zeros.  In assembly because
// the compiler, which cannot tell the stages apart, would wait for it before every read of shared memory; all_waves() waits.
// It writes no register.  m0, which holds the place in shared memory, is an operand, so that the compiler knows what is in it.  Five wait states have to stand between a
// vector instruction that writes a scalar register (v_readlane, where the compiler has kept the descriptor in a lane) and its use by a load, one between a write of
// m0 and its use; inside the assembly the compiler does not see to it.
template <int AT>
__device__ __forceinline__ void fill(u32x4 from, unsigned offset, unsigned to) {
    asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to + AT), "v"(offset), "s"(from) : "memory");
}
// All but the wave's last `IN_FLIGHT` fills have arrived, all its reads are done; then those of all waves.
template <int IN_FLIGHT>
__device__ __forceinline__ void all_waves() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(IN_FLIGHT) : "memory"); }

// A buffer descriptor of the memory from `base` on.  Lanes without a piece are sent NOWHERE, beyond it, where the hardware reads zeros: all
// others stay inside their operand.
__device__ __forceinline__ u32x4 descriptor(const char *base) {
    const uint64_t at = (uint64_t)(uintptr_t)base;
    return u32x4{(unsigned)at, (unsigned)(at >> 32) & 0xFFFFu, 0x7FFFFFF0u, 0x00020000u};
}
constexpr unsigned NOWHERE = 0x80000000u;

struct Product {
    // Operand a: [rows][inner] (along) or [inner][rows] (across), operand b: [cols][inner] or [inner][cols].  Two parts: forward, the
    // columns of b (gate, up); of dx, the inner dimension (dg and du, Wg and Wu); of dW, the rows of a.  dg and du lie in panels (see k_slopes).
    const char *a[2], *b[2];
    int64_t lda, ldb, panel;             // bytes from row to row, and from panel to panel
    int64_t rows, cols, inner;           // inner: of one part, in whole pieces where an operand lies along it
    int64_t inner_b;                     // steps that b has (across: rows)
    char *out[3];                        // h, g, u; dx; dWg, dWu
    int64_t ldo;                         // elements
    int tiles_m, tiles_n;
    unsigned whole, splits;              // the first tiles are whole blocks' work; of the others each is split among so many blocks,
    float *partial;                      // which leave their sums here: [tile][split][row of tiles][tile][thread][4]
    const float *back;                   // of fp16 slopes: what the results are multiplied by (see k_slopes); or NULL
    __device__ __forceinline__ float scale() const { return back ? *back : 1.0f; }
};

// Blocks go to the eight XCDs in turn: each takes a run of tiles of its own.
__device__ __forceinline__ unsigned in_runs(unsigned block, unsigned all) {
    const unsigned each = all / 8, more = all % 8, xcd = block % 8;
    return xcd * each + (xcd < more ? xcd : more) + block / 8;
}
// Where tile t of the result lies.  Runs go four tiles of rows wide, so that what an XCD's blocks read at a time stays in its L2 (eight wide:
// 4096 tokens of 4096 x 11008 forward 603 us, so 593; 8192 backward 2395 and 2353).
template <int MODE, int BM, int BN>
struct Place {
    int part;                            // dW: the first half of the tiles of rows is dWg
    int64_t row0, col0;
    __device__ __forceinline__ Place(const Product &p, unsigned t) {
        constexpr unsigned WIDE = 4;
        const unsigned band = t / (WIDE * p.tiles_n), first = band * WIDE, in = t - band * WIDE * p.tiles_n;
        const unsigned high = p.tiles_m - first < WIDE ? p.tiles_m - first : WIDE;
        const int tm = first + in % high, tn = in / high, of_part = p.tiles_m / 2;
        part = MODE == WEIGHT_GRAD && tm >= of_part;
        row0 = (int64_t)(tm - part * of_part) * BM;
        col0 = (int64_t)tn * (MODE == FORWARD ? BN / 2 : BN);
    }
};

// Of each 16x16 tile a lane holds four columns, 4 * (lane / 16) on, of row lane % 16.  Two tiles of columns side by side are stored
// together: quads exchange halves, so that each lane has eight columns in a row.
template <int DT>
__device__ __forceinline__ void store8(const Product &p, char *out, int64_t m, int64_t n, const f32x4 &left, const f32x4 &right) {
    const int quad = (threadIdx.x >> 4) & 3;
    const u32x2_t a{pack2<DT>(left[0], left[1]), pack2<DT>(left[2], left[3])}, b{pack2<DT>(right[0], right[1]), pack2<DT>(right[2], right[3])};
    const auto s0 = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto s1 = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    const u32x4 v{s0[0], s1[0], s0[1], s1[1]};
    n += (quad & 1) * 16 + (quad >> 1) * 8;
    if (m >= p.rows || n >= p.cols) return;
    if (n + 8 <= p.cols) {
        store_piece<DT>(out, m * p.ldo + n, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (n + e < p.cols) reinterpret_cast<unsigned short *>(out)[m * p.ldo + n + e] = (unsigned short)(v[e / 2] >> (16 * (e & 1)));
    }
}
// What a wave does with a finished row of its tiles.
template <int DT, int MODE, int ACT, int BM, int BN>
__device__ __forceinline__ void finish(const Product &p, const Place<MODE, BM, BN> &at, int64_t m, int wn, float scale, f32x4 (&acc)[4]) {
    if constexpr (MODE == FORWARD) {
        f32x4 h[2];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) h[j][q] = act<ACT>(acc[j][q]) * acc[j + 2][q];
        const int64_t n = at.col0 + wn * 32;
        store8<DT>(p, p.out[0], m, n, h[0], h[1]);
        if (p.out[1]) {
            store8<DT>(p, p.out[1], m, n, acc[0], acc[1]);
            store8<DT>(p, p.out[2], m, n, acc[2], acc[3]);
        }
    } else {
        if constexpr (DT == PARO_F16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] *= scale;
        }
#pragma unroll
        for (int j = 0; j < 4; j += 2) store8<DT>(p, at.part ? p.out[1] : p.out[0], m, at.col0 + (wn * 4 + j) * 16, acc[j], acc[j + 1]);
    }
}

template <int DT, int MODE, int ACT, int BM, int BN, int WAVES_M, int WAVES_N>
__device__ __forceinline__ void product(const Product p, unsigned block, unsigned blocks) {
    constexpr int THREADS_ = 64 * WAVES_M * WAVES_N;
    constexpr int TM = BM / WAVES_M / 16, TN = BN / WAVES_N / 16;             // 16x16 tiles of a wave
    constexpr int A_BYTES = BM * ROW_BYTES, B_BYTES = BN * ROW_BYTES, PART = A_BYTES;
    constexpr int FILLS = A_BYTES / (THREADS_ * 16);           // of a part, by each wave
    constexpr bool A_ACROSS = MODE == WEIGHT_GRAD, A_PANELS = MODE != FORWARD, B_ACROSS = MODE != FORWARD;
    static_assert(TN == 4 && A_BYTES == B_BYTES, "a wave's columns are two pairs of tiles, and a part of the ring takes either operand");
    extern __shared__ __attribute__((aligned(1024))) char ring[];
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_char *)ring;
    const int w = wave_of(), lane = threadIdx.x & 63, wm = w / WAVES_N, wn = w % WAVES_N;
    // The block's tile, and its share of the inner dimension.
    const bool is_whole = block < p.whole;
    const unsigned others = is_whole ? 0 : (blocks - p.whole) / p.splits, among = is_whole ? 0 : block - p.whole;
    const unsigned split = is_whole ? 0 : among / others, split_tile = is_whole ? 0 : in_runs(among - split * others, others);
    const unsigned splits = is_whole ? 1 : p.splits;
    const Place<MODE, BM, BN> at(p, is_whole ? in_runs(block, p.whole) : p.whole + split_tile);
    const int64_t row0 = at.row0, col0 = at.col0;
    const int out_part = at.part;
    const float scale = DT == PARO_F16 && MODE != FORWARD ? p.scale() : 1.0f;       // loaded long before it is needed

    // A lane's pieces: their offsets from where the stage begins, and the step (along: the first of eight) of each.  The pieces of a
    // stage are exchanged within 256 bytes such that the lanes that read at a time meet all banks.  Pieces of rows or columns that the operand
    // does not have are nowhere.
    unsigned a_at[FILLS], b_at[FILLS];
    int a_step[FILLS], b_step[FILLS];
    const auto along = [&](int row, bool there, int64_t memory_row, int64_t ld, unsigned &at, int &step) {
        const int piece = (lane & 7) ^ ((row >> 1) & 7);
        at = there ? (unsigned)(memory_row * ld) + piece * 16 : NOWHERE;
        step = piece * 8;
    };
    // in_panels: the columns lie in panels of 64, `panel` bytes apart
    const auto across = [&](int k, int piece, int64_t columns_left, int64_t ld, bool in_panels, unsigned &at, int &step) {
        const int block = (piece >> 1) ^ ((k & 3) | ((k >> 1) & 4)), column = (block * 2 + (piece & 1)) * 8;
        at = column < columns_left ? (unsigned)(k * ld) + (in_panels ? (unsigned)((column >> 6) * p.panel) + (column & 63) * 2 : column * 2) : NOWHERE;
        step = k;
    };
    // Forward: this wave fills rows of b that are the gate's (even waves) or the up projection's, from this row on.
    const int b_part = MODE == FORWARD ? w & 1 : 0;
    const int64_t b_row0 = MODE == FORWARD ? col0 + (w >> 1) * 32 : 0;
#pragma unroll
    for (int i = 0; i < FILLS; ++i) {
        if constexpr (A_ACROSS) {
            constexpr int PIECES = BM / 8;
            across((w * FILLS + i) * (64 / PIECES) + lane / PIECES, lane % PIECES, p.rows - row0, ROW_BYTES, true, a_at[i], a_step[i]);
        } else {
            const int r = (w * FILLS + i) * 8 + lane / 8;
            along(r, r < p.rows - row0, r, A_PANELS ? ROW_BYTES : p.lda, a_at[i], a_step[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < FILLS; ++i) {
        if constexpr (B_ACROSS) {
            constexpr int PIECES = BN / 8;
            across((w * FILLS + i) * (64 / PIECES) + lane / PIECES, lane % PIECES, p.cols - col0, p.ldb, false, b_at[i], b_step[i]);
        } else {                                    // 32 rows of the gate's, then 32 of the up projection's, for each wave's 64 columns
            static_assert(B_ACROSS || FILLS == 4, "a wave fills 32 rows of b");
            const int r = i * 8 + lane / 8;
            along((w * FILLS + i) * 8 + lane / 8, b_row0 + r < p.cols, r, p.ldb, b_at[i], b_step[i]);
        }
    }

    const int per_part = (int)((p.inner + STEPS - 1) / STEPS), parts = MODE == INPUT_GRAD ? 2 : 1;
    const int stages_all = per_part * parts;
    const int from = (int)((int64_t)stages_all * split / splits), to = (int)((int64_t)stages_all * (split + 1) / splits);

    // What the next stage is filled from.
    u32x4 a_from, b_from;
    int a_left, b_left, a_until, b_until;           // steps left of the part; stages until the part ends, or the block's share of it
    const int64_t a_stage = A_ACROSS ? STEPS * ROW_BYTES : A_PANELS ? p.panel : ROW_BYTES, b_stage = B_ACROSS ? STEPS * p.ldb : ROW_BYTES;
    const auto begin_a = [&](int part, int stage) {
        const int64_t k0 = (int64_t)stage * STEPS;
        a_from = descriptor(A_ACROSS   ? (out_part ? p.a[1] : p.a[0]) + row0 / 64 * p.panel + k0 * ROW_BYTES
                            : A_PANELS ? (part ? p.a[1] : p.a[0]) + (k0 / 64) * p.panel + row0 * ROW_BYTES
                                       : (part ? p.a[1] : p.a[0]) + row0 * p.lda + k0 * 2);
        a_left = (int)(p.inner - k0);
        a_until = (to < (part + 1) * per_part ? to - part * per_part : per_part) - stage;
    };
    const auto begin_b = [&](int part, int stage) {
        const int64_t k0 = (int64_t)stage * STEPS;
        b_from = descriptor(B_ACROSS ? (part ? p.b[1] : p.b[0]) + k0 * p.ldb + col0 * 2 : (b_part ? p.b[1] : p.b[0]) + b_row0 * p.ldb + k0 * 2);
        b_left = (int)(p.inner_b - k0);
        b_until = (to < (part + 1) * per_part ? to - part * per_part : per_part) - stage;
    };
    const auto advance = [](u32x4 &d, int64_t bytes) {
        const uint64_t at = ((uint64_t)d[1] << 32 | d[0]) + (uint64_t)bytes;
        d[0] = (unsigned)at;
        d[1] = (unsigned)(at >> 32);
    };
    // Past the last stage they go on with zeros from nowhere: the waits count on as many fills each time.
    bool second_a = from >= per_part, second_b = second_a;
    begin_a(second_a, from - (second_a ? per_part : 0));
    begin_b(second_b, from - (second_b ? per_part : 0));
    const auto next_a = [&]() {
        advance(a_from, a_stage);
        a_left -= STEPS;
        if (--a_until == 0) {
            if (MODE == INPUT_GRAD && !second_a && to > per_part) {
                second_a = true;
                begin_a(1, 0);
            } else {
                a_left = INT32_MIN / 2;
            }
        }
    };
    const auto next_b = [&]() {
        advance(b_from, b_stage);
        b_left -= STEPS;
        if (--b_until == 0) {
            if (MODE == INPUT_GRAD && !second_b && to > per_part) {
                second_b = true;
                begin_b(1, 0);
            } else {
                b_left = INT32_MIN / 2;
            }
        }
    };
    const unsigned lds_wave = lds0 + w * FILLS * 1024;
    const auto fill_a = [&](auto i, unsigned to_part) { fill<i * 1024>(a_from, a_step[i] < a_left ? a_at[i] : NOWHERE, lds_wave + to_part); };
    const auto fill_b = [&](auto i, unsigned to_part) { fill<i * 1024>(b_from, b_step[i] < b_left ? b_at[i] : NOWHERE, lds_wave + to_part); };

    // Where a lane reads a fragment: rows lane % 16 of a tile, steps 8 * (lane / 16) on.
    const int quad = lane >> 4, of16 = lane & 15;
    const int along_row = of16 * ROW_BYTES, along_key = (of16 >> 1);
    const int across_key = (of16 >> 2) | ((quad & 1) << 2);
    const auto read_along = [&](const char *at, int tile, int half) {
        return *reinterpret_cast<const short8_t *>(at + tile * 16 * ROW_BYTES + along_row + (((half * 4 + quad) ^ along_key) << 4));
    };
    const auto read_across = [&](const char *at, int tile, int half, int width) {     // tile: of 16 rows (or columns) of `width` in all
        const char *where = at + (half * 32 + quad * 8 + (of16 >> 2)) * (width * 2) + ((tile ^ across_key) << 5) + (of16 & 3) * 8;
        const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)where);
        const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t *)(where + 4 * width * 2));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    f32x4 acc[TM][TN] = {};
    short8_t fa[2][TM], fb[2][TN];                  // fragments of the two halves of a stage
    const auto read_b = [&](unsigned at, int half, int j) {
        if constexpr (B_ACROSS) return read_across(ring + at, wn * TN + j, half, BN);
        else return read_along(ring + at + wn * TN * 16 * ROW_BYTES, j, half);
    };
    const auto read_a = [&](unsigned at, int half, int i) {
        if constexpr (A_ACROSS) return read_across(ring + at, wm * TM + i, half, BM);
        else return read_along(ring + at + wm * TM * 16 * ROW_BYTES, i, half);
    };
    // The products of one half of a stage, from the fragments, in groups of one tile of rows; before each group some of the other half's
    // fragments are read (from parts a and b) and what `before` does, in this order.
    const auto multiply = [&](auto half_, unsigned a, unsigned b, auto &&before) {
        constexpr int half = half_, other = half ^ 1;
        static_for<0, TM>([&](auto i_) {
            constexpr int i = i_;
            __builtin_amdgcn_sched_barrier(0);
            before(i_);
            if constexpr (2 * i < TN) {
                fb[other][2 * i] = read_b(b, other, 2 * i);
                fb[other][2 * i + 1] = read_b(b, other, 2 * i + 1);
            } else if constexpr (2 * i - TN < TM) {
                fa[other][2 * i - TN] = read_a(a, other, 2 * i - TN);
                fa[other][2 * i - TN + 1] = read_a(a, other, 2 * i - TN + 1);
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mfma<DT>(fb[half][j], fa[half][i], acc[i][j]);
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto two_on = [](unsigned part) { return part >= 3 * PART ? part - 3 * PART : part + 2 * PART; };

    if (from < to) {
        // a(0) b(0) a(1) b(1) a(2)
        static_for<0, 5>([&](auto n) {
            static_for<0, FILLS>([&](auto i) {
                if constexpr (n % 2 == 0) fill_a(i, n * PART);
                else fill_b(i, n * PART);
            });
            if constexpr (n % 2 == 0) next_a();
            else next_b();
        });
        all_waves<3 * FILLS>();
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[0][j] = read_b(PART, 0, j);
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[0][i] = read_a(0, 0, i);
        // In the middle of stage t all waves have read its parts: they are filled with b(t + 2) and a(t + 3), beside the second half's products;
        // and stage t + 1 has arrived, whose b was filled a stage's time ago and whose a two.
        unsigned a = 0, b = PART;
        for (int t = from; t < to; ++t) {
            multiply(std::integral_constant<int, 0>{}, a, b, [](auto) {});
            all_waves<FILLS>();
            const unsigned a_free = a, b_free = b;
            a = two_on(a);
            b = two_on(b);
            multiply(std::integral_constant<int, 1>{}, a, b, [&](auto i) {
                constexpr int each = 2 * FILLS / TM;            // 1 or 2
                static_for<0, each>([&](auto e) {
                    constexpr std::integral_constant<int, (i * each + e) % FILLS> k;
                    if constexpr (i * each + e < FILLS) fill_b(k, a_free);
                    else fill_a(k, b_free);
                });
            });
            next_b();
            next_a();
        }
        all_waves<0>();                             // nothing is on its way into the shared memory of the block that comes next
    }

    if (splits > 1) {
        float *sums = p.partial + ((int64_t)(split_tile * splits + split) * (TM * TN) * THREADS_ + threadIdx.x) * 4;
#pragma unroll
        for (int i = 0; i < TM; ++i)
            if (row0 + (wm * TM + i) * 16 + of16 < p.rows)
#pragma unroll
                for (int j = 0; j < TN; ++j) *reinterpret_cast<f32x4 *>(sums + (int64_t)(i * TN + j) * THREADS_ * 4) = acc[i][j];
        return;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) finish<DT, MODE, ACT>(p, at, row0 + (wm * TM + i) * 16 + of16, wn, scale, acc[i]);
}

template <int DT, int MODE, int ACT, int BM, int BN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void k_product(Product p) {
    product<DT, MODE, ACT, BM, BN, WAVES_M, WAVES_N>(p, blockIdx.x, gridDim.x);
}

// Both products of the backward pass in one launch: neither fills the chip on its own, or not to the end.
template <int DT, int BM, int BN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void k_products(Product dx, Product dw, unsigned of_dx) {
    if (blockIdx.x < of_dx) product<DT, INPUT_GRAD, PARO_SILU, BM, BN, WAVES_M, WAVES_N>(dx, blockIdx.x, of_dx);
    else product<DT, WEIGHT_GRAD, PARO_SILU, BM, BN, WAVES_M, WAVES_N>(dw, blockIdx.x - of_dx, gridDim.x - of_dx);
}

// Adds up the sums of a split tile's blocks, in order: a block for each row of a wave's tiles.
template <int DT, int MODE, int ACT, int BM, int BN, int WAVES_M, int WAVES_N>
__global__ __launch_bounds__(64 * WAVES_M * WAVES_N) void k_join(Product p) {
    constexpr int THREADS_ = 64 * WAVES_M * WAVES_N, TM = BM / WAVES_M / 16, TN = 4;
    const int w = wave_of(), i = blockIdx.y;
    const Place<MODE, BM, BN> at(p, p.whole + blockIdx.x);
    const int64_t m = at.row0 + ((w / WAVES_N) * TM + i) * 16 + (threadIdx.x & 15);
    const float scale = DT == PARO_F16 && MODE != FORWARD ? p.scale() : 1.0f;
    constexpr unsigned U = 4;                       // shares in flight, the last ones too (one by one: 26 tokens of 1231 x 16256 backward 107 us, so 99; 16: 98)
    f32x4 acc[TN] = {};
    if (m < p.rows) {
        const float *sums = p.partial + ((int64_t)blockIdx.x * p.splits * (TM * TN) * THREADS_ + (int64_t)i * TN * THREADS_ + threadIdx.x) * 4;
        for (unsigned s = 0; s < p.splits; s += U) {
            f32x4 part[U][TN];
#pragma unroll
            for (unsigned u = 0; u < U; ++u)
                if (s + u < p.splits)
#pragma unroll
                    for (int j = 0; j < TN; ++j) part[u][j] = *reinterpret_cast<const f32x4 *>(sums + ((int64_t)(s + u) * TM * TN + j) * THREADS_ * 4);
#pragma unroll
            for (unsigned u = 0; u < U; ++u)
                if (s + u < p.splits)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[j] += part[u][j];
        }
    }
    finish<DT, MODE, ACT>(p, at, m, w % WAVES_N, scale, acc);
}

// Forward for few tokens: the weights are read once, straight into registers as fragments, and nothing else counts.  A block takes F_TILES x
// 16 hidden elements; its waves share the inner dimension, 128 steps at a time in turn, and join their sums in shared memory.  Rows need no
// alignment.  Rows of weights and tokens past the last one are read as the last one, and not stored.
constexpr int FEW_WAVES = 4, FEW_STEPS = 128;

template <int DT>
__device__ __forceinline__ short8_t piece_or_zeros(const void *row, int64_t k, int64_t dim) {
    if (k + 8 <= dim) return __builtin_bit_cast(short8_t, load_piece<DT>(row, k));
    u32x4 v{0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (k + e < dim) v[e / 2] |= (unsigned)static_cast<const unsigned short *>(row)[k + e] << (16 * (e & 1));
    return __builtin_bit_cast(short8_t, v);
}

template <int DT, int ACT, int F_TILES, int N_TILES>
__global__ __launch_bounds__(64 * FEW_WAVES) void k_few(const char *x, const char *wg, const char *wu, int64_t n, int64_t dim, int64_t hidden, int64_t ldx,
                                                        int64_t ldh, char *h, char *gate, char *up) {
    __shared__ f32x4 sums[FEW_WAVES][F_TILES * 2 * N_TILES][64];
    const int w = wave_of(), lane = threadIdx.x & 63, quad = lane >> 4, of16 = lane & 15;
    const int64_t f0 = (int64_t)blockIdx.x * (F_TILES * 16);
    const char *weights[F_TILES][2], *tokens[N_TILES];
#pragma unroll
    for (int i = 0; i < F_TILES; ++i) {
        const int64_t f = f0 + i * 16 + of16 < hidden ? f0 + i * 16 + of16 : hidden - 1;
        weights[i][0] = wg + f * dim * 2;
        weights[i][1] = wu + f * dim * 2;
    }
#pragma unroll
    for (int t = 0; t < N_TILES; ++t) tokens[t] = x + (t * 16 + of16 < n ? t * 16 + of16 : n - 1) * ldx * 2;

    f32x4 acc[F_TILES][2][N_TILES] = {};
    for (int64_t k0 = (int64_t)w * FEW_STEPS; k0 < dim; k0 += FEW_WAVES * FEW_STEPS) {
        constexpr int PIECES = FEW_STEPS / 32;
        if (k0 + FEW_STEPS <= dim) {
            short8_t a[PIECES][F_TILES][2], b[PIECES][N_TILES];
#pragma unroll
            for (int c = 0; c < PIECES; ++c) {
                const int64_t k = k0 + c * 32 + quad * 8;
#pragma unroll
                for (int i = 0; i < F_TILES; ++i)
#pragma unroll
                    for (int of = 0; of < 2; ++of) a[c][i][of] = __builtin_bit_cast(short8_t, load_piece<DT>(weights[i][of], k));
#pragma unroll
                for (int t = 0; t < N_TILES; ++t) b[c][t] = __builtin_bit_cast(short8_t, load_piece<DT>(tokens[t], k));
            }
#pragma unroll
            for (int c = 0; c < PIECES; ++c)
#pragma unroll
                for (int i = 0; i < F_TILES; ++i)
#pragma unroll
                    for (int of = 0; of < 2; ++of)
#pragma unroll
                        for (int t = 0; t < N_TILES; ++t) acc[i][of][t] = mfma<DT>(a[c][i][of], b[c][t], acc[i][of][t]);
        } else {
            for (int64_t k1 = k0; k1 < dim; k1 += 32) {
                const int64_t k = k1 + quad * 8;
                short8_t b[N_TILES];
#pragma unroll
                for (int t = 0; t < N_TILES; ++t) b[t] = piece_or_zeros<DT>(tokens[t], k, dim);
#pragma unroll
                for (int i = 0; i < F_TILES; ++i)
#pragma unroll
                    for (int of = 0; of < 2; ++of) {
                        const short8_t a = piece_or_zeros<DT>(weights[i][of], k, dim);
#pragma unroll
                        for (int t = 0; t < N_TILES; ++t) acc[i][of][t] = mfma<DT>(a, b[t], acc[i][of][t]);
                    }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < F_TILES; ++i)
#pragma unroll
        for (int of = 0; of < 2; ++of)
#pragma unroll
            for (int t = 0; t < N_TILES; ++t) sums[w][(i * 2 + of) * N_TILES + t][lane] = acc[i][of][t];
    __syncthreads();
    // A lane holds four hidden elements, 4 * (lane / 16) on, of token lane % 16 of each pair of tiles.
    for (int pair = w; pair < F_TILES * N_TILES; pair += FEW_WAVES) {
        const int i = pair / N_TILES, t = pair - i * N_TILES;
        f32x4 g{}, u{};
#pragma unroll
        for (int k = 0; k < FEW_WAVES; ++k) {
            g += sums[k][(i * 2) * N_TILES + t][lane];
            u += sums[k][(i * 2 + 1) * N_TILES + t][lane];
        }
        const int64_t m = t * 16 + of16, f = f0 + i * 16 + quad * 4;
        if (m >= n) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (f + q >= hidden) break;
            store_one<DT>(h, m * ldh + f + q, act<ACT>(g[q]) * u[q]);
            if (gate) {
                store_one<DT>(gate, m * ldh + f + q, g[q]);
                store_one<DT>(up, m * ldh + f + q, u[q]);
            }
        }
    }
}

// Backward for few tokens: each weight is read once, each of its gradients written once, in one launch, and nothing else counts.  A block takes
// a share of the hidden elements and 512 columns (256): a lane holds its eight columns (four) of every token's x and dx, the sums in fp32, and walks down
// the rows of the weights; dg and du are formed in fp32, and not rounded, by the block.  Rows need no alignment; the last piece of a row starts early, and some elements
// are computed and stored twice, alike.  The shares' dx are added up, in order, by k_few_join.
constexpr int FEW_ROWS = 64;             // hidden elements whose dg and du a block holds at a time
constexpr int few_columns(int64_t n) { return n <= 8 ? 8 : 4; }      // of a lane: registers

// COLUMNS elements of a two-byte type at any element: 4 or 8.
template <int COLUMNS>
__device__ __forceinline__ u32x4 load_columns(const void *base, int64_t elem) {
    if constexpr (COLUMNS == 8) return load_piece<PARO_BF16>(base, elem);
    const u32x2 v = load_half_piece(base, elem);
    return u32x4{v[0], v[1], 0, 0};
}
template <int COLUMNS>
__device__ __forceinline__ void store_columns(void *base, int64_t elem, u32x4 v) {
    if constexpr (COLUMNS == 8) store_piece<PARO_BF16>(base, elem, v);
    else store_half_piece(base, elem, u32x2{v[0], v[1]});
}

template <int DT, int ACT, int N>
__global__ __launch_bounds__(64 * FEW_WAVES) void k_few_grad(const void *dh, const void *gate, const void *up, const void *x, const void *wg, const void *wu,
                                                             int n, int64_t dim, int64_t hidden, int64_t ldx, int64_t ldh, int64_t share, void *dwg, void *dwu,
                                                             float *partial) {
    constexpr int COLUMNS = few_columns(N);
    __shared__ __attribute__((aligned(16))) float slopes[2][FEW_ROWS][N];
    __shared__ f32x4 sums[N][COLUMNS / 4][64];
    const int w = wave_of(), lane = threadIdx.x & 63;
    const int64_t first = (int64_t)blockIdx.x * share, last = first + share < hidden ? first + share : hidden;
    const int64_t column = ((int64_t)blockIdx.y * 64 + lane) * COLUMNS;
    const bool there = column < dim;
    const int64_t c = column + COLUMNS <= dim ? column : dim - COLUMNS;
    u32x4 xs[N];
    float acc[N][COLUMNS] = {};
#pragma unroll
    for (int t = 0; t < N; ++t) {
        xs[t] = u32x4{0, 0, 0, 0};
        if (there && t < n) xs[t] = load_columns<COLUMNS>(x, t * ldx + c);
    }
    for (int64_t f0 = first; f0 < last; f0 += FEW_ROWS) {
        const int rows = (int)(last - f0 < FEW_ROWS ? last - f0 : FEW_ROWS);
        __syncthreads();
        for (int e = threadIdx.x; e < FEW_ROWS * N; e += 64 * FEW_WAVES) {
            const int r = e % FEW_ROWS, t = e / FEW_ROWS;           // neighbours read neighbours
            float dg = 0.0f, du = 0.0f;
            if (r < rows && t < n) {
                const int64_t at = t * ldh + f0 + r;
                const float d = load_one<DT>(dh, at);
                float a, da;
                act_and_slope<ACT>(load_one<DT>(gate, at), a, da);
                dg = d * load_one<DT>(up, at) * da;
                du = d * a;
            }
            slopes[0][r][t] = dg;
            slopes[1][r][t] = du;
        }
        __syncthreads();
        if (!there) continue;
        u32x4 next[2];
        const auto load = [&](int r) {
            next[0] = load_columns<COLUMNS>(wg, (f0 + r) * dim + c);
            next[1] = load_columns<COLUMNS>(wu, (f0 + r) * dim + c);
        };
        if (w < rows) load(w);
        for (int r = w; r < rows; r += FEW_WAVES) {
            const u32x4 now[2] = {next[0], next[1]};
            if (r + FEW_WAVES < rows) load(r + FEW_WAVES);
#pragma unroll
            for (int of = 0; of < 2; ++of) {
                float weight[8], dw[8] = {};
                unpack<DT>(now[of], weight);
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    const float s = slopes[of][r][t];
                    float xt[8];
                    unpack<DT>(xs[t], xt);
#pragma unroll
                    for (int e = 0; e < COLUMNS; ++e) {
                        acc[t][e] = fmaf(s, weight[e], acc[t][e]);
                        dw[e] = fmaf(s, xt[e], dw[e]);
                    }
                }
                store_columns<COLUMNS>(of ? dwu : dwg, (f0 + r) * dim + c, pack<DT>(dw));
            }
        }
    }
    // the waves' dx, one after the other
    for (int k = 0; k < FEW_WAVES; ++k) {
        __syncthreads();
        if (k != w || !there) continue;
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int q = 0; q < COLUMNS / 4; ++q) {
                f32x4 v{acc[t][4 * q], acc[t][4 * q + 1], acc[t][4 * q + 2], acc[t][4 * q + 3]};
                if (k) v += sums[t][q][lane];
                if (k == FEW_WAVES - 1) {
                    if (t < n) store_piece<PARO_F32>(partial, ((int64_t)blockIdx.x * n + t) * dim + c + 4 * q, __builtin_bit_cast(u32x4, v));
                } else {
                    sums[t][q][lane] = v;
                }
            }
    }
}

// Adds up the shares' dx: a block for 64 columns of a token, its waves each a part of the shares.
template <int DT>
__global__ __launch_bounds__(512) void k_few_join(const float *partial, int n, int64_t dim, int shares, int64_t ldx, void *dx) {
    __shared__ float sums[8][64];
    const int w = wave_of(), lane = threadIdx.x & 63;
    const int64_t column = (int64_t)blockIdx.x * 64 + lane, t = blockIdx.y;
    const int each = (shares + 7) / 8, from = w * each, to = from + each < shares ? from + each : shares;
    float sum = 0.0f;
    if (column < dim)
#pragma unroll 8
        for (int s = from; s < to; ++s) sum += partial[((int64_t)s * n + t) * dim + column];
    sums[w][lane] = sum;
    __syncthreads();
    if (w != 0 || column >= dim) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) sum += sums[k][lane];
    store_one<DT>(dx, t * ldx + column, sum);
}

// dg, then du, each in panels of 64 hidden elements: [panel][tokens][64], zeros past the last element.  What a tile's stage reads of them is then a
// run of memory, for dx (256 tokens of a panel) as for dW (64 tokens of four), where rows of 11008 would be 22 KB apart
// (8192 tokens of 4096 x 11008 2302 us, so 2285; this kernel 150 and 141).  Rounded to the
// weights' type, which is what the matrix cores take.  A wave takes eight tokens of a panel.
//
// The product of three fp16 numbers may lie beyond 65504, or where fp16 keeps a binary place or two.  So each block writes down its largest dg or du, of
// the finite ones, and a second launch looks at them: if the largest is below 1 or above 65504 it forms all slopes again, times the power of two that
// brings the largest to between 2^14 and 2^15, and the products' results are multiplied by its inverse.  Either way what a slope loses
// is half an ulp, or 2^-25 of the largest.
struct Slopes {
    const void *dh, *gate, *up;
    int64_t ld, tokens, hidden, panels;
    char *out;
    float *back, *largest;               // of fp16: what the results are multiplied by; of each block of the first launch
    int blocks;
};
__device__ __forceinline__ float block_most(float v, float *room) {
#pragma unroll
    for (int step = 32; step >= 1; step /= 2) v = fmaxf(v, __shfl_xor(v, step));
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    return fmaxf(fmaxf(room[0], room[1]), fmaxf(room[2], room[3]));
}

template <int DT, int ACT, bool AGAIN>
__global__ __launch_bounds__(256) void k_slopes(Slopes s) {
    constexpr bool WATCHED = DT == PARO_F16;
    static_assert(WATCHED || !AGAIN, "other types have the range");
    __shared__ float room[4];
    const int lane = threadIdx.x & 63;
    const int64_t panel = (int64_t)blockIdx.x * 4 + wave_of(), f = panel * 64 + (lane & 7) * 8;
    float factor = 1.0f, most = 0.0f;
    if constexpr (AGAIN) {
        constexpr int U = 8;                        // all of a launch of 2048 blocks at once
        for (int i = threadIdx.x; i < s.blocks; i += U * 256) {
            float of[U];
#pragma unroll
            for (int k = 0; k < U; ++k) of[k] = i + k * 256 < s.blocks ? s.largest[i + k * 256] : 0.0f;
#pragma unroll
            for (int k = 0; k < U; ++k) most = fmaxf(most, of[k]);
        }
        most = block_most(most, room);
        const bool fits = most == 0.0f || (most >= 1.0f && most <= 65504.0f);
        const int exponent = (int)(__float_as_uint(most) >> 23) - 127;      // at least -80: three times 2^-24, and a slope's own smallness
        const int up = fits ? 0 : 14 - (exponent > -100 ? exponent : -100);
        if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *s.back = __uint_as_float((unsigned)(127 - up) << 23);
        if (fits) return;
        factor = __uint_as_float((unsigned)(127 + up) << 23);
    }
    for (int64_t m = (int64_t)blockIdx.y * 8 + lane / 8; panel < s.panels && m < s.tokens; m += (int64_t)gridDim.y * 8) {
        float d[8] = {}, g[8] = {}, u[8] = {}, dg[8], du[8];
        const int64_t at = m * s.ld + f;
        if (f + 8 <= s.hidden) {
            unpack<DT>(load_stream<DT>(s.dh, at), d);
            unpack<DT>(load_stream<DT>(s.gate, at), g);
            unpack<DT>(load_stream<DT>(s.up, at), u);
        } else {
            for (int e = 0; e < 8; ++e)
                if (f + e < s.hidden) {
                    d[e] = load_one<DT>(s.dh, at + e);
                    g[e] = load_one<DT>(s.gate, at + e);
                    u[e] = load_one<DT>(s.up, at + e);
                }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a, da;
            act_and_slope<ACT>(g[e], a, da);
            dg[e] = d[e] * u[e] * da;
            du[e] = d[e] * a;
            if constexpr (AGAIN) {
                dg[e] *= factor;
                du[e] *= factor;
            } else if constexpr (WATCHED) {
                most = fmaxf(most, fabsf(dg[e]) <= 3.4e38f ? fabsf(dg[e]) : 0.0f);
                most = fmaxf(most, fabsf(du[e]) <= 3.4e38f ? fabsf(du[e]) : 0.0f);
            }
        }
        const int64_t to = (panel * s.tokens + m) * 64 + (lane & 7) * 8;
        store_piece<DT>(s.out, to, pack<DT>(dg));
        store_piece<DT>(s.out, s.panels * s.tokens * 64 + to, pack<DT>(du));
    }
    if constexpr (WATCHED && !AGAIN) {
        most = block_most(most, room);
        if (threadIdx.x == 0) s.largest[blockIdx.y * gridDim.x + blockIdx.x] = most;
    }
}
// At most so many blocks, in whole columns of them: of fp16 few enough that each of the second launch reads the largest of all, and of that one, which
// mostly ends there, as few as fill the chip (2048: 4000 tokens of 512 x 1024 backward 50 us, so 47; in a type that needs none of this 43).
constexpr int64_t WATCHED_BLOCKS = 2048, AGAIN_BLOCKS = 512;
dim3 slopes_grid(const paro_gated_t &d, int64_t panels, int64_t blocks) {
    const int64_t x = (panels + 3) / 4, y = (d.n + 7) / 8;
    return dim3((unsigned)x, (unsigned)std::min(y, std::max<int64_t>(1, blocks / x)));
}

// Rows that the fills cannot take - a row or the distance between two is no multiple of 16 bytes - copied to where they can, zeros behind:
// up to three arrays of one width in a launch.  A thread takes pieces as they lie in the copy (a row for each block: 197 tokens of 231 x 8576
// 30 us, so 21).  A piece that ends past its row is loaded whole where the array goes on, and masked.
struct Copies {
    const void *from[3];
    void *to[3];
    int64_t ld[3], rows[3];
    int64_t cols, width;
};
constexpr int ALIGN_PIECES = 4;
__global__ __launch_bounds__(256) void k_align(Copies a) {
    const int which = blockIdx.y;
    const void *from = a.from[which];
    const int64_t ld = a.ld[which], rows = a.rows[which], all = rows * (a.width / 8), end = (rows - 1) * ld + a.cols;
    const unsigned of_row = (unsigned)(a.width / 8);
    for (int64_t first = (int64_t)blockIdx.x * (256 * ALIGN_PIECES); first < all; first += (int64_t)gridDim.x * (256 * ALIGN_PIECES)) {
        const int64_t row0 = first / of_row;
        const unsigned past = (unsigned)(first - row0 * of_row) + threadIdx.x;
        u32x4 v[ALIGN_PIECES];
        int left[ALIGN_PIECES];
#pragma unroll
        for (int i = 0; i < ALIGN_PIECES; ++i) {
            const unsigned down = (past + i * 256) / of_row;
            const int64_t r = row0 + down, c = (int64_t)(past + i * 256 - down * of_row) * 8;
            left[i] = (int)(a.cols - c);
            v[i] = u32x4{0, 0, 0, 0};
            if (r >= rows) continue;
            if (r * ld + c + 8 <= end) {
                v[i] = load_piece<PARO_BF16>(from, r * ld + c);
            } else {
                for (int e = 0; e < 8; ++e)
                    if (e < left[i]) v[i][e / 2] |= (unsigned)static_cast<const unsigned short *>(from)[r * ld + c + e] << (16 * (e & 1));
            }
        }
#pragma unroll
        for (int i = 0; i < ALIGN_PIECES; ++i) {
            const int64_t to = first + threadIdx.x + i * 256;
#pragma unroll
            for (int q = 0; q < 4; ++q) v[i][q] &= left[i] >= 2 * q + 2 ? 0xFFFFFFFFu : left[i] == 2 * q + 1 ? 0xFFFFu : 0u;
            if (to < all) store_piece<PARO_BF16>(a.to[which], to * 8, v[i]);
        }
    }
}

// ---------------------------------------------------------------- host
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t up_to(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
constexpr int COMPUTE_UNITS = 256;

// Whether rows can be filled as they are (their array is 16-byte aligned then: see check_inputs).
bool fills_take(int64_t ld, int64_t cols) { return ld % 8 == 0 && cols % 8 == 0; }

struct Shape {                           // of a product's launch
    bool large;                          // tiles of 256 x 256, else 128 x 128
    int64_t tiles_m, tiles_n, whole, splits;
    double cost;
    int64_t blocks() const { return whole + (tiles_m * tiles_n - whole) * splits; }
    int64_t partial_bytes() const { return splits > 1 ? (tiles_m * tiles_n - whole) * splits * (large ? 256 * 256 : 128 * 128) * 4 : 0; }
};
// Which tiles, and how the inner dimension is split: what is quickest by this reckoning, in us.  A round of tiles takes its stages, 1.55 each of
// a 256 x 256 tile, one a compute unit, 1.2 of two of 128 x 128.  The tiles beyond whole rounds may be split so that their blocks fill the chip
// once, into at most 32 shares (488 tokens of 128 x 17536 backward 61 us, with 16 66, with 64 69) of at least eight stages; then their sums are written and read at 2.5 TB/s, with a launch of 5.  Against measured
// times (bf16, silu, forward with the projections stored), large tiles | small ones: 300 tokens of 2048 x 5632 40 | 38, reckoned 38 | 38; 512 of 4096 x 11008 108 (by now 99) | 133, 99 | 124;
// 2000 of 4096 x 512 43 | 35, 44 | 36; 4000 of 1024 x 4096 77 | 109, 50 | 77 (it leaves out the stores of the result, alike in both).
// rows and columns: of the result (of WEIGHT_GRAD of one part, of FORWARD of both parts)
Shape shape_of(int mode, int64_t rows, int64_t cols, int64_t inner) {
    const int64_t stages = ceil_div(inner, STEPS) * (mode == INPUT_GRAD ? 2 : 1);
    Shape best{};
    best.cost = -1.0;
    for (const bool large : {true, false}) {
        const int64_t side = large ? 256 : 128, at_once = large ? COMPUTE_UNITS : 2 * COMPUTE_UNITS;
        Shape s{large, ceil_div(rows, side) * (mode == WEIGHT_GRAD ? 2 : 1), ceil_div(cols, mode == FORWARD ? side / 2 : side), 0, 1, 0.0};
        const int64_t tiles = s.tiles_m * s.tiles_n, rest = tiles % at_once;
        const double filled = (double)rows / (double)(ceil_div(rows, side) * side), stage = large ? 1.55 : 1.2;
        for (int64_t splits = 1; splits == 1 || (rest && rest * splits <= at_once && splits <= 32 && stages / splits >= 8); ++splits) {
            s.splits = splits;
            s.whole = splits == 1 ? tiles : tiles - rest;
            const int64_t in_turn = splits == 1 ? ceil_div(tiles, at_once) * stages : tiles / at_once * stages + ceil_div(stages, splits);
            s.cost = (double)in_turn * stage + (splits == 1 ? 0.0 : 5.0 + (double)s.partial_bytes() * filled / 2.5e6);
            if (best.cost < 0.0 || s.cost < best.cost) best = s;
        }
    }
    return best;
}

// The backward pass's two products: each for itself, or both in one launch of small tiles, all tiles of a product in equal shares.  Then the blocks take
// what all stages take on a full chip and half a short block's more, or the longest block's; by themselves there is a launch more, 5 us.  Kernel times of the
// whole pass (bf16), by themselves | together: 100 tokens of 768 x 2048 25 | 20, 474 of 384 x 896 30 | 20, 500 of 1024 x 2816 43 | 34, 1000 of 2048 x 2048
// 62 | 54, 128 of 4096 x 4096 64 | 55, 4000 of 512 x 1024 60 | 46; but 600 of 4096 x 11008 281 | 345, 3740 of 640 x 5504 188 | 193.
struct Shapes {
    Shape dx, dw;
    bool together;
    int64_t dw_partial() const { return together ? up_to(dx.partial_bytes(), 256) : 0; }
    int64_t partial_bytes() const { return std::max(dx.partial_bytes(), dw_partial() + dw.partial_bytes()); }
};
Shapes shapes_of(int64_t n, int64_t dim, int64_t hidden) {
    Shapes best{shape_of(INPUT_GRAD, n, dim, hidden), shape_of(WEIGHT_GRAD, hidden, dim, n), false};
    double least = best.dx.cost + best.dw.cost + 5.0;
    const auto small = [](int64_t tiles_m, int64_t tiles_n, int64_t splits) {
        return Shape{false, tiles_m, tiles_n, splits == 1 ? tiles_m * tiles_n : 0, splits, 0.0};
    };
    const int64_t of_dx = ceil_div(hidden, STEPS) * 2, of_dw = ceil_div(n, STEPS), side_m = ceil_div(n, 128), side_h = ceil_div(hidden, 128) * 2,
                  side_d = ceil_div(dim, 128);
    const double filled = (double)n / (double)(side_m * 128);
    const double all = (double)(side_m * side_d * of_dx + side_h * side_d * of_dw) / (2 * COMPUTE_UNITS);
    for (const int64_t dw_splits : {1, 2, 4, 8, 16}) {
        if (dw_splits > 1 && of_dw / dw_splits < 8) break;
        const Shape dw = small(side_h, side_d, dw_splits);
        for (const int64_t dx_splits : {1, 2, 3, 4, 6, 8, 11, 16, 23, 32}) {
            if (dx_splits > 1 && of_dx / dx_splits < 8) break;
            const Shape dx = small(side_m, side_d, dx_splits);
            const int64_t a = ceil_div(of_dx, dx_splits), b = ceil_div(of_dw, dw_splits);
            const double cost = 1.2 * std::max((double)std::max(a, b), all + 0.5 * (double)std::min(a, b)) + (dx_splits > 1 ? 5.0 : 0.0) +
                                (dw_splits > 1 ? 5.0 : 0.0) + ((double)dx.partial_bytes() * filled + (double)dw.partial_bytes()) / 2.5e6;
            if (cost < least) {
                least = cost;
                best = Shapes{dx, dw, true};
            }
        }
    }
    return best;
}

template <class Kernel>
int room_for(Kernel kernel, unsigned lds_bytes) {
    if (lds_bytes <= 65536) return PARO_OK;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_bytes);
    return e == hipSuccess ? PARO_OK : fail(PARO_EHIP, std::string("shared memory: ") + hipGetErrorString(e));
}
void place(Product &p, const Shape &s, float *partial) {
    p.tiles_m = (int)s.tiles_m;
    p.tiles_n = (int)s.tiles_n;
    p.whole = (unsigned)s.whole;
    p.splits = (unsigned)s.splits;
    p.partial = partial;
}
template <int DT, int MODE, int ACT, int BM, int BN, int WAVES_M, int WAVES_N>
void launch_join(const Product &p, const Shape &s, hipStream_t st) {
    if (s.splits > 1)
        hipLaunchKernelGGL((k_join<DT, MODE, ACT, BM, BN, WAVES_M, WAVES_N>), dim3((unsigned)(s.tiles_m * s.tiles_n - s.whole), BM / WAVES_M / 16),
                           dim3(64 * WAVES_M * WAVES_N), 0, st, p);
}

template <int DT, int MODE, int ACT, int BM, int BN, int WAVES_M, int WAVES_N>
int launch_tiles(const Product &p, const Shape &s, hipStream_t st) {
    constexpr unsigned LDS_BYTES = 5 * BM * ROW_BYTES;
    const auto kernel = k_product<DT, MODE, ACT, BM, BN, WAVES_M, WAVES_N>;
    if (const int rc = room_for(kernel, LDS_BYTES)) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)s.blocks()), dim3(64 * WAVES_M * WAVES_N), LDS_BYTES, st, p);
    launch_join<DT, MODE, ACT, BM, BN, WAVES_M, WAVES_N>(p, s, st);
    return PARO_OK;
}

template <int DT, int MODE, int ACT>
int launch_product(Product p, const Shape &s, float *partial, hipStream_t st) {
    place(p, s, partial);
    return s.large ? launch_tiles<DT, MODE, ACT, 256, 256, 2, 4>(p, s, st) : launch_tiles<DT, MODE, ACT, 128, 128, 2, 2>(p, s, st);
}

template <int DT>
int launch_products(Product dx, Product dw, const Shapes &s, float *partial, hipStream_t st) {
    constexpr unsigned LDS_BYTES = 5 * 128 * ROW_BYTES;
    place(dx, s.dx, partial);
    place(dw, s.dw, partial + s.dw_partial() / 4);
    const auto kernel = k_products<DT, 128, 128, 2, 2>;
    if (const int rc = room_for(kernel, LDS_BYTES)) return rc;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(s.dx.blocks() + s.dw.blocks())), dim3(64 * 2 * 2), LDS_BYTES, st, dx, dw, (unsigned)s.dx.blocks());
    launch_join<DT, INPUT_GRAD, PARO_SILU, 128, 128, 2, 2>(dx, s.dx, st);
    launch_join<DT, WEIGHT_GRAD, PARO_SILU, 128, 128, 2, 2>(dw, s.dw, st);
    return PARO_OK;
}

struct Room {                            // parts of the workspace, in bytes
    int64_t x, wg, wu, slopes, largest, partial, all;
};
int64_t ld_x(const paro_gated_t &d) { return d.ld_x ? d.ld_x : d.dim; }
int64_t ld_h(const paro_gated_t &d) { return d.ld_h ? d.ld_h : d.hidden; }

// Which backward passes k_few_grad takes (otherwise tiles, of which few rows are filled, in us, 4096 x 11008 where no size is named): 1 token 84
// (123), 2665 x 16768, whose rows have to be copied, 116 (250), 4 85 (121), 8 94 (117); 9 122 (123), 16 129 (117), 1024 x 1024 23 (22), so with more than 8 only
// where rows have to be copied, 16 of 1601 x 4099 38 (56), 12 of 2665 x 16768 139 (249), or are short, 512 x 22016 41 (64), 384 x 384 17 (21); and into how many
// shares of the hidden elements.
bool few_tokens_grad(const paro_gated_t &d) {
    return d.n >= 1 && d.dim >= 8 && (d.n <= 8 || (d.n <= 16 && (!fills_take(d.dim, d.dim) || d.dim <= 512)));
}
int64_t few_shares(const paro_gated_t &d) {
    const int64_t wanted = std::min<int64_t>(256, std::max<int64_t>(16, 1024 / ceil_div(d.dim, 64 * few_columns(d.n))));
    return ceil_div(d.hidden, std::max<int64_t>(FEW_WAVES, ceil_div(d.hidden, wanted)));
}

Room room_of(const paro_gated_t &d, bool grad) {
    const int64_t width = up_to(d.dim, 8);
    Room r{};
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += up_to(bytes, 256);
        return here;
    };
    if (!fills_take(ld_x(d), d.dim)) r.x = take(d.n * width * 2);
    if (!fills_take(d.dim, d.dim)) {
        r.wg = take(d.hidden * width * 2);
        r.wu = take(d.hidden * width * 2);
    }
    int64_t partial = 0;
    if (grad) {
        r.slopes = take(2 * up_to(d.hidden, 64) * d.n * 2);
        if (d.dtype == PARO_F16) {
            const dim3 grid = slopes_grid(d, ceil_div(d.hidden, 64), WATCHED_BLOCKS);
            r.largest = take((1 + (int64_t)grid.x * grid.y) * 4);
        }
        partial = shapes_of(d.n, d.dim, d.hidden).partial_bytes();
    } else {
        partial = shape_of(FORWARD, d.n, d.hidden, d.dim).partial_bytes();
    }
    r.partial = take(partial);
    r.all = std::max<int64_t>(at, 16);
    if (grad && few_tokens_grad(d)) {                       // its shares from the start on, in no less room than tiles would take: at odd
        r.partial = 0;                                      // sizes no less than the forward pass's, so that one workspace has one size
        r.all = std::max(r.all, few_shares(d) * d.n * d.dim * 4);
    }
    return r;
}

int check(const std::string &f, const paro_gated_t *d) {
    if (!d) return fail(PARO_EINVAL, f + "d is NULL");
    if (d->dtype != PARO_BF16 && d->dtype != PARO_F16) return fail(PARO_EINVAL, f + "dtype must be PARO_BF16 or PARO_F16");
    if (d->act != PARO_SILU && d->act != PARO_GELU) return fail(PARO_EINVAL, f + "act must be PARO_SILU or PARO_GELU");
    if (d->n < 0 || d->n > (1 << 22)) return fail(PARO_EINVAL, f + "n must be in [0, 2^22]");
    if (d->dim < 1 || d->dim > (1 << 20) || d->hidden < 1 || d->hidden > (1 << 20)) return fail(PARO_EINVAL, f + "dim and hidden must be in [1, 2^20]");
    if ((d->ld_x && d->ld_x < d->dim) || (d->ld_h && d->ld_h < d->hidden)) return fail(PARO_EINVAL, f + "a row is longer than its distance to the next");
    if (d->ld_x > (1 << 21) || d->ld_h > (1 << 21)) return fail(PARO_EINVAL, f + "ld_x and ld_h are at most 2^21");
    return PARO_OK;
}
// Where rows of x or of the weights lie on multiples of 16 bytes, so does their array.
int check_inputs(const std::string &f, const paro_gated_t *d, const void *x, const void *w_gate, const void *w_up) {
    const int64_t of_w = fills_take(d->dim, d->dim) ? 16 : 2, of_x = fills_take(ld_x(*d), d->dim) ? 16 : 2;
    int rc = PARO_OK;
    const auto check_one = [&](const void *p, int64_t size, const char *name) {
        if (rc) return;
        rc = check_array(p, 2, f + name);
        if (!rc && (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1))) rc = fail(PARO_EALIGN, f + name + " is not 16-byte aligned, as its rows are");
    };
    check_one(w_gate, of_w, "w_gate");
    check_one(w_up, of_w, "w_up");
    if (d->n) check_one(x, of_x, "x");
    return rc;
}
int check_room(const std::string &f, const Room &r, const void *workspace, int64_t bytes) {
    const int rc = check_array(workspace, 16, f + "workspace");
    if (rc) return rc;
    return bytes < r.all ? fail(PARO_ERANGE, f + "the workspace is smaller than paro_gated_workspace says") : PARO_OK;
}

// x and the weights as operands: as they are, or copies that the fills take.
struct Inputs {
    const char *x, *wg, *wu;
    int64_t ldx, ldw;
};
Inputs inputs_of(const paro_gated_t &d, const void *x, const void *wg, const void *wu, char *ws, const Room &r, hipStream_t st) {
    Inputs in{static_cast<const char *>(x), static_cast<const char *>(wg), static_cast<const char *>(wu), ld_x(d), d.dim};
    Copies c{};
    c.cols = d.dim;
    c.width = up_to(d.dim, 8);
    unsigned copies = 0;
    int64_t most = 0;
    const auto copy = [&](const char *&rows, int64_t ld, int64_t n, int64_t room) {
        c.from[copies] = rows;
        c.ld[copies] = ld;
        c.rows[copies] = n;
        most = std::max(most, n);
        c.to[copies++] = ws + room;
        rows = ws + room;
    };
    if (!fills_take(d.dim, d.dim)) {
        copy(in.wg, d.dim, d.hidden, r.wg);
        copy(in.wu, d.dim, d.hidden, r.wu);
        in.ldw = c.width;
    }
    if (!fills_take(in.ldx, d.dim)) {
        copy(in.x, in.ldx, d.n, r.x);
        in.ldx = c.width;
    }
    if (copies)
        hipLaunchKernelGGL(k_align, dim3((unsigned)std::min<int64_t>(ceil_div(most * (c.width / 8), 256 * ALIGN_PIECES), 1 << 20), copies), dim3(256), 0,
                           st, c);
    return in;
}

// Which forward passes k_few takes (otherwise tiles of 128 rows, most of them empty, in us): up to 16 tokens, 4096 x 11008 with 1 token 38 (44), 8 44
// (48), 12 47 (47), 4096 x 4096 with 16 19 (21), 4099 x 11003 with 16 90 (127); up to 64 over small weights, 1024 x 4096 with 32 12 (17), 768 x 2048 with
// 64 12 (15), but 2048 x 5632 with 32 21 (19), 4096 x 11008 with 32 63 (50): beyond, the tokens that every block reads again outweigh.
bool few_tokens(int64_t n, int64_t dim, int64_t hidden) { return n <= 16 || (n <= 64 && dim * hidden <= (int64_t)4 << 20); }

template <int DT, int ACT>
int forward(const paro_gated_t &d, const void *x, const void *wg, const void *wu, void *h, void *gate, void *up, char *ws, const Room &r,
            hipStream_t st) {
    if (few_tokens(d.n, d.dim, d.hidden)) {
#define PARO_FEW(F_TILES, N_TILES)                                                                                                         \
    hipLaunchKernelGGL((k_few<DT, ACT, F_TILES, N_TILES>), dim3((unsigned)ceil_div(d.hidden, 16 * F_TILES)), dim3(64 * FEW_WAVES), 0, st,          \
                       static_cast<const char *>(x), static_cast<const char *>(wg), static_cast<const char *>(wu), d.n, d.dim, d.hidden,   \
                       ld_x(d), ld_h(d), static_cast<char *>(h), static_cast<char *>(gate),             \
                       static_cast<char *>(up))
        if (d.n <= 16) PARO_FEW(1, 1);
        else if (d.n <= 32) PARO_FEW(1, 2);
        else PARO_FEW(1, 4);
#undef PARO_FEW
        return PARO_OK;
    }
    const Inputs in = inputs_of(d, x, wg, wu, ws, r, st);
    Product p{};
    p.a[0] = in.x;
    p.b[0] = in.wg;
    p.b[1] = in.wu;
    p.lda = in.ldx * 2;
    p.ldb = in.ldw * 2;
    p.rows = d.n;
    p.cols = d.hidden;
    p.inner = p.inner_b = up_to(d.dim, 8);
    p.out[0] = static_cast<char *>(h);
    p.out[1] = static_cast<char *>(gate);
    p.out[2] = static_cast<char *>(up);
    p.ldo = ld_h(d);
    return launch_product<DT, FORWARD, ACT>(p, shape_of(FORWARD, d.n, d.hidden, d.dim), reinterpret_cast<float *>(ws + r.partial), st);
}

template <int DT, int ACT>
int backward(const paro_gated_t &d, const void *dh, const void *gate, const void *up, const void *x, const void *wg, const void *wu, void *dx,
             void *dwg, void *dwu, char *ws, const Room &r, hipStream_t st) {
    Product p{};
    if (d.n == 0) {                                         // no token, no stage: the tiles of dWg and dWu are zeros
        p.rows = d.hidden;
        p.cols = p.ldo = d.dim;
        p.out[0] = static_cast<char *>(dwg);
        p.out[1] = static_cast<char *>(dwu);
        return launch_product<DT, WEIGHT_GRAD, PARO_SILU>(p, shape_of(WEIGHT_GRAD, d.hidden, d.dim, 0), nullptr, st);
    }
    if (few_tokens_grad(d)) {
        const int64_t shares = few_shares(d);
        float *sums = reinterpret_cast<float *>(ws + r.partial);
#define PARO_FEW_GRAD(N)                                                                                                                  \
    hipLaunchKernelGGL((k_few_grad<DT, ACT, N>), dim3((unsigned)shares, (unsigned)ceil_div(d.dim, 64 * few_columns(N))), dim3(64 * FEW_WAVES), 0, st, dh, gate, up, x, \
                       wg, wu, (int)d.n, d.dim, d.hidden, ld_x(d), ld_h(d), ceil_div(d.hidden, shares), dwg, dwu, sums)
        if (d.n <= 1) PARO_FEW_GRAD(1);
        else if (d.n <= 4) PARO_FEW_GRAD(4);
        else if (d.n <= 8) PARO_FEW_GRAD(8);
        else PARO_FEW_GRAD(16);
#undef PARO_FEW_GRAD
        hipLaunchKernelGGL((k_few_join<DT>), dim3((unsigned)ceil_div(d.dim, 64), (unsigned)d.n), dim3(512), 0, st, sums, (int)d.n, d.dim, (int)shares, ld_x(d), dx);
        return PARO_OK;
    }
    const Inputs in = inputs_of(d, x, wg, wu, ws, r, st);
    const int64_t panels = ceil_div(d.hidden, 64);
    char *slopes = ws + r.slopes;
    float *partial = reinterpret_cast<float *>(ws + r.partial);
    const dim3 grid = DT == PARO_F16 ? slopes_grid(d, panels, WATCHED_BLOCKS) : dim3((unsigned)ceil_div(panels, 4), (unsigned)std::min<int64_t>(ceil_div(d.n, 8), 65535));
    float *largest = reinterpret_cast<float *>(ws + r.largest);
    const Slopes of{dh, gate, up, ld_h(d), d.n, d.hidden, panels, slopes, largest, largest + 1, (int)(grid.x * grid.y)};
    hipLaunchKernelGGL((k_slopes<DT, ACT, false>), grid, dim3(256), 0, st, of);
    if constexpr (DT == PARO_F16) {
        hipLaunchKernelGGL((k_slopes<DT, ACT, true>), slopes_grid(d, panels, AGAIN_BLOCKS), dim3(256), 0, st, of);
        p.back = largest;
    }
    p.panel = d.n * ROW_BYTES;
    p.a[0] = slopes;
    p.a[1] = slopes + panels * p.panel;
    p.b[0] = in.wg;
    p.b[1] = in.wu;
    p.ldb = in.ldw * 2;
    p.rows = d.n;
    p.cols = d.dim;
    p.inner = panels * 64;
    p.inner_b = d.hidden;
    p.out[0] = static_cast<char *>(dx);
    p.ldo = ld_x(d);
    Product q = p;
    q.b[0] = in.x;
    q.b[1] = nullptr;
    q.ldb = in.ldx * 2;
    q.rows = d.hidden;
    q.inner = q.inner_b = d.n;
    q.out[0] = static_cast<char *>(dwg);
    q.out[1] = static_cast<char *>(dwu);
    q.ldo = d.dim;
    const Shapes s = shapes_of(d.n, d.dim, d.hidden);
    if (s.together) return launch_products<DT>(p, q, s, partial, st);
    const int rc = launch_product<DT, INPUT_GRAD, PARO_SILU>(p, s.dx, partial, st);
    return rc ? rc : launch_product<DT, WEIGHT_GRAD, PARO_SILU>(q, s.dw, partial, st);
}

#define PARO_BY_TYPE(CALL)                                            \
    (d->dtype == PARO_BF16 ? d->act == PARO_SILU ? CALL(PARO_BF16, PARO_SILU) : CALL(PARO_BF16, PARO_GELU) \
                           : d->act == PARO_SILU ? CALL(PARO_F16, PARO_SILU) : CALL(PARO_F16, PARO_GELU))

}  // namespace

extern "C" {

int64_t paro_gated_workspace(const paro_gated_t *d, int grad) {
    int64_t bytes = 0;
    const int rc = guarded([&]() -> int {
        const int bad = check("paro_gated_workspace: ", d);
        if (!bad) bytes = room_of(*d, grad != 0).all;
        return bad;
    });
    return rc ? rc : bytes;
}

int paro_gated(const paro_gated_t *d, const void *x, const void *w_gate, const void *w_up, void *h, void *gate, void *up, void *workspace,
               int64_t workspace_bytes, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_gated: ";
        int rc;
        if ((rc = check(f, d)) || d->n == 0) return rc;
        if ((rc = check_inputs(f, d, x, w_gate, w_up)) || (rc = check_array(h, 2, f + "h"))) return rc;
        if (!gate != !up) return fail(PARO_EINVAL, f + "gate and up are stored both or neither");
        if (gate && ((rc = check_array(gate, 2, f + "gate")) || (rc = check_array(up, 2, f + "up")))) return rc;
        const Room r = room_of(*d, false);
        if ((rc = check_room(f, r, workspace, workspace_bytes))) return rc;
        hipStream_t st = static_cast<hipStream_t>(stream);
        char *ws = static_cast<char *>(workspace);
#define PARO_FORWARD(DT, ACT) forward<DT, ACT>(*d, x, w_gate, w_up, h, gate, up, ws, r, st)
        if ((rc = PARO_BY_TYPE(PARO_FORWARD))) return rc;
#undef PARO_FORWARD
        PARO_LAUNCHED("paro_gated");
        return PARO_OK;
    });
}

int paro_gated_grad(const paro_gated_t *d, const void *dh, const void *gate, const void *up, const void *x, const void *w_gate, const void *w_up,
                    void *dx, void *dw_gate, void *dw_up, void *workspace, int64_t workspace_bytes, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_gated_grad: ";
        int rc;
        if ((rc = check(f, d))) return rc;
        if ((rc = check_inputs(f, d, x, w_gate, w_up)) || (rc = check_array(dw_gate, 2, f + "dw_gate")) || (rc = check_array(dw_up, 2, f + "dw_up")))
            return rc;
        if (d->n && ((rc = check_array(dh, 2, f + "dh")) || (rc = check_array(gate, 2, f + "gate")) || (rc = check_array(up, 2, f + "up")) ||
                     (rc = check_array(dx, 2, f + "dx"))))
            return rc;
        const Room r = room_of(*d, true);
        if ((rc = check_room(f, r, workspace, workspace_bytes))) return rc;
        hipStream_t st = static_cast<hipStream_t>(stream);
        char *ws = static_cast<char *>(workspace);
#define PARO_BACKWARD(DT, ACT) backward<DT, ACT>(*d, dh, gate, up, x, w_gate, w_up, dx, dw_gate, dw_up, ws, r, st)
        if ((rc = PARO_BY_TYPE(PARO_BACKWARD))) return rc;
#undef PARO_BACKWARD
        PARO_LAUNCHED("paro_gated_grad");
        return PARO_OK;
    });
}

}  // extern "C"
