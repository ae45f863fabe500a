// Embedding lookup with scaling and its gradient (gfx950).
//
//   out[i]  = scale * table[t_i - first]                      zeros where the table does not hold token t_i
//   grad[v] = scale * sum over { i : t_i - first = v } of dout[i]
//
// Both move bytes and do next to no arithmetic: the lookup reads and writes n rows, the gradient reads n rows and writes
// every row of the table's gradient.  The sums run in fp32, in an order that the tokens alone fix (no atomics on data: run-to-
// run identical), scaled and rounded once.
#include "operators.hpp"

namespace {

constexpr int WAVES = 4;                 // waves of a block: each works for itself
constexpr int THREADS = 64 * WAVES;
constexpr int COMPUTE_UNITS = 256;
constexpr int64_t MAX_BLOCKS = 1 << 22;  // of a launch (tiles counted); beyond, waves take several rows

__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
__device__ __forceinline__ int lane_of() { return threadIdx.x & 63; }

template <class Token>
__device__ __forceinline__ int64_t row_of(const Token *tokens, int64_t i, int64_t first, int64_t rows) {
    const uint64_t r = (uint64_t)(int64_t)tokens[i] - (uint64_t)first;
    return r < (uint64_t)rows ? (int64_t)r : -1;
}

// ---------------------------------------------------------------- lookup
// A wave copies a tile of a row: PIECES pieces a lane, all in flight.  The last piece of a row whose width is no multiple of a
// piece starts early and writes some elements twice, with the same values; rows narrower than a piece go element by element.
constexpr int PIECES = 4;

template <int DT, class Token>
__global__ __launch_bounds__(THREADS) void k_embed(const void *table, const Token *tokens, int64_t n, int64_t first, int64_t rows,
                                                   int64_t dim, float scale, void *out, int64_t ld_out) {
    constexpr int E = Elem<DT>::E;
    const int64_t at = (int64_t)blockIdx.y * (64 * PIECES * E) + lane_of() * E;
    for (int64_t i = (int64_t)blockIdx.x * WAVES + wave_of(); i < n; i += (int64_t)gridDim.x * WAVES) {
        const int64_t r = row_of(tokens, i, first, rows);
        if (dim < E) {
            if (lane_of() < dim) store_one<DT>(out, i * ld_out + lane_of(), r < 0 ? 0.0f : load_one<DT>(table, r * dim + lane_of()) * scale);
            continue;
        }
        u32x4 raw[PIECES];
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int64_t e = at + p * 64 * E;
            raw[p] = u32x4{0, 0, 0, 0};
            if (r >= 0 && e < dim) raw[p] = load_piece<DT>(table, r * dim + (e < dim - E ? e : dim - E));
        }
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int64_t e = at + p * 64 * E;
            if (e >= dim) continue;
            float x[E];
            unpack<DT>(raw[p], x);
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = r < 0 ? 0.0f : x[j] * scale;
            store_piece<DT>(out, i * ld_out + (e < dim - E ? e : dim - E), pack<DT>(x));
        }
    }
}

// ---------------------------------------------------------------- tokens sorted by row, in order
// A block takes SORT_ROWS rows of the table and reads a slice of the tokens: its sixteen waves walk consecutive parts of it twice - to
// count theirs for each row in counters of their own and, after a scan over rows, slices and waves, to write them to their places.
// Tokens of one row keep their order, nothing is atomic, no block waits for another.  A wave collects its block's tokens, one in many, in
// a ring and works on 64 at a time.  Up to SLICE tokens are one slice and one launch; of more, a launch before counts every slice's.
constexpr int SORT_BITS = 9, SORT_ROWS = 1 << SORT_BITS, SORT_WAVES = 16, SORT_THREADS = 64 * SORT_WAVES;
constexpr int SORT_RING = 128, SORT_AHEAD = 8;     // tokens a lane loads ahead
constexpr int64_t SLICE = SORT_AHEAD * SORT_THREADS;  // 32768 tokens in one slice 30 us, in slices of 4096 25, of 8192 18
constexpr int64_t MAX_SLICES = 16;

// Lanes with the same row as this one, among `in`.
__device__ __forceinline__ uint64_t same_row(int row, uint64_t in) {
#pragma unroll
    for (int b = 0; b < SORT_BITS; ++b) {
        const uint64_t set = __ballot((row >> b) & 1);
        in &= (row >> b) & 1 ? set : ~set;
    }
    return in;
}

// The slices' counts: of each row [slices][rows], and of the tokens in rows before a block's [slices][blocks].
struct SliceCounts {
    int *of_row, *below;
};

template <class Token, bool COUNT>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_tokens(const Token *tokens, int64_t n, int64_t first, int64_t rows, int64_t slice,
                                                              SliceCounts counts, int *start, int *order, int *row_at) {
    __shared__ int count[SORT_WAVES][SORT_ROWS];
    __shared__ int ring_row[SORT_WAVES][SORT_RING], ring_at[SORT_WAVES][SORT_RING];
    __shared__ int wave_total[SORT_ROWS / 64];
    __shared__ int below_of[SORT_WAVES];
    const int w = wave_of(), lane = lane_of();
    const int64_t lo = (int64_t)blockIdx.x * SORT_ROWS;
    const int in_range = (int)(lo + SORT_ROWS < rows ? SORT_ROWS : rows - lo);
    const int64_t from_token = blockIdx.y * slice, to_token = from_token + slice < n ? from_token + slice : n;
    const int64_t part = (slice + SORT_THREADS - 1) / SORT_THREADS * 64;
    const int64_t begin = from_token + w * part, end = begin + part < to_token ? begin + part : to_token;
    const uint64_t before = ((uint64_t)1 << lane) - 1;

    uint64_t next[SORT_AHEAD];
    const auto load = [&](int64_t from) {
#pragma unroll
        for (int u = 0; u < SORT_AHEAD; ++u) {
            const int64_t i = from + u * 64 + lane;
            next[u] = i < end ? (uint64_t)(int64_t)tokens[i] - (uint64_t)first : ~(uint64_t)0;
        }
    };
    // visit(row, i, place) for the tokens of the block's rows, in order; place counts on from what the wave's counter of the row holds.
    // Returns how many tokens lie in rows before the block's.  The first tokens are loaded before it is called.
    const auto walk = [&](auto &&visit) {
        int below = 0, held = 0, head = 0;
        const auto number = [&](int of) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            const int row = ring_row[w][(head + lane) & (SORT_RING - 1)], at = ring_at[w][(head + lane) & (SORT_RING - 1)];
            const uint64_t same = same_row(row, of == 64 ? ~(uint64_t)0 : ((uint64_t)1 << of) - 1);
            if (lane < of) {
                const int place = count[w][row], rank = __popcll(same & before);
                if (rank == 0) count[w][row] = place + __popcll(same);
                visit(row, at, place + rank);
            }
            head += of;
            held -= of;
        };
        for (int64_t from = begin; from < end; from += SORT_AHEAD * 64) {
            uint64_t now[SORT_AHEAD];
#pragma unroll
            for (int u = 0; u < SORT_AHEAD; ++u) now[u] = next[u];
            if (from + SORT_AHEAD * 64 < end) load(from + SORT_AHEAD * 64);
#pragma unroll
            for (int u = 0; u < SORT_AHEAD; ++u) {
                below += __popcll(__ballot(now[u] < (uint64_t)lo));
                const bool mine = now[u] - (uint64_t)lo < (uint64_t)in_range;
                const uint64_t in = __ballot(mine);
                if (!in) continue;
                if (mine) {
                    const int to = (head + held + __popcll(in & before)) & (SORT_RING - 1);
                    ring_row[w][to] = (int)(now[u] - (uint64_t)lo);
                    ring_at[w][to] = (int)(from + u * 64 + lane);
                }
                held += __popcll(in);
                if (held >= 64) number(64);
            }
        }
        if (held) number(held);
        return below;
    };

    load(begin);
    for (int r = lane; r < SORT_ROWS; r += 64) count[w][r] = 0;
    const int below = walk([](int, int, int) {});
    if constexpr (!COUNT) load(begin);              // for the second walk, on their way during the scan
    if (lane == 0) below_of[w] = below;
    __syncthreads();

    // The row of each of the first threads: tokens before it in the block's range, then where each wave's begin.
    const int mine = threadIdx.x;
    int total = 0, sum = 0, before_slice = 0;
    if (mine < SORT_ROWS) {
#pragma unroll
        for (int k = 0; k < SORT_WAVES; ++k) total += count[k][mine];
        if constexpr (COUNT) {
            if (mine < in_range) counts.of_row[blockIdx.y * rows + lo + mine] = total;
            if (mine == 0) {
                int all = 0;
                for (int k = 0; k < SORT_WAVES; ++k) all += below_of[k];
                counts.below[blockIdx.y * gridDim.x + blockIdx.x] = all;
            }
            return;
        }
        if (gridDim.y > 1) {
            int of_slice[MAX_SLICES];               // all on their way at once
#pragma unroll
            for (unsigned s = 0; s < MAX_SLICES; ++s) of_slice[s] = s < gridDim.y && mine < in_range ? counts.of_row[s * rows + lo + mine] : 0;
            total = 0;
#pragma unroll
            for (unsigned s = 0; s < MAX_SLICES; ++s) {
                total += of_slice[s];
                before_slice += s < blockIdx.y ? of_slice[s] : 0;
            }
        }
        sum = total;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const int other = __shfl_up(sum, step);
            if (lane >= step) sum += other;
        }
        if (lane == 63) wave_total[w] = sum;
    }
    if constexpr (COUNT) return;
    __syncthreads();
    if (mine < SORT_ROWS) {
        int at = sum - total;
        for (int k = 0; k < w; ++k) at += wave_total[k];
        if (gridDim.y > 1) {
            int below_in[MAX_SLICES];
#pragma unroll
            for (unsigned s = 0; s < MAX_SLICES; ++s) below_in[s] = s < gridDim.y ? counts.below[s * gridDim.x + blockIdx.x] : 0;
#pragma unroll
            for (unsigned s = 0; s < MAX_SLICES; ++s) at += below_in[s];
        } else {
#pragma unroll
            for (int k = 0; k < SORT_WAVES; ++k) at += below_of[k];
        }
        if (blockIdx.y == 0 && mine < in_range) {
            start[lo + mine] = at;
            if (lo + mine == rows - 1) start[rows] = at + total;
        }
        at += before_slice;
#pragma unroll
        for (int k = 0; k < SORT_WAVES; ++k) {
            const int c = count[k][mine];
            count[k][mine] = at;
            at += c;
        }
    }
    __syncthreads();

    walk([&](int row, int i, int place) {
        order[place] = i;
        row_at[place] = (int)lo + row;
    });
}

// Pieces a lane of the sums takes at most (2: GPT-2's table 51 us, not 47, 32768 tokens of 4096 179, not 138); one where that would leave too few
// waves (few_waves, below), and no more than a row has for it (4 whatever the width: 60000 tokens of 640 90 us, so 84; of 64 fp32 elements 66, so 60).
// 16 rows' pieces are in flight in any case.
constexpr int GRAD_PIECES = 4;
// ---------------------------------------------------------------- sums over the sorted tokens
// What a lane loads of a row of dout: as many elements as a piece of the gradient has, so that every store instruction of a wave covers
// whole cache lines (fp32 gradients of two-byte rows in pieces of dout, 32 bytes a lane: GPT-2's table 56 us, so 40).
template <int DT, int GT>
struct RowPiece {
    static constexpr int N = Elem<GT>::E;
    static constexpr bool HALF = N < Elem<DT>::E;
    u32x4 raw;
    __device__ __forceinline__ void load(const void *dout, int64_t elem) {
        if constexpr (HALF) {
            const u32x2 r = load_half_piece_stream(dout, elem);
            raw[0] = r[0];
            raw[1] = r[1];
        } else {
            raw = load_stream<DT>(dout, elem);
        }
    }
    __device__ __forceinline__ void add_to(float (&acc)[N]) const {
        float x[Elem<DT>::E];
        unpack<DT>(raw, x);
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] += x[j];
    }
};

// acc += dout's rows in the first `all` lanes of `mine`, in order, for the lane's pieces of a tile of columns.
template <int DT, int GT, int C>
__device__ __forceinline__ void add_listed(float (&acc)[C][Elem<GT>::E], const void *dout, int64_t ld, int mine, int all, const int64_t (&col)[C], int64_t dim) {
    constexpr int U = 16 / C;                       // rows in flight; for four pieces 2: 52 and 149 us, 6: 46 and 145
    const auto add = [&](int k, auto count_) {
        constexpr int count = count_;
        RowPiece<DT, GT> piece[count][C];
#pragma unroll
        for (int u = 0; u < count; ++u) {
            const int64_t row = (int64_t)__builtin_amdgcn_readlane(mine, k + u) * ld;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (col[c] < dim) piece[u][c].load(dout, row + col[c]);
        }
#pragma unroll
        for (int u = 0; u < count; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (col[c] < dim) piece[u][c].add_to(acc[c]);
    };
    int k = 0;
    for (; k + U <= all; k += U) add(k, std::integral_constant<int, U>{});
    static_for<1, 5>([&](auto i) {                  // the rest in halves; row by row 30000 tokens of 128 43 us, so 38
        constexpr int fewer = U >> i;
        if constexpr (fewer > 0)
            if (k + fewer <= all) {
                add(k, std::integral_constant<int, fewer>{});
                k += fewer;
            }
    });
}

// acc += dout[order[a .. b)], in order.  The places of 64 tokens are loaded at once, one a lane (each by a scalar load that its row waits for:
// GPT-2's table 64 us, so 47; 32768 tokens of 4096 155 and 138).
template <int DT, int GT, int C>
__device__ __forceinline__ void add_rows(float (&acc)[C][Elem<GT>::E], const void *dout, int64_t ld, const int *order, int a, int b,
                                         const int64_t (&col)[C], int64_t dim) {
    const int *at = order + a, *end = order + b;        // addresses: 64 beyond the last place may take more than 32 bits
    for (; at < end; at += 64)
        add_listed<DT, GT>(acc, dout, ld, at + lane_of() < end ? at[lane_of()] : 0, end - at < 64 ? (int)(end - at) : 64, col, dim);
}

// Columns of a lane's pieces; the last piece of a row starts early, past the row: dim.
template <int E, int C>
__device__ __forceinline__ void columns(int64_t (&col)[C], int64_t dim) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t e = (int64_t)blockIdx.y * (64 * C * E) + c * 64 * E + lane_of() * E;
        col[c] = e >= dim ? dim : e < dim - E ? e : dim - E;
    }
}

template <int GT, int C>
__device__ __forceinline__ void store_row(float (&acc)[C][Elem<GT>::E], void *grad, int64_t v, const int64_t (&col)[C], int64_t dim, float scale) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (col[c] >= dim) continue;
#pragma unroll
        for (int j = 0; j < Elem<GT>::E; ++j) acc[c][j] *= scale;
        store_stream<GT>(grad, v * dim + col[c], pack<GT>(acc[c]));
    }
}

// A lane's pieces of a span of the gradient as it lies in memory, `step` elements apart.
template <int C>
struct SpanPieces {
    int64_t elem[C], row[C], left[C];               // first element, its row, what that row has from it on
    unsigned empty[C];                              // bit 0: the row has no token, bit 1: the next one has none
    __device__ __forceinline__ void place(int64_t from, int step, int piece, int64_t row0, int64_t dim) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            elem[c] = from + c * step + lane_of() * piece;
            const int64_t at = elem[c] > 0 ? elem[c] : 0;
            row[c] = row0 + (unsigned)(at - row0 * dim) / (unsigned)dim;
            left[c] = (row[c] + 1) * dim - elem[c];
        }
    }
    // Zeros where the row is empty.  A piece that a row with tokens shares goes element by element.
    template <int GT>
    __device__ __forceinline__ void store(void *grad, int64_t all) const {
        constexpr int E = Elem<GT>::E;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (elem[c] >= 0 && elem[c] + E <= all && (empty[c] & 1) && (left[c] >= E || (empty[c] & 2))) {
                store_stream<GT>(grad, elem[c], u32x4{0, 0, 0, 0});
            } else {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (elem[c] + j >= 0 && elem[c] + j < all && (empty[c] & (j < left[c] ? 1 : 2))) store_one<GT>(grad, elem[c] + j, 0.0f);
            }
        }
    }
};
template <int GT, int C>
__device__ __forceinline__ void store_zeros(void *grad, int64_t from) {
#pragma unroll
    for (int c = 0; c < C; ++c) store_stream<GT>(grad, from + (c * 64 + lane_of()) * Elem<GT>::E, u32x4{0, 0, 0, 0});
}

// Zeros for the rows without a token, in a span of the gradient as it lies in memory: aligned pieces, whatever the rows' width, and all lanes
// have some, however narrow the rows are (a wave for each row: 35224 rows of 7443 fp32 elements 277 us, so 188; 87603 of 128 24 and 15). 
template <int GT, int C>
__device__ __forceinline__ void zeros_of_span(void *grad, const int *start, int64_t from, int64_t rows, int64_t dim) {
    constexpr int E = Elem<GT>::E;
    const int64_t row0 = (from > 0 ? from : 0) / dim, all = rows * dim;
    if (from + 64 * C * E <= (row0 + 1) * dim) {    // of one row: nothing to find out by lane (32768 tokens of 4096 145 us without, 133)
        if (start[row0] != start[row0 + 1]) return;
        if (from >= 0) return store_zeros<GT, C>(grad, from);
    }
    SpanPieces<C> at;
    at.place(from, 64 * E, E, row0, dim);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t v = at.row[c], v0 = v < rows ? v : rows, v1 = v + 1 < rows ? v + 1 : rows, v2 = v + 2 < rows ? v + 2 : rows;
        const int s0 = start[v0], s1 = start[v1], s2 = start[v2];
        at.empty[c] = (s0 == s1 ? 1 : 0) | (s1 == s2 ? 2 : 0);
    }
    at.template store<GT>(grad, all);
}

// Three kinds of blocks, in the order in which they start: what reads goes before what only writes, since a read that waits behind a stream of
// stores takes microseconds (GPT-2's table 52 us with the rows in their own order, so 47; 32768 tokens of 4096 141 and 138).
//   segments   a wave takes a segment of the sorted tokens: runs of more than `seg` are summed segment by segment, in parallel.  Of one
//              segment such a run holds the beginning (slot 0), or the end and not the beginning (slot 1)
//   runs       a wave takes a place among the sorted tokens, and sums the run that begins there, if a short one does
//   the rest   a wave takes a span of the table's gradient and writes zeros where no token is of the row
template <int DT, int GT, int C>
__global__ __launch_bounds__(THREADS) void k_sums(const void *dout, int64_t ld, const int *start, const int *order, const int *row_at, int64_t rows,
                                                  int64_t dim, int seg, unsigned seg_blocks, unsigned run_blocks, float scale, float *partial, void *grad) {
    constexpr int E = Elem<GT>::E;
    int64_t col[C];
    columns<E>(col, dim);
    if (blockIdx.x < seg_blocks) {
        const int64_t s = (int64_t)blockIdx.x * WAVES + wave_of();
        const int held = start[rows];
        if (s * seg >= held) return;
        const int a = (int)(s * seg), b = held - a > seg ? a + seg : held;      // the last segment's full end may take more than 32 bits
        const int rows_of[2] = {row_at[a], row_at[b - 1]};
        for (int slot = 0; slot < 2; ++slot) {
            if (slot == 1 && rows_of[1] == rows_of[0]) break;
            const int from = start[rows_of[slot]], to = start[rows_of[slot] + 1];
            if (to - from <= seg) continue;
            float acc[C][E] = {};
            add_rows<DT, GT>(acc, dout, ld, order, from > a ? from : a, to < b ? to : b, col, dim);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (col[c] < dim)
#pragma unroll
                    for (int j = 0; j < E; j += 4) store_piece<PARO_F32>(partial, (2 * s + slot) * dim + col[c] + j, pack<PARO_F32>(&acc[c][j]));
        }
    } else if (blockIdx.x < seg_blocks + run_blocks) {
        const int held = start[rows];
        for (int64_t a = (int64_t)(blockIdx.x - seg_blocks) * WAVES + wave_of(); a < held; a += (int64_t)run_blocks * WAVES) {
            const int v = row_at[a], b = start[v + 1];
            if (start[v] != a || b - a > seg) continue;
            float acc[C][E] = {};
            add_rows<DT, GT>(acc, dout, ld, order, (int)a, b, col, dim);
            store_row<GT>(acc, grad, v, col, dim, scale);
        }
    } else {
        const unsigned first = seg_blocks + run_blocks, blocks = gridDim.x - first;
        const int64_t lead = (reinterpret_cast<uintptr_t>(grad) & 127) / Elem<GT>::BYTES, all = rows * dim;
        for (int64_t s = ((int64_t)blockIdx.y * blocks + (blockIdx.x - first)) * WAVES + wave_of(); s * (64 * GRAD_PIECES * E) - lead < all;
             s += (int64_t)blocks * gridDim.y * WAVES)
            zeros_of_span<GT, GRAD_PIECES>(grad, start, s * (64 * GRAD_PIECES * E) - lead, rows, dim);
    }
}

// A wave adds up the segments of the long run that begins in its segment, if one does: the last one there.  Four columns a lane and 16
// segments in flight: few waves have anything to do, and the longest run, which many segments hold, decides.
template <int GT>
__global__ __launch_bounds__(THREADS) void k_join(const int *start, const int *row_at, int64_t rows, int64_t dim, int seg, float scale,
                                                  const float *partial, void *grad) {
    constexpr int U = 16;
    int64_t col[1];
    columns<4>(col, dim);
    const int64_t s0 = (int64_t)blockIdx.x * WAVES + wave_of();
    const int held = start[rows];
    if (s0 * seg >= held) return;
    const int a = (int)(s0 * seg), end = held - a > seg ? a + seg : held;
    const int v = row_at[end - 1], from = start[v], to = start[v + 1];
    if (from < a || to - from <= seg || col[0] >= dim) return;
    float acc[4] = {};
    for (int64_t s = s0; s * seg < to; s += U) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if ((s + u) * seg < to) raw[u] = load_piece<PARO_F32>(partial, (2 * (s + u) + ((s + u) * seg < from ? 1 : 0)) * dim + col[0]);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if ((s + u) * seg < to) {
                float x[4];
                unpack<PARO_F32>(raw[u], x);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[q] += x[q];
            }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q] *= scale;
    if constexpr (GT == PARO_F32) store_piece<GT>(grad, v * dim + col[0], pack<GT>(acc));
    else
#pragma unroll
        for (int q = 0; q < 4; ++q) store_one<GT>(grad, v * dim + col[0] + q, acc[q]);
}

// Up to 64 tokens: each wave has all of them, one a lane, and needs neither the sort nor its launch.  A wave takes a token, and sums its row if it is the row's
// first; the others write zeros as above.  With the sort: 64 tokens of 3200, 2828 rows 16 us, so 9.6; 64 of 64, 100000 rows 13 and 8.7; 60 of 4096,
// 32000 rows 52 and 46.
constexpr int FEW_TOKENS = 64;
template <int DT, int GT, int C>
__global__ __launch_bounds__(THREADS) void k_few_tokens(const void *dout, int64_t ld, const void *tokens, bool wide, int n, int64_t first, int64_t rows, int64_t dim,
                                                        unsigned token_blocks, float scale, void *grad) {
    constexpr int E = Elem<GT>::E, SPAN = 64 * C * E;
    const int lane = lane_of();
    int mine = -1;                                  // the row of the lane's token
    if (lane < n) mine = (int)(wide ? row_of(static_cast<const int64_t *>(tokens), lane, first, rows) : row_of(static_cast<const int32_t *>(tokens), lane, first, rows));
    if (blockIdx.x < token_blocks) {
        const int i = blockIdx.x * WAVES + wave_of();
        if (i >= n) return;
        const int v = __builtin_amdgcn_readlane(mine, i);
        const uint64_t same = __ballot(mine == v), before = ((uint64_t)1 << lane) - 1;
        if (v < 0 || __builtin_ctzll(same) != i) return;
        const int to = same >> lane & 1 ? __popcll(same & before) : __popcll(same) + __popcll(~same & before);
        int64_t col[C];
        columns<E>(col, dim);
        float acc[C][E] = {};
        add_listed<DT, GT>(acc, dout, ld, __builtin_amdgcn_ds_permute(to * 4, lane), __popcll(same), col, dim);
        store_row<GT>(acc, grad, v, col, dim, scale);
        return;
    }
    const unsigned blocks = gridDim.x - token_blocks;
    const int64_t lead = (reinterpret_cast<uintptr_t>(grad) & 127) / Elem<GT>::BYTES, all = rows * dim;
    for (int64_t s = ((int64_t)blockIdx.y * blocks + (blockIdx.x - token_blocks)) * WAVES + wave_of(); s * SPAN - lead < all; s += (int64_t)blocks * gridDim.y * WAVES) {
        const int64_t from = s * SPAN - lead, row0 = (from > 0 ? from : 0) / dim;
        const int64_t past = row0 + (unsigned)(from + SPAN - row0 * dim) / (unsigned)dim;       // no element of the span is of a later row
        uint64_t inside = __ballot(mine >= row0 && mine <= past);
        if (!inside && from >= 0 && from + SPAN <= all) {
            store_zeros<GT, C>(grad, from);
            continue;
        }
        SpanPieces<C> at;
        at.place(from, 64 * E, E, row0, dim);
#pragma unroll
        for (int c = 0; c < C; ++c) at.empty[c] = 3;
        for (; inside; inside &= inside - 1) {
            const int v = __builtin_amdgcn_readlane(mine, __builtin_ctzll(inside));
#pragma unroll
            for (int c = 0; c < C; ++c) at.empty[c] &= ~((v == at.row[c] ? 1 : 0) | (v == at.row[c] + 1 ? 2 : 0));
        }
        at.template store<GT>(grad, all);
    }
}

// Rows narrower than a piece: a thread for each element.
template <int DT, int GT>
__global__ __launch_bounds__(THREADS) void k_narrow_sums(const void *dout, int64_t ld, const int *start, const int *order, int64_t rows,
                                                         int64_t dim, float scale, void *grad) {
    for (int64_t e = (int64_t)blockIdx.x * THREADS + threadIdx.x; e < rows * dim; e += (int64_t)gridDim.x * THREADS) {
        const int64_t v = e / dim, c = e - v * dim;
        float sum = 0.0f;
#pragma unroll 4
        for (int k = start[v]; k < start[v + 1]; ++k) sum += load_one<DT>(dout, order[k] * ld + c);
        store_one<GT>(grad, e, sum * scale);
    }
}

// ---------------------------------------------------------------- host
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// A wave for each row and tile.
dim3 grid_for(int64_t rows, int64_t tiles) {
    return dim3((unsigned)std::max<int64_t>(1, std::min(MAX_BLOCKS / tiles, ceil_div(rows, WAVES))), (unsigned)tiles);
}

// Tokens of a segment: short, so that many waves share a long run; and no more than MAX_SEGMENTS, which one wave adds up where all
// tokens are of one row.
constexpr int64_t MAX_SEGMENTS = 2048;
int segment_of(int64_t n) {
    int seg = 32;
    while (n / seg > MAX_SEGMENTS) seg *= 2;
    return seg;
}

// Tokens of a slice of the sort: all of them, or SLICE, or fewer where the table has so few rows that a block for each slice of SLICE would
// leave most of the chip idle (20000 tokens, 5000 rows in slices of 8192 56 us, of 2048 49; but 32768 tokens, 32000 rows 134 and 142).
int64_t slice_of(int64_t n, int64_t rows) {
    if (n <= SLICE) return SLICE;
    const int64_t to_fill = COMPUTE_UNITS / ceil_div(rows, SORT_ROWS);
    const int64_t slices = std::min<int64_t>(MAX_SLICES, std::max(ceil_div(n, SLICE), to_fill));
    return std::max<int64_t>(SLICE / 4, ceil_div(ceil_div(n, slices), SORT_THREADS) * SORT_THREADS);
}

struct GradRoom {                        // parts of the workspace, in bytes
    int64_t start, order, row_at, of_row, below, partial, all;
};
GradRoom grad_room(int64_t n, int64_t rows, int64_t dim) {
    const auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
    const int64_t slices = n > SLICE ? ceil_div(n, slice_of(n, rows)) : 0;
    GradRoom g;
    g.start = 0;
    g.order = up((rows + 1) * 4);
    g.row_at = g.order + up(n * 4);
    g.of_row = g.row_at + up(n * 4);
    g.below = g.of_row + up(slices * rows * 4);
    g.partial = g.below + up(slices * ceil_div(rows, SORT_ROWS) * 4);
    g.all = g.partial + (n > segment_of(n) ? up(2 * ceil_div(n, segment_of(n)) * dim * 4) : 0);
    return g;
}

int check_embed(const std::string &f, int64_t n, int64_t rows, int64_t dim) {
    if (n < 0 || n > INT32_MAX) return fail(PARO_EINVAL, f + "n must be in [0, 2^31)");
    if (rows < 1 || rows > (1 << 30)) return fail(PARO_EINVAL, f + "rows must be in [1, 2^30]");
    if (dim < 1 || dim > (1 << 24)) return fail(PARO_EINVAL, f + "dim must be in [1, 2^24]");
    return PARO_OK;
}
int check_tokens(const std::string &f, const void *tokens, int token_dtype, int64_t n) {
    if (token_dtype != PARO_I32 && token_dtype != PARO_I64) return fail(PARO_EINVAL, f + "token_dtype must be PARO_I32 or PARO_I64");
    return n ? check_array(tokens, token_dtype == PARO_I64 ? 8 : 4, f + "tokens") : PARO_OK;
}

template <int DT, class Token>
void launch_embed(const void *table, const void *tokens, int64_t n, int64_t first, int64_t rows, int64_t dim, float scale, void *out,
                  int64_t ld, hipStream_t st) {
    hipLaunchKernelGGL((k_embed<DT, Token>), grid_for(n, ceil_div(dim, 64 * PIECES * Elem<DT>::E)), dim3(THREADS), 0, st, table,
                       static_cast<const Token *>(tokens), n, first, rows, dim, scale, out, ld);
}

// Blocks that write the zeros, of `tiles` rows of blocks.
template <int GT>
unsigned zero_blocks(int64_t rows, int64_t dim, int64_t tiles) {
    const int64_t spans = rows * dim / (64 * GRAD_PIECES * Elem<GT>::E) + 2;
    return (unsigned)std::max<int64_t>(1, std::min(MAX_BLOCKS / 2 / tiles, ceil_div(spans, tiles * WAVES)));
}

template <int DT, int GT>
void launch_few(const void *dout, int64_t ld, const void *tokens, int token_dtype, int64_t n, int64_t first, float scale, void *grad, int64_t rows,
                int64_t dim, hipStream_t st) {
    const int64_t tiles = ceil_div(dim, 64 * GRAD_PIECES * Elem<GT>::E);
    const unsigned token_blocks = (unsigned)ceil_div(n, WAVES);
    hipLaunchKernelGGL((k_few_tokens<DT, GT, GRAD_PIECES>), dim3(token_blocks + zero_blocks<GT>(rows, dim, tiles), (unsigned)tiles), dim3(THREADS), 0, st, dout, ld,
                       tokens, token_dtype == PARO_I64, (int)n, first, rows, dim, token_blocks, scale, grad);
}

// Whether the tokens' waves, of GRAD_PIECES a lane, would be too few to keep the memory busy: up to six a SIMD.  Then one piece a lane and more waves
// (four | one: 2000 tokens of 2048, 2000 rows 29 us | 20, 803 of 6519 33 | 26, 5157 of 896 in fp32 31 | 27; but 8191 of 768 to fp32 45 | 47, 20000 of
// 2048 49 | 59).
template <int GT>
bool few_waves(int64_t n, int64_t dim) {
    return n * ceil_div(dim, 64 * GRAD_PIECES * Elem<GT>::E) <= 6 * 4 * COMPUTE_UNITS;
}

template <int DT, int GT, int C>
void launch_sums(const void *dout, int64_t ld, int64_t n, float scale, void *grad, int64_t rows, int64_t dim, char *ws, const GradRoom &g,
                 hipStream_t st) {
    const int *start = reinterpret_cast<int *>(ws + g.start), *order = reinterpret_cast<int *>(ws + g.order);
    if (dim < Elem<DT>::E) {
        hipLaunchKernelGGL((k_narrow_sums<DT, GT>), dim3((unsigned)std::min(MAX_BLOCKS, ceil_div(rows * dim, THREADS))), dim3(THREADS), 0, st, dout,
                           ld, start, order, rows, dim, scale, grad);
        return;
    }
    const int seg = segment_of(n), *row_at = reinterpret_cast<int *>(ws + g.row_at);
    float *partial = reinterpret_cast<float *>(ws + g.partial);
    const unsigned seg_blocks = n > seg ? (unsigned)ceil_div(ceil_div(n, seg), WAVES) : 0;
    const int64_t tiles = ceil_div(dim, 64 * C * Elem<GT>::E);
    const unsigned run_blocks = n ? grid_for(n, 2 * tiles).x : 0;
    hipLaunchKernelGGL((k_sums<DT, GT, C>), dim3(seg_blocks + run_blocks + zero_blocks<GT>(rows, dim, tiles), (unsigned)tiles), dim3(THREADS), 0, st, dout,
                       ld, start, order, row_at, rows, dim, seg, seg_blocks, run_blocks, scale, partial, grad);
    if (seg_blocks)
        hipLaunchKernelGGL((k_join<GT>), dim3(seg_blocks, (unsigned)ceil_div(dim, 64 * 4)), dim3(THREADS), 0, st, start, row_at, rows, dim, seg,
                           scale, partial, grad);
}

}  // namespace

extern "C" {

int paro_embed(const void *table, int dtype, int64_t rows, int64_t dim, const void *tokens, int token_dtype, int64_t n, int64_t first_token,
               float scale, void *out, int64_t ld_out, void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_embed: ";
        int rc;
        if (!is_dtype(dtype)) return fail(PARO_EINVAL, f + "bad dtype");
        if ((rc = check_embed(f, n, rows, dim))) return rc;
        if (ld_out == 0) ld_out = dim;
        if (ld_out < dim) return fail(PARO_EINVAL, f + "ld_out is smaller than dim");
        if (too_large(rows, dim, size_of(dtype)) || too_large(n, ld_out, size_of(dtype))) return fail(PARO_EINVAL, f + "too large");
        if ((rc = check_tokens(f, tokens, token_dtype, n))) return rc;
        if (n == 0) return PARO_OK;
        if ((rc = check_array(table, size_of(dtype), f + "table"))) return rc;
        if ((rc = check_array(out, size_of(dtype), f + "out"))) return rc;
        hipStream_t st = static_cast<hipStream_t>(stream);
#define PARO_EMBED(DT, TOKEN) launch_embed<DT, TOKEN>(table, tokens, n, first_token, rows, dim, scale, out, ld_out, st)
#define PARO_EMBED_OF(DT) (token_dtype == PARO_I64 ? PARO_EMBED(DT, int64_t) : PARO_EMBED(DT, int32_t))
        if (dtype == PARO_F32) PARO_EMBED_OF(PARO_F32);
        else if (dtype == PARO_F16) PARO_EMBED_OF(PARO_F16);
        else PARO_EMBED_OF(PARO_BF16);
#undef PARO_EMBED_OF
#undef PARO_EMBED
        PARO_LAUNCHED("paro_embed");
        return PARO_OK;
    });
}

int64_t paro_embed_grad_workspace(int64_t n, int64_t rows, int64_t dim) {
    int64_t bytes = 0;
    const int rc = guarded([&]() -> int {
        const int bad = check_embed("paro_embed_grad_workspace: ", n, rows, dim);
        if (!bad) bytes = grad_room(n, rows, dim).all;
        return bad;
    });
    return rc ? rc : bytes;
}

int paro_embed_grad(const void *dout, int dtype, int64_t ld_dout, const void *tokens, int token_dtype, int64_t n, int64_t first_token,
                    float scale, void *grad, int grad_dtype, int64_t rows, int64_t dim, void *workspace, int64_t workspace_bytes,
                    void *stream) {
    return guarded([&]() -> int {
        const std::string f = "paro_embed_grad: ";
        int rc;
        if (!is_dtype(dtype) || (grad_dtype != dtype && grad_dtype != PARO_F32))
            return fail(PARO_EINVAL, f + "bad dtype (the gradient's is dout's or PARO_F32)");
        if ((rc = check_embed(f, n, rows, dim))) return rc;
        if (ld_dout == 0) ld_dout = dim;
        if (ld_dout < dim) return fail(PARO_EINVAL, f + "ld_dout is smaller than dim");
        if (too_large(rows, dim, 4) || too_large(n, ld_dout, size_of(dtype))) return fail(PARO_EINVAL, f + "too large");
        if ((rc = check_tokens(f, tokens, token_dtype, n))) return rc;
        if (n && (rc = check_array(dout, size_of(dtype), f + "dout"))) return rc;
        if ((rc = check_array(grad, size_of(grad_dtype), f + "grad"))) return rc;
        if ((rc = check_array(workspace, 16, f + "workspace"))) return rc;
        const GradRoom g = grad_room(n, rows, dim);
        if (workspace_bytes < g.all) return fail(PARO_ERANGE, f + "the workspace is smaller than paro_embed_grad_workspace says");
        hipStream_t st = static_cast<hipStream_t>(stream);
        if (n <= FEW_TOKENS && dim * size_of(dtype) >= 16) {
#define PARO_FEW(DT, GT) launch_few<DT, GT>(dout, ld_dout, tokens, token_dtype, n, first_token, scale, grad, rows, dim, st)
            if (dtype == PARO_F32) PARO_FEW(PARO_F32, PARO_F32);
            else if (dtype == PARO_F16 && grad_dtype == PARO_F16) PARO_FEW(PARO_F16, PARO_F16);
            else if (dtype == PARO_F16) PARO_FEW(PARO_F16, PARO_F32);
            else if (grad_dtype == PARO_BF16) PARO_FEW(PARO_BF16, PARO_BF16);
            else PARO_FEW(PARO_BF16, PARO_F32);
#undef PARO_FEW
            PARO_LAUNCHED("paro_embed_grad");
            return PARO_OK;
        }
        char *ws = static_cast<char *>(workspace);
        int *start = reinterpret_cast<int *>(ws + g.start), *order = reinterpret_cast<int *>(ws + g.order);
        int *row_at = reinterpret_cast<int *>(ws + g.row_at);
        const int64_t slice = slice_of(n, rows);
        const dim3 sort_grid((unsigned)ceil_div(rows, SORT_ROWS), (unsigned)std::max<int64_t>(1, ceil_div(n, slice)));
        const SliceCounts counts{reinterpret_cast<int *>(ws + g.of_row), reinterpret_cast<int *>(ws + g.below)};
#define PARO_SORT(TOKEN, COUNT)                                                                                                        \
    hipLaunchKernelGGL((k_sort_tokens<TOKEN, COUNT>), sort_grid, dim3(SORT_THREADS), 0, st, static_cast<const TOKEN *>(tokens), n, first_token, \
                       rows, slice, counts, start, order, row_at)
        if (token_dtype == PARO_I64) {
            if (sort_grid.y > 1) PARO_SORT(int64_t, true);
            PARO_SORT(int64_t, false);
        } else {
            if (sort_grid.y > 1) PARO_SORT(int32_t, true);
            PARO_SORT(int32_t, false);
        }
#undef PARO_SORT
        PARO_LAUNCHED("paro_embed_grad");
#define PARO_SUMS(DT, GT)                                                                                                              \
    (dim <= 64 * Elem<GT>::E || few_waves<GT>(n, dim) ? launch_sums<DT, GT, 1>                                                         \
     : dim <= 128 * Elem<GT>::E                       ? launch_sums<DT, GT, 2>                                                         \
                                                      : launch_sums<DT, GT, GRAD_PIECES>)(dout, ld_dout, n, scale, grad, rows, dim, ws, g, st)
        if (dtype == PARO_F32) PARO_SUMS(PARO_F32, PARO_F32);
        else if (dtype == PARO_F16 && grad_dtype == PARO_F16) PARO_SUMS(PARO_F16, PARO_F16);
        else if (dtype == PARO_F16) PARO_SUMS(PARO_F16, PARO_F32);
        else if (grad_dtype == PARO_BF16) PARO_SUMS(PARO_BF16, PARO_BF16);
        else PARO_SUMS(PARO_BF16, PARO_F32);
#undef PARO_SUMS
        PARO_LAUNCHED("paro_embed_grad");
        return PARO_OK;
    });
}

}  // extern "C"
