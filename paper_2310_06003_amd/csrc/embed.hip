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
// A block takes SORT_ROWS rows of the table and reads all tokens: its sixteen waves take consecutive parts of them, count
// theirs for each row in counters of their own, and - after a scan over rows and waves - write them to their places in a second
// walk.  Tokens of one row keep their order, nothing is atomic, no block waits for another: one launch.
constexpr int SORT_BITS = 9, SORT_ROWS = 1 << SORT_BITS, SORT_WAVES = 16, SORT_THREADS = 64 * SORT_WAVES;

// Lanes with the same value as this one, among `in`.
__device__ __forceinline__ uint64_t same_row(int row, uint64_t in) {
#pragma unroll
    for (int b = 0; b < SORT_BITS; ++b) {
        const uint64_t set = __ballot((row >> b) & 1);
        in &= (row >> b) & 1 ? set : ~set;
    }
    return in;
}

template <class Token>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_tokens(const Token *tokens, int64_t n, int64_t first, int64_t rows, int *start,
                                                              int *order, int *row_at) {
    __shared__ int count[SORT_WAVES][SORT_ROWS];
    __shared__ int scan[SORT_ROWS];
    __shared__ int below_of[SORT_WAVES];
    const int w = wave_of(), lane = lane_of();
    const int64_t lo = (int64_t)blockIdx.x * SORT_ROWS, hi = lo + SORT_ROWS < rows ? lo + SORT_ROWS : rows;
    const int64_t part = (n + SORT_THREADS - 1) / SORT_THREADS * 64;
    const int64_t begin = w * part, end = begin + part < n ? begin + part : n;
    for (int r = threadIdx.x; r < SORT_WAVES * SORT_ROWS; r += SORT_THREADS) (&count[0][0])[r] = 0;
    __syncthreads();

    const uint64_t before = ((uint64_t)1 << lane) - 1;
    int below = 0;
    const auto walk = [&](auto &&visit) {
        for (int64_t i0 = begin; i0 < end; i0 += 256) {          // four loads in flight
            int64_t r[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int64_t i = i0 + u * 64 + lane;
                r[u] = i < end ? row_of(tokens, i, first, rows) : -1;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) visit(i0 + u * 64 + lane, r[u]);
        }
    };
    walk([&](int64_t, int64_t r) {
        below += __popcll(__ballot(r >= 0 && r < lo));
        const uint64_t in = __ballot(r >= lo && r < hi);
        if (!in) return;
        const int row = (int)(r - lo) & (SORT_ROWS - 1);
        const uint64_t same = same_row(row, in);
        if (r >= lo && r < hi && !(same & before)) count[w][row] += __popcll(same);
    });
    if (lane == 0) below_of[w] = below;
    __syncthreads();

    int base = 0;
    for (int k = 0; k < SORT_WAVES; ++k) base += below_of[k];
    int total = 0;
    const int mine = threadIdx.x;
    if (mine < SORT_ROWS) {
        for (int k = 0; k < SORT_WAVES; ++k) total += count[k][mine];
        scan[mine] = total;
    }
    __syncthreads();
    for (int step = 1; step < SORT_ROWS; step *= 2) {
        const int other = mine < SORT_ROWS && mine >= step ? scan[mine - step] : 0;
        __syncthreads();
        if (mine < SORT_ROWS) scan[mine] += other;
        __syncthreads();
    }
    if (mine < SORT_ROWS) {
        int at = base + scan[mine] - total;
        if (lo + mine < hi) start[lo + mine] = at;
        if (lo + mine == rows - 1) start[rows] = at + total;
        for (int k = 0; k < SORT_WAVES; ++k) {
            const int c = count[k][mine];
            count[k][mine] = at;
            at += c;
        }
    }
    __syncthreads();

    walk([&](int64_t i, int64_t r) {
        const uint64_t in = __ballot(r >= lo && r < hi);
        if (!in) return;
        const int row = (int)(r - lo) & (SORT_ROWS - 1);
        const uint64_t same = same_row(row, in);
        if (r >= lo && r < hi) {
            const int at = count[w][row], rank = __popcll(same & before);
            order[at + rank] = (int)i;
            row_at[at + rank] = (int)r;
            if (rank == 0) count[w][row] = at + __popcll(same);
        }
    });
}

// ---------------------------------------------------------------- sums over the sorted tokens
// acc += dout[order[a .. b)], in order, for the lane's pieces of a tile of columns.
template <int DT, int C>
__device__ __forceinline__ void add_rows(float (&acc)[C][Elem<DT>::E], const void *dout, int64_t ld, const int *order, int a, int b,
                                         const int64_t (&col)[C], int64_t dim) {
    constexpr int E = Elem<DT>::E, U = 4;
    for (int k = a; k < b; k += U) {
        u32x4 raw[U][C];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = (int64_t)order[k + u < b ? k + u : b - 1] * ld;
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (k + u < b && col[c] < dim) raw[u][c] = load_piece<DT>(dout, row + col[c]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (k + u < b && col[c] < dim) {
                    float x[E];
                    unpack<DT>(raw[u][c], x);
#pragma unroll
                    for (int j = 0; j < E; ++j) acc[c][j] += x[j];
                }
    }
}

// Columns of a lane's pieces; the last piece of a row starts early, past the row: dim.
template <int E, int C>
__device__ __forceinline__ void columns(int64_t (&col)[C], int64_t tile, int64_t dim) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t e = tile * (64 * C * E) + c * 64 * E + lane_of() * E;
        col[c] = e >= dim ? dim : e < dim - E ? e : dim - E;
    }
}

// Runs of more than `seg` tokens are summed segment by segment of the sorted order, in parallel.  Of one segment such a run
// holds the beginning (slot 0), or the end and not the beginning (slot 1).
template <int DT, int C>
__global__ __launch_bounds__(THREADS) void k_segment_sums(const void *dout, int64_t ld, const int *start, const int *order, const int *row_at,
                                                          int64_t rows, int64_t dim, int seg, float *partial) {
    constexpr int E = Elem<DT>::E;
    const int64_t s = (int64_t)blockIdx.x * WAVES + wave_of();
    const int held = start[rows], a = (int)(s * seg), b = a + seg < held ? a + seg : held;
    if (a >= b) return;
    int64_t col[C];
    columns<E>(col, blockIdx.y, dim);
    const int rows_of[2] = {row_at[a], row_at[b - 1]};
    for (int slot = 0; slot < 2; ++slot) {
        if (slot == 1 && rows_of[1] == rows_of[0]) break;
        const int from = start[rows_of[slot]], to = start[rows_of[slot] + 1];
        if (to - from <= seg) continue;
        float acc[C][E] = {};
        add_rows<DT>(acc, dout, ld, order, from > a ? from : a, to < b ? to : b, col, dim);
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (col[c] < dim)
#pragma unroll
                for (int j = 0; j < E; j += 4)
                    store_piece<PARO_F32>(partial, (2 * s + slot) * dim + col[c] + j, pack<PARO_F32>(&acc[c][j]));
    }
}

// A wave writes a tile of a row of the table's gradient: of a short run its tokens' sum, of a long one its segments', and
// zeros where no token is.
template <int DT, int GT, int C>
__global__ __launch_bounds__(THREADS) void k_row_sums(const void *dout, int64_t ld, const int *start, const int *order, int64_t rows,
                                                      int64_t dim, int seg, const float *partial, float scale, void *grad) {
    constexpr int E = Elem<DT>::E, G = Elem<GT>::E;
    static_assert(G <= E, "the gradient is at least as wide as what is summed");
    for (int64_t v = (int64_t)blockIdx.x * WAVES + wave_of(); v < rows; v += (int64_t)gridDim.x * WAVES) {
        const int a = start[v], b = start[v + 1];
        int64_t col[C];
        columns<E>(col, blockIdx.y, dim);
        float acc[C][E] = {};
        if (b - a <= seg) {
            add_rows<DT>(acc, dout, ld, order, a, b, col, dim);
        } else {
            for (int64_t s = a / seg; s * seg < b; ++s) {
                const int slot = s * seg < a ? 1 : 0;
#pragma unroll
                for (int c = 0; c < C; ++c)
                    if (col[c] < dim)
#pragma unroll
                        for (int j = 0; j < E; j += 4) {
                            float x[4];
                            unpack<PARO_F32>(load_piece<PARO_F32>(partial, (2 * s + slot) * dim + col[c] + j), x);
#pragma unroll
                            for (int q = 0; q < 4; ++q) acc[c][j + q] += x[q];
                        }
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (col[c] >= dim) continue;
#pragma unroll
            for (int j = 0; j < E; ++j) acc[c][j] *= scale;
#pragma unroll
            for (int j = 0; j < E; j += G) store_piece<GT>(grad, v * dim + col[c] + j, pack<GT>(&acc[c][j]));
        }
    }
}

// Rows narrower than a piece: a thread for each element.
template <int DT, int GT>
__global__ __launch_bounds__(THREADS) void k_narrow_sums(const void *dout, int64_t ld, const int *start, const int *order, int64_t rows,
                                                         int64_t dim, float scale, void *grad) {
    for (int64_t e = (int64_t)blockIdx.x * THREADS + threadIdx.x; e < rows * dim; e += (int64_t)gridDim.x * THREADS) {
        const int64_t v = e / dim, c = e - v * dim;
        float sum = 0.0f;
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

// Tokens of a segment: what a long run's parts and their number cost in a row are alike near the square root.
int segment_of(int64_t n) {
    int seg = 64;
    while ((int64_t)seg * seg < n) seg *= 2;
    return seg;
}
constexpr int GRAD_PIECES = 2;           // pieces a lane of the gradient's kernels

struct GradRoom {                        // parts of the workspace, in bytes
    int64_t start, order, row_at, partial, all;
};
GradRoom grad_room(int64_t n, int64_t rows, int64_t dim) {
    const auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
    GradRoom g;
    g.start = 0;
    g.order = up((rows + 1) * 4);
    g.row_at = g.order + up(n * 4);
    g.partial = g.row_at + up(n * 4);
    g.all = g.partial + up(2 * ceil_div(n, segment_of(n)) * dim * 4);
    return g;
}

int check_embed(const std::string &f, int64_t n, int64_t rows, int64_t dim) {
    if (n < 0 || n > INT32_MAX) return fail(PARO_EINVAL, f + "n must be in [0, 2^31)");
    if (rows < 1 || rows >= INT32_MAX) return fail(PARO_EINVAL, f + "rows must be in [1, 2^31 - 1)");
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

template <int DT, int GT>
void launch_sums(const void *dout, int64_t ld, int64_t n, float scale, void *grad, int64_t rows, int64_t dim, char *ws, const GradRoom &g,
                 hipStream_t st) {
    const int *start = reinterpret_cast<int *>(ws + g.start), *order = reinterpret_cast<int *>(ws + g.order);
    if (dim < Elem<DT>::E) {
        hipLaunchKernelGGL((k_narrow_sums<DT, GT>), dim3((unsigned)std::min(MAX_BLOCKS, ceil_div(rows * dim, THREADS))), dim3(THREADS), 0, st, dout,
                           ld, start, order, rows, dim, scale, grad);
        return;
    }
    const int seg = segment_of(n);
    const int64_t tiles = ceil_div(dim, 64 * GRAD_PIECES * Elem<DT>::E);
    float *partial = reinterpret_cast<float *>(ws + g.partial);
    if (n > seg)
        hipLaunchKernelGGL((k_segment_sums<DT, GRAD_PIECES>), dim3((unsigned)ceil_div(ceil_div(n, seg), WAVES), (unsigned)tiles), dim3(THREADS), 0,
                           st, dout, ld, start, order, reinterpret_cast<int *>(ws + g.row_at), rows, dim, seg, partial);
    hipLaunchKernelGGL((k_row_sums<DT, GT, GRAD_PIECES>), grid_for(rows, tiles), dim3(THREADS), 0, st, dout, ld, start, order, rows, dim, seg,
                       partial, scale, grad);
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
        char *ws = static_cast<char *>(workspace);
        int *start = reinterpret_cast<int *>(ws + g.start), *order = reinterpret_cast<int *>(ws + g.order);
        int *row_at = reinterpret_cast<int *>(ws + g.row_at);
        const dim3 sort_grid((unsigned)ceil_div(rows, SORT_ROWS));
        if (token_dtype == PARO_I64)
            hipLaunchKernelGGL((k_sort_tokens<int64_t>), sort_grid, dim3(SORT_THREADS), 0, st, static_cast<const int64_t *>(tokens), n, first_token,
                               rows, start, order, row_at);
        else
            hipLaunchKernelGGL((k_sort_tokens<int32_t>), sort_grid, dim3(SORT_THREADS), 0, st, static_cast<const int32_t *>(tokens), n, first_token,
                               rows, start, order, row_at);
        PARO_LAUNCHED("paro_embed_grad");
#define PARO_SUMS(DT, GT) launch_sums<DT, GT>(dout, ld_dout, n, scale, grad, rows, dim, ws, g, st)
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
