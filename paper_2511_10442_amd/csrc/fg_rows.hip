// Rows by index: lookup, copies into an order by expert, weighted sums of rows, and the gradients of rows that are named once and of weights.
// Sums are held in 32 bits and rounded once.
#include "fg_pieces.hpp"

namespace fg {

namespace {

// ---- lookup ------------------------------------------------------------------------------------------------------------

// out[i] = scale * table[index[i]].  Bound by memory: 64k rows of 4 KiB, 349 MB that have to move, 60 us (5.8 TB/s); 64 rows of 8 KiB 2.6 us,
// a launch and two trips to memory.

template <typename T, int N, bool STREAM, int SEGS>
__global__ __launch_bounds__(kBlock) void k_lookup(const T* __restrict__ table, int64_t table_stride, uint32_t n_rows, const int32_t* __restrict__ index,
                                                   float scale, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T, N> P;
    constexpr int S = SEGS ? SEGS : 1;
    each_span<N, SEGS>(d, [&](const Span<S>& at) {
        const int32_t name = index[at.row];
        typename P::Vec v[S] = {};
        if ((uint32_t)name < n_rows) {
#pragma unroll
            for (int s = 0; s < S; ++s) v[s] = load_piece<T, N>(table + (int64_t)name * table_stride + at.col[s]);
#pragma unroll
            for (int s = 0; s < S; ++s) v[s] = narrow<T, N>(wide<T, N>(v[s]) * scale);
        }
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (at.there[s]) store_piece<T, N, STREAM>(out + at.row * out_stride + at.col[s], v[s]);
    });
}

// ---- a token's row to its places ---------------------------------------------------------------------------------------

// out[place[i][j]] = x[i], read once and written k times (the other way round, a copy from token to place for every place, reads every row k times:
// 32k rows of 4 KiB to 8 places each 305 us).  226 us, 1.2 GB at 5.3 TB/s.

template <typename T, int N, int SEGS>
__global__ __launch_bounds__(kBlock) void k_dispatch(const T* __restrict__ x, int64_t x_stride, const int32_t* __restrict__ place, int32_t k,
                                                     uint32_t n_rows, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T, N> P;
    constexpr int S = SEGS ? SEGS : 1;
    each_span<N, SEGS>(d, [&](const Span<S>& at) {
        typename P::Vec v[S];
#pragma unroll
        for (int s = 0; s < S; ++s) v[s] = load_piece<T, N>(x + at.row * x_stride + at.col[s]);
        const int32_t* p = place + at.row * k;
        for (int32_t j = 0; j < k; ++j) {
            const int32_t to = p[j];
            if ((uint32_t)to < n_rows)
#pragma unroll
                for (int s = 0; s < S; ++s)
                    if (at.there[s]) store_piece<T, N>(out + (int64_t)to * out_stride + at.col[s], v[s]);
        }
    });
}

// ---- weighted sums -----------------------------------------------------------------------------------------------------

// out[i] = sum over j of weights[i][j] rows[index[i][j]], eight rows' pieces under way at a time.  Where every row is named once, 32k sums of 8 rows of
// 4 KiB take 207 us (1.2 GB at 5.8 TB/s); messages along a graph, 200k points of 64 float32 with 40 neighbours each in no order, 282 us: 2 GB of
// rows leave the last-level cache at 7.3 TB/s.  `walk` is the order in which the sums are made: points of a neighbourhood one after the other, on one XCD
// (shared), find each other's neighbours in its L2.  200k uniform points in three dimensions, 40 nearest neighbours: 291 us in no order, 97 in that of
// their bins (100k: 137 and 53; 1M, 32 neighbours: 1234 and 530).
// (n_rows > 0: an entry that names no row reads row 0 and adds zeros in its place, so that no load waits behind a branch)
template <typename T, int N, bool WEIGHTED, bool STREAM, int SEGS>
__global__ __launch_bounds__(kBlock) void k_combine(const T* __restrict__ rows, int64_t rows_stride, uint32_t n_rows, const int32_t* __restrict__ index,
                                                    const float* __restrict__ weights, int32_t k, const int32_t* __restrict__ walk, int64_t t, T* __restrict__ out,
                                                    int64_t out_stride, Deal d, bool shared)
{
    typedef Piece<T, N> P;
    constexpr int S = SEGS ? SEGS : 1;
    const int64_t block = shared ? by_xcd(blockIdx.x, gridDim.x) : blockIdx.x;
    each_span<N, SEGS>(d, block, gridDim.x, [&](const Span<S>& at) {
        int64_t row = at.row;
        if (walk) {
            row = (uint32_t)walk[row];
            if (row >= t) return;
        }
        typename P::Wide sum[S] = {};
        const int64_t base = row * k;
        in_chunks<8>(k, [&](auto count, int32_t j, int there) {
            constexpr int U = count.value;
            int32_t name[U];
            float w[U];
            typename P::Vec v[U][S];
            load_words<U>(index + base + j, there, name);
            if (WEIGHTED) load_words<U>(weights + base + j, there, w);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool named = u < there && (uint32_t)name[u] < n_rows;
#pragma unroll
                for (int s = 0; s < S; ++s) v[u][s] = load_piece<T, N, STREAM>(rows + (named ? (int64_t)name[u] : 0) * rows_stride + at.col[s]);
                if (WEIGHTED) w[u] = named ? w[u] : 0.0f;
                name[u] = named;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const typename P::Wide x = wide<T, N>(only_if<T, N>(name[u], v[u][s]));
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[s][i] = WEIGHTED ? __builtin_fmaf(x[i], w[u], sum[s][i]) : sum[s][i] + x[i];
                }
        });
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (at.there[s]) store_piece<T, N, STREAM>(out + row * out_stride + at.col[s], narrow<T, N>(sum[s]));
    });
}

// ---- gradients of weights, and of rows that are named once -------------------------------------------------------------

// `lanes` lanes (8 to 32: WAVES == 0; 64, 128 or 256: WAVES wavefronts, which meet in LDS) take a token: they walk along its row and those of up
// to eight of its k, so that the token's gradient is loaded once for the eight.  ROWS: grad_rows[index[i][j]] = weights[i][j] grad_out[i] is written on
// the way.  32k tokens of 8 rows of 4 KiB: 437 us, 2.3 GB at 5.2 TB/s; 4k tokens of 3 rows of 2000 bytes: 12 us.
template <typename T, int N, bool ROWS, bool WEIGHTED, bool STREAM, int WAVES>
__global__ __launch_bounds__(kBlock, ROWS ? 3 : 4) void k_combine_grad(const T* __restrict__ grad_out, int64_t grad_stride, int64_t t, int32_t c,
                                                         const T* __restrict__ rows, int64_t rows_stride, uint32_t n_rows,
                                                         const int32_t* __restrict__ index, const float* __restrict__ weights, int32_t k,
                                                         T* __restrict__ grad_rows, int64_t grad_rows_stride, float* __restrict__ grad_weights,
                                                         int lanes)
{
    typedef Piece<T, N> P;
    __shared__ float part[kBlock / 64][8];
    const int lane = threadIdx.x & (lanes - 1);
    const int log = __builtin_ctz(lanes), each = kBlock >> log;
    const int64_t turns = (t + each - 1) / each;
    const bool dots = grad_weights && n_rows > 0;
    for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x) {
        const int group = WAVES ? __builtin_amdgcn_readfirstlane(threadIdx.x >> log) : threadIdx.x >> log;
        const int64_t row = turn * each + group;
        const bool there = row < t;
        const int64_t base = there ? row * k : 0;
        in_chunks<8>(k, [&](auto count, int32_t j, int here) {
            constexpr int U = count.value;
            int32_t name[U];
            float w[U], dot[U];
            load_words<U>(index + base + j, here, name);
            if (WEIGHTED) load_words<U>(weights + base + j, here, w);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= here || (uint32_t)name[u] >= n_rows) name[u] = -1;
                dot[u] = 0.0f;
            }
            for (int32_t turn_col = lane * N; there && turn_col < c; turn_col += lanes * N) {
                const int32_t col = turn_col > c - N ? c - N : turn_col, skip = turn_col - col;
                const typename P::Wide g = wide<T, N>(load_piece<T, N>(grad_out + row * grad_stride + col));
                if (dots) {
                    typename P::Vec v[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) v[u] = load_piece<T, N, STREAM>(rows + (name[u] < 0 ? 0 : (int64_t)name[u]) * rows_stride + col);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const typename P::Wide x = wide<T, N>(v[u]);
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (i >= skip) dot[u] = __builtin_fmaf(x[i], g[i], dot[u]);
                    }
                }
                if constexpr (ROWS)
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (name[u] >= 0) {
                            float by = WEIGHTED ? w[u] : 1.0f;
                            if (WEIGHTED) asm volatile("" : "+v"(by));       // the rows' products would otherwise be made ahead, in 64 registers
                            store_piece<T, N, STREAM>(grad_rows + (int64_t)name[u] * grad_rows_stride + col, narrow<T, N>(WEIGHTED ? g * by : g));
                        }
            }
            if (!grad_weights) return;
            // (products with row 0, of entries that name none, are dropped here, NaN and all)
#pragma unroll
            for (int u = 0; u < U; ++u) dot[u] = name[u] < 0 ? 0.0f : dot[u];
            const int some = WAVES ? 64 : lanes, at = threadIdx.x & (some - 1), u = share_of<U>(at, some);
            float sum = add_up<U>(dot, at, some);
            bool writes = (at & (some / U - 1)) == 0;
            if constexpr (WAVES > 1) {
                const int wave = threadIdx.x >> 6;
                if (writes) part[wave][u] = sum;
                __syncthreads();
                writes = writes && wave % WAVES == 0;
                if (writes)
#pragma unroll
                    for (int o = 1; o < WAVES; ++o) sum += part[wave + o][u];
                __syncthreads();
            }
            if (writes && there && u < here) grad_weights[base + j + u] = sum;
        });
    }
}

template <typename T, int N>
hipError_t lookup(RowsIn table, int64_t n_rows, int64_t c, const int32_t* index, int64_t m, float scale, RowsOut out, hipStream_t stream)
{
    const Deal d = deal<T, N>(m, c, 2);
#define FG_LOOKUP(STREAM) \
    FG_LAUNCH_DEAL(2, d, blocks_for(d, kMostBlocks), stream, FG_LOOKUP_OF(STREAM), (const T*)table.at, table.stride, (uint32_t)n_rows, index, scale, (T*)out.at, out.stride, d)
#define FG_LOOKUP_OF(STREAM) k_lookup<T, N, STREAM
    if (2 * m * c * (int64_t)sizeof(T) < kStream) FG_LOOKUP(false); else FG_LOOKUP(true);
#undef FG_LOOKUP_OF
#undef FG_LOOKUP
    return hipSuccess;
}

template <typename T, int N>
hipError_t dispatch(RowsIn x, int64_t t, int64_t c, const int32_t* place, int32_t k, int64_t n_rows, RowsOut out, hipStream_t stream)
{
    const Deal d = deal<T, N>(t, c, 4);
#define FG_DISPATCH k_dispatch<T, N
    FG_LAUNCH_DEAL(4, d, blocks_for(d, kMostBlocks), stream, FG_DISPATCH, (const T*)x.at, x.stride, place, k, (uint32_t)n_rows, (T*)out.at, out.stride, d);
#undef FG_DISPATCH
    return hipSuccess;
}

template <typename T, int N>
hipError_t combine(RowsIn rows, int64_t n_rows, int64_t c, const int32_t* index, const float* weights, int64_t t, int32_t k, const int32_t* walk,
                   RowsOut out, hipStream_t stream)
{
    if (n_rows == 0) return lookup<T, N>(rows, 0, c, index, t, 1.0f, out, stream);       // zeros
    const Deal d = deal<T, N>(t, c, 2);
    const bool shared = t * k >= kShared * n_rows;
    const unsigned grid = shared ? to_xcds(blocks_for(d, kMostUneven)) : blocks_for(d, kMostBlocks).x;
#define FG_COMBINE(WEIGHTED, STREAM)                                                                                                        \
    FG_LAUNCH_DEAL(2, d, grid, stream, FG_COMBINE_OF(WEIGHTED, STREAM), (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, \
                   walk, t, (T*)out.at, out.stride, d, shared)
#define FG_COMBINE_OF(WEIGHTED, STREAM) k_combine<T, N, WEIGHTED, STREAM
    const bool past = n_rows >= t * k && (t * k + t) * c * (int64_t)sizeof(T) >= kStream;      // (rows that are named again are worth keeping)
    if (weights) { if (past) FG_COMBINE(true, true); else FG_COMBINE(true, false); }
    else if (past) FG_COMBINE(false, true);
    else FG_COMBINE(false, false);
#undef FG_COMBINE_OF
#undef FG_COMBINE
    return hipSuccess;
}

template <typename T, int N, bool ROWS, bool WEIGHTED>
hipError_t combine_grad(RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index, const float* weights, int32_t k,
                        RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    const int64_t pieces = (c + N - 1) / N;
    // a wavefront or less for a token; more, so that a row is one trip to memory, while the chip has room for it (4k tokens, 2000 bytes a row: 20 us
    // with one, 13 with two)
    int lanes = (int)lanes_for(pieces < 64 ? pieces : 64);
    while (lanes < kBlock && lanes < pieces && lanes * t <= kFill) lanes *= 2;
    const dim3 grid = blocks_for(t, kBlock / lanes);
#define FG_COMBINE_GRAD(STREAM, WAVES)                                                                                                             \
    FG_LAUNCH((k_combine_grad<T, N, ROWS, WEIGHTED, STREAM, WAVES>), grid, dim3(kBlock), 0, stream, (const T*)grad_out.at, grad_out.stride, t,      \
              (int32_t)c, (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)grad_rows.at, grad_rows.stride, grad_weights, lanes)
    constexpr bool kOnce = ROWS && N > 1;                     // (ROWS: no row is named twice)
    if (lanes == 256) FG_COMBINE_GRAD(false, 4);
    else if (lanes == 128) FG_COMBINE_GRAD(false, 2);
    else if (lanes == 64 && kOnce && (2 * t * k + t) * c * (int64_t)sizeof(T) >= kStream) FG_COMBINE_GRAD(kOnce, 1);
    else if (lanes == 64) FG_COMBINE_GRAD(false, 1);
    else FG_COMBINE_GRAD(false, 0);
#undef FG_COMBINE_GRAD
    return hipSuccess;
}

template <typename T, int N>
hipError_t combine_grad_of(RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index, const float* weights, int32_t k,
                           RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    if (!grad_rows.at) return combine_grad<T, N, false, false>(grad_out, t, c, rows, n_rows, index, nullptr, k, grad_rows, grad_weights, stream);
    if (!weights) return combine_grad<T, N, true, false>(grad_out, t, c, rows, n_rows, index, weights, k, grad_rows, grad_weights, stream);
    return combine_grad<T, N, true, true>(grad_out, t, c, rows, n_rows, index, weights, k, grad_rows, grad_weights, stream);
}

}  // namespace

hipError_t launch_lookup(int32_t type, RowsIn table, int64_t n_rows, int64_t c, const int32_t* index, int64_t m, float scale, RowsOut out,
                         hipStream_t stream)
{
    FG_BY_TYPE(type, c, (lookup<T, N>(table, n_rows, c, index, m, scale, out, stream)))
}

hipError_t launch_dispatch(int32_t type, RowsIn x, int64_t t, int64_t c, const int32_t* place, int32_t k, int64_t n_rows, RowsOut out,
                           hipStream_t stream)
{
    FG_BY_TYPE(type, c, (dispatch<T, N>(x, t, c, place, k, n_rows, out, stream)))
}

hipError_t launch_combine(int32_t type, RowsIn rows, int64_t n_rows, int64_t c, const int32_t* index, const float* weights, int64_t t, int32_t k,
                          const int32_t* walk, RowsOut out, hipStream_t stream)
{
    FG_BY_TYPE(type, c, (combine<T, N>(rows, n_rows, c, index, weights, t, k, walk, out, stream)))
}

hipError_t launch_combine_grad(int32_t type, RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index,
                               const float* weights, int32_t k, RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    FG_BY_TYPE(type, c, (combine_grad_of<T, N>(grad_out, t, c, rows, n_rows, index, weights, k, grad_rows, grad_weights, stream)))
}

}  // namespace fg
