// Sums of rows by index: the gradient of a lookup's table, and of rows that a weighted sum names any number of times, by the sorted index.
#include <type_traits>
#include "fg_pieces.hpp"

namespace fg {

namespace {

// ---- sums over the entries of a row ------------------------------------------------------------------------------------

// Rows that are named often are summed in parts: `chunk` entries of the sorted index that all name one row, and kChunks such chunks, are summed
// by themselves and put together afterwards, so that one lane adds up some hundreds of a row's entries or parts.  (Beyond 500000 entries of one row it is thousands: the
// join's lane has the chunks of chunks, 4096 at most, one after the other.  500000 entries of one row, 64 float32, 63 us, of which the join 34; 4M 458 and 251, where 4M
// entries of 100000 rows take 209.)  chunk is kChunk.  Rows of a
// graph are all named often, and as chunks they would be read by a few scattered lanes: there it grows to four times the mean of a row's
// entries, as far as the rows alone give 512 lanes for every entry of a chunk, so that one lane's share stays small beside the whole (a power of two;
// 20k points, 40 neighbours of 64 float32: 57 us with chunks of 32, 42 with 256; 9k points, 100 neighbours of 128 78 and 50; but entries whose rows follow
// Zipf's law, 1M of 5000 rows of 64 bf16, 308 us with 64 lanes, 90 with 256, 62 so, by now 55; 66k of 105 rows of 2112 147, 90, 80).
//   k_row_sums   chunks of one row each, a row's first and last with its entries before and after them: their sums; rows without such a chunk
//   k_row_parts  chunks of chunks (where there are enough entries)
//   k_row_join   rows with a chunk: chunks up to the first whole chunk of chunks, those, and chunks again
// The long rows' entries are read while the many short ones are written.  Few entries and rows: k_row_sums_few alone, a launch instead of two or three.
// Sums are held in 32 bits and rounded once.  No atomics: the order of a sum goes by the sorted index and the sizes.
//
// Bound by memory: the gradient of 131072 x 2048 float32 from 64k tokens in bf16, the commonest of which comes 4000 times, takes 245 us + 13 for the
// long rows (1.33 GB at 5.2 TB/s); 131072 x 4096 bf16 from 20k tokens 157, what filling it with zeros takes.  In a graph of 100k points with
// 40 neighbours each, 64 float32 a point, 235 us with the weights' gradient: 125 for the points' rows (1 GB out of the last-level cache), 60 for a
// weight and 50 for its gradient an entry, 4 bytes each in a line of its own.  (The products in a kernel of their own: 170 + 150.)  The 40 nearest
// of 100k uniform points: 256, taken in the order of the points' bins (walk) 94.
constexpr int kChunk = 32, kChunks = 32;
constexpr int64_t kPartsFrom = 16;           // chunks of chunks from which on it is looked whether there are any

struct SumArgs {
    const int32_t *index, *order, *bounds;
    const float* weights;
    float* grad_weights;     // DOTS
    int32_t m;
    int64_t n_rows;
    int64_t chunks;          // m / chunk
    Divide by_fan;
    const int32_t* walk;     // the order in which rows are taken, or NULL
    float scale;
    int32_t shift;           // log2 of chunk
    float *parts, *parts2;   // sums of chunks, and of chunks of chunks (NULL: none)
};

// Adds the entries [from, to) of the sorted index to sum.  DOTS: their products with `row` (the piece of the row that they name) are added up over
// the `lanes` lanes that share it and written as their weights' gradients; `real`: this lane has a piece.  AHEAD: a list's next entries are on
// their way while the rows of these are (rows by Zipf's law, 1M entries of 5000 rows of 64 bf16 64 -> 55 us, 50000 of 20000 of 300 29.8 -> 27.6; with products 20k
// points, 40 neighbours of 64 float32 42 -> 45, with the output past the caches, 131072 entries of as many rows of 1024, 164 -> 169: not there).
template <typename T, int N, bool WEIGHTED, bool DOTS, bool AHEAD, int S>
__device__ __forceinline__ void add_entries(typename Piece<T, N>::Wide (&sum)[S], const SumArgs& a, const T* __restrict__ grad, int64_t grad_stride,
                                            int32_t from, int32_t to, const Span<S>& at, const typename Piece<T, N>::Wide& row, bool real, int lanes)
{
    typedef Piece<T, N> P;
    constexpr int MOST = 16 / S < 8 ? 16 / S : 8;
    int32_t ahead[MOST];
    bool have = false;
    in_chunks<MOST>(to - from, [&](auto count, int32_t p, int there) {
        constexpr int U = count.value;
        int32_t entry[U];
        float w[U];
        typename P::Vec v[U][S];
        if (AHEAD && U == MOST && have) {
#pragma unroll
            for (int u = 0; u < U; ++u) entry[u] = ahead[u];
        } else {
            load_words<U>(a.order + from + p, there, entry);
        }
        if (AHEAD && U == MOST) {
            have = to - from - p >= 2 * MOST;
            if (have) load_words<MOST>(a.order + from + p + MOST, MOST, ahead);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if ((uint32_t)entry[u] >= (uint32_t)a.m) entry[u] = 0;         // (no order of fg_index_sort's: nothing outside is read)
            w[u] = WEIGHTED ? a.weights[entry[u]] : 1.0f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int s = 0; s < S; ++s) v[u][s] = load_piece<T, N>(grad + (int64_t)a.by_fan((uint32_t)entry[u]) * grad_stride + at.col[s]);
        float dot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (WEIGHTED) w[u] = u < there ? w[u] : 0.0f;
            float products = 0.0f;
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const typename P::Wide x = wide<T, N>(only_if<T, N>(u < there && (!DOTS || real), v[u][s]));
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    sum[s][i] = WEIGHTED ? __builtin_fmaf(x[i], w[u], sum[s][i]) : sum[s][i] + x[i];
                    if (DOTS) products = __builtin_fmaf(x[i], row[i], products);
                }
            }
            dot[u] = products;
        }
        if constexpr (DOTS) {
            const int lane = threadIdx.x & (lanes - 1), mine = share_of<U>(lane, lanes);
            const float product = add_up<U>(dot, lane, lanes);
            if ((lane & (lanes / U - 1)) == 0 && mine < there) {
                const uint32_t e = (uint32_t)a.order[from + p + mine];
                if (e < (uint32_t)a.m) a.grad_weights[e] = product;
            }
        }
    });
}

// Adds the sums [from, to) of `parts`, one after the other every `stride`.
template <typename T, int N>
__device__ __forceinline__ void add_parts(typename Piece<T, N>::Wide& sum, const float* __restrict__ parts, int64_t stride, int32_t from, int32_t to)
{
    typedef typename Piece<T, N>::Wide Wide;
    constexpr int U = N > 4 ? 4 : 8;
#pragma unroll 1
    for (int32_t q = from; q < to; q += U) {
        Wide v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *reinterpret_cast<const Wide*>(parts + (q + u < to ? q + u : q) * stride);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (q + u < to) sum += v[u];
    }
}

// Whether the entries [p, p + n) of the sorted index all name one row, and which.
__device__ __forceinline__ bool one_row(const SumArgs& a, int32_t p, int32_t n, int32_t& name)
{
    const uint32_t e0 = a.order[p], e1 = a.order[p + n - 1];
    if (e0 >= (uint32_t)a.m || e1 >= (uint32_t)a.m) return false;
    name = a.index[e0];
    return name == a.index[e1] && (uint32_t)name < (uint32_t)a.n_rows;
}

// (bounds that are no fg_index_sort's: nothing outside is read)
__device__ __forceinline__ void within(const SumArgs& a, int32_t& from, int32_t& to)
{
    from = from < 0 ? 0 : (from > a.m ? a.m : from);
    to = to < 0 ? 0 : (to > a.m ? a.m : to);
}
__device__ __forceinline__ int32_t first_chunk(const SumArgs& a, int32_t from) { return (int32_t)(((int64_t)from + (1 << a.shift) - 1) >> a.shift); }

template <typename T, int N, typename TO, bool ACCUMULATE, bool STREAM, int S>
__device__ __forceinline__ void store_sum(float scale, typename Piece<T, N>::Wide (&sum)[S], TO* __restrict__ out, int64_t out_stride, int64_t row,
                                          const Span<S>& at)
{
    typedef TO OutVec __attribute__((ext_vector_type(N), aligned(sizeof(TO))));
    typedef typename Piece<T, N>::Wide Wide;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (!at.there[s] || at.skip[s] >= N) continue;
        TO* p = out + row * out_stride + at.col[s];
        Wide x = sum[s] * scale;
        if (!ACCUMULATE || at.skip[s] == 0) {
            if (ACCUMULATE) x += __builtin_convertvector(*reinterpret_cast<const OutVec*>(p), Wide);
            store_vec<STREAM>(p, __builtin_convertvector(x, OutVec));
        } else {
            // (added once: elements that the piece before covers are left to it)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i >= at.skip[s]) p[i] = (TO)(x[i] + (float)p[i]);
        }
    }
}

// The first chunk_blocks workgroups have the chunks (dc), the others the rows (d).
template <typename T, int N, typename TO, bool WEIGHTED, bool ACCUMULATE, bool DOTS, bool STREAM, int SEGS>
__global__ __launch_bounds__(kBlock, DOTS && sizeof(T) == 2 ? 3 : 4) void k_row_sums(SumArgs a, const int32_t* __restrict__ index,
                                                                                     const int32_t* __restrict__ order, const int32_t* __restrict__ bounds,
                                                                                     const float* __restrict__ weights, const T* __restrict__ grad,
                                                                                     int64_t grad_stride, const T* __restrict__ rows, int64_t rows_stride,
                                                                                     TO* __restrict__ out, int64_t out_stride, Deal dc, Deal d,
                                                                                     unsigned chunk_blocks, bool shared)
{
    typedef Piece<T, N> P;
    constexpr int S = SEGS ? SEGS : 1;
    a.index = index; a.order = order; a.bounds = bounds; a.weights = weights;        // (arguments of their own: nothing stored changes them)
    const bool chunk = blockIdx.x < chunk_blocks;
    int64_t block = chunk ? blockIdx.x : blockIdx.x - chunk_blocks;
    const int64_t blocks = chunk ? chunk_blocks : gridDim.x - chunk_blocks;
    if (!chunk && shared) block = by_xcd(block, blocks);
    const Deal& all = chunk ? dc : d;
    each_span<N, SEGS>(all, block, blocks, [&](const Span<S>& at) {
        int64_t name = at.row;
        int32_t from, to;
        if (chunk) {
            const int32_t q = (int32_t)at.row;
            int32_t of;
            if (!one_row(a, q << a.shift, 1 << a.shift, of)) return;
            name = of;
            from = a.bounds[name];
            to = a.bounds[name + 1];
            within(a, from, to);
            if (first_chunk(a, from) < q) from = q << a.shift;
            if (to >> a.shift > q + 1) to = (q + 1) << a.shift;
        } else {
            if (a.walk) {
                name = (uint32_t)a.walk[name];
                if (name >= a.n_rows) return;
            }
            from = a.bounds[name];
            to = a.bounds[name + 1];
            within(a, from, to);
            if (first_chunk(a, from) < to >> a.shift) return;              // k_row_join
            if (ACCUMULATE && from >= to) return;
        }
        const bool real = !DOTS || at.skip[0] < N;
        typename P::Wide sum[S] = {}, row = {};
        // (a lane without a piece has zeros of the row too: it would add zero times the row's last piece, infinities and all)
        if (DOTS && from < to) row = wide<T, N>(only_if<T, N>(real, load_piece<T, N>(rows + name * rows_stride + at.col[0])));
        add_entries<T, N, WEIGHTED, DOTS, !DOTS && !STREAM, S>(sum, a, grad, grad_stride, from, to, at, row, real, (int)d.pieces);
        if (chunk) {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (real && at.there[s]) *reinterpret_cast<typename P::Wide*>(a.parts + (at.row * d.pieces + at.piece[s]) * N) = sum[s];
        } else {
            // (no entries: zeros, whatever the scale)
            store_sum<T, N, TO, ACCUMULATE, STREAM, S>(from < to ? a.scale : 0.0f, sum, out, out_stride, name, at);
        }
    });
}

// Few entries, spread over many rows: a wavefront for 64 pieces of a row; where a row has more than kAlone entries after all, the workgroup's wavefronts
// take a share of them each and meet in LDS.  Against chunks and their join, us (entries, rows x width): 1000 of 5003 x 257 float32 5.5 / 10.3, 500 of
// 100 x 64 4.3 / 7.5, 100 of 30 x 512 3.3 / 4.6, 64 of 30000 x 256 10.5 / 11.3; but 1000 of 100 x 2048 17.9 / 15.3, 1000 of 3 x 300 21 / 10, 2000 of 2000 x
// 4096 32 / 16.  (All 1000 of one row of many: 21 / 10.)  Lanes behind a row's last piece idle: 48 of 64 with 16 pieces, 63 of the second wavefront's with 65;
// pieces one after the other over the lanes, as deal() would have them there, were not tried.
constexpr int kFewBlock = 512, kAlone = 32;
constexpr int64_t kFewEntries = 1024, kFewUnits = 32768;
inline bool takes_few(int64_t m, int64_t n_rows, int64_t units) { return m <= kFewEntries && m <= 8 * n_rows && units <= kFewUnits; }
template <typename T, int N, typename TO, bool WEIGHTED, bool ACCUMULATE>
__global__ __launch_bounds__(kFewBlock) void k_row_sums_few(SumArgs a, const int32_t* __restrict__ order, const int32_t* __restrict__ bounds,
                                                            const float* __restrict__ weights, const T* __restrict__ grad, int64_t grad_stride,
                                                            TO* __restrict__ out, int64_t out_stride, Deal d)
{
    constexpr int kW = kFewBlock / 64;
    typedef typename Piece<T, N>::Wide Wide;
    __shared__ int32_t range[kW][2];
    __shared__ Wide part[kW][64];
    a.order = order; a.bounds = bounds; a.weights = weights;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    auto span = [&](int w, int64_t& row) {
        const int64_t unit = (int64_t)blockIdx.x * kW + w;
        row = d.by_waves_far(unit);
        return span_of<N, 1>(d, row, (uint32_t)(unit - row * d.waves) * 64 + lane);
    };
    int64_t row;
    const Span<1> at = span(wave, row);
    int32_t from = 0, to = 0;
    const bool there = row < a.n_rows;
    if (there) {
        from = bounds[row];
        to = bounds[row + 1];
        within(a, from, to);
    }
    if (lane == 0) { range[wave][0] = from; range[wave][1] = to; }
    if (there && to - from <= kAlone && !(ACCUMULATE && from >= to)) {
        Wide sum[1] = {}, none = {};
        add_entries<T, N, WEIGHTED, false, false, 1>(sum, a, grad, grad_stride, from, to, at, none, true, 0);
        store_sum<T, N, TO, ACCUMULATE, false, 1>(from < to ? a.scale : 0.0f, sum, out, out_stride, row, at);
    }
    __syncthreads();
    for (int w = 0; w < kW; ++w) {
        const int32_t f = range[w][0], n = range[w][1] - f;
        if (n <= kAlone) continue;
        const int32_t share = (n + kW - 1) / kW, mine = wave * share < n ? wave * share : n, end = mine + share < n ? mine + share : n;
        int64_t of;
        const Span<1> there_at = span(w, of);
        Wide sum[1] = {}, none = {};
        add_entries<T, N, WEIGHTED, false, false, 1>(sum, a, grad, grad_stride, f + mine, f + end, there_at, none, true, 0);
        part[wave][lane] = sum[0];
        __syncthreads();
        if (wave == w) {
            sum[0] = part[0][lane];
#pragma unroll
            for (int i = 1; i < kW; ++i) sum[0] += part[i][lane];
            store_sum<T, N, TO, ACCUMULATE, false, 1>(a.scale, sum, out, out_stride, row, at);
        }
        __syncthreads();
    }
}

template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_row_parts(SumArgs a, Deal d)
{
    each_span<N, 0>(d, [&](const Span<1>& at) {
        int32_t name;
        if (!one_row(a, (int32_t)(at.row * kChunks) << a.shift, kChunks << a.shift, name)) return;
        typename Piece<T, N>::Wide sum = {};
        add_parts<T, N>(sum, a.parts + at.piece[0] * N, (int64_t)d.pieces * N, (int32_t)at.row * kChunks, (int32_t)(at.row + 1) * kChunks);
        *reinterpret_cast<typename Piece<T, N>::Wide*>(a.parts2 + (at.row * d.pieces + at.piece[0]) * N) = sum;
    });
}

// NONE: and the weights' gradients of entries that name no row
template <typename T, int N, typename TO, bool ACCUMULATE, bool NONE>
__global__ __launch_bounds__(kBlock) void k_row_join(SumArgs a, TO* __restrict__ out, int64_t out_stride, Deal d)
{
    if (NONE) {
        int64_t p = a.bounds[a.n_rows];
        for (p = (p < 0 ? 0 : p) + (int64_t)blockIdx.x * kBlock + threadIdx.x; p < a.m; p += (int64_t)gridDim.x * kBlock) {
            const uint32_t e = (uint32_t)a.order[p];
            if (e < (uint32_t)a.m) a.grad_weights[e] = 0.0f;
        }
    }
    each_span<N, 0>(d, [&](const Span<1>& at) {
        const int32_t q0 = (int32_t)at.row;
        int32_t name;
        if (!one_row(a, q0 << a.shift, 1 << a.shift, name)) return;
        int32_t from = a.bounds[name], to = a.bounds[name + 1];
        within(a, from, to);
        if (first_chunk(a, from) != q0) return;                            // the row's first chunk has the row
        const int32_t q1 = to >> a.shift;
        const int64_t stride = (int64_t)d.pieces * N;
        const float *parts = a.parts + at.piece[0] * N, *parts2 = a.parts2 + at.piece[0] * N;
        const int32_t r0 = a.parts2 ? (q0 + kChunks - 1) / kChunks : q1, r1 = a.parts2 ? q1 / kChunks : 0;
        typename Piece<T, N>::Wide sum[1] = {};
        if (r0 < r1) {
            add_parts<T, N>(sum[0], parts, stride, q0, r0 * kChunks);
            add_parts<T, N>(sum[0], parts2, stride, r0, r1);
            add_parts<T, N>(sum[0], parts, stride, r1 * kChunks, q1);
        } else {
            add_parts<T, N>(sum[0], parts, stride, q0, q1);
        }
        store_sum<T, N, TO, ACCUMULATE, false, 1>(a.scale, sum, out, out_stride, name, at);
    });
}

template <typename T, int N, typename TO, bool WEIGHTED, bool ACCUMULATE, bool DOTS>
hipError_t row_sums(const RowSums& r, const SumArgs& a, hipStream_t stream)
{
    const T* grad = (const T*)r.grad.at;
    const T* rows = (const T*)r.rows.at;
    // with products a row's lanes are a power of two, so that they lie in one wavefront
    uint32_t pieces = (uint32_t)((r.c + N - 1) / N);
    if (DOTS) pieces = lanes_for(pieces);
    SumArgs b = a;
    if constexpr (!DOTS) {
        Deal d = deal(r.n_rows, r.c, pieces, 1);
        d.waves = (pieces + 63) / 64;                        // a wavefront for 64 pieces whatever the width
        d.by_waves_far = DivideFar(d.waves);
        d.units = r.n_rows * d.waves;
        if (takes_few(r.m, r.n_rows, d.units)) {
            FG_LAUNCH((k_row_sums_few<T, N, TO, WEIGHTED, ACCUMULATE>), blocks_for(d.units, kFewBlock / 64), dim3(kFewBlock), 0, stream, b, b.order, b.bounds,
                      b.weights, grad, r.grad.stride, (TO*)r.out.at, r.out.stride, d);
            return hipSuccess;
        }
    }
    int64_t chunk = kChunk;
    b.shift = 5;
    // (and with very many entries: chunks of chunks that one lane may have to add up stay below 4096)
    while (chunk < 65536 && ((chunk < 4 * (r.m / r.n_rows) && 2 * chunk * 512 <= r.n_rows * pieces) || r.m / (chunk * kChunks) > 4096)) { chunk *= 2; ++b.shift; }
    b.chunks = r.m / chunk;
    b.parts = r.partials;
    b.parts2 = nullptr;
    const Deal d = deal(r.n_rows, r.c, pieces, DOTS ? 1 : 2);
    Deal dc = deal(b.chunks, r.c, pieces, d.segs);
    if (dc.segs != d.segs) {                                 // few chunks: the same kernel's all the same
        dc.segs = d.segs;
        dc.waves = d.waves;
        dc.by_waves_far = d.by_waves_far;
        dc.units = b.chunks * dc.waves;
    }
    const bool shared = r.fan > 1 && r.m >= kShared * r.n_rows;       // (fan == 1: no row of grad is read twice)
    const unsigned chunk_blocks = b.chunks ? to_xcds(blocks_for(dc, kMostUneven)) : 0, row_blocks = to_xcds(blocks_for(d, kMostUneven));
#define FG_SUMS(STREAM) k_row_sums<T, N, TO, WEIGHTED, ACCUMULATE, DOTS, STREAM
#define FG_SUMS_ARGS                                                                                                                     \
    b, b.index, b.order, b.bounds, b.weights, grad, r.grad.stride, rows, r.rows.stride, (TO*)r.out.at, r.out.stride, dc, d, chunk_blocks, shared
    const bool past = !ACCUMULATE && !DOTS && (r.n_rows * (int64_t)sizeof(TO) + r.m / r.fan * (int64_t)sizeof(T)) * r.c >= kStream;
    const unsigned grid = chunk_blocks + row_blocks;
    if constexpr (DOTS) FG_LAUNCH_DEAL(1, d, grid, stream, FG_SUMS(false), FG_SUMS_ARGS);
    else if (!past) FG_LAUNCH_DEAL(2, d, grid, stream, FG_SUMS(false), FG_SUMS_ARGS);
    else FG_LAUNCH_DEAL(2, d, grid, stream, FG_SUMS(!ACCUMULATE), FG_SUMS_ARGS);
#undef FG_SUMS_ARGS
#undef FG_SUMS
    if (!b.chunks && !DOTS) return hipSuccess;
    if (b.chunks / kChunks >= kPartsFrom) {
        b.parts2 = r.partials + b.chunks * ((int64_t)pieces * N);
        const Deal dp = deal(b.chunks / kChunks, r.c, pieces, 0);
        FG_LAUNCH((k_row_parts<T, N>), blocks_for(dp.total, kBlock), dim3(kBlock), 0, stream, b, dp);
    }
    const Deal dj = deal(b.chunks, r.c, pieces, 0);
    FG_LAUNCH((k_row_join<T, N, TO, ACCUMULATE, DOTS>), blocks_for(dj.total > 0 ? dj.total : 1, kBlock), dim3(kBlock), 0, stream, b, (TO*)r.out.at, r.out.stride, dj);
    return hipSuccess;
}

template <typename T, int N, typename TO>
hipError_t row_sums_of(const RowSums& r, const SumArgs& a, hipStream_t stream)
{
    if constexpr (std::is_same<T, TO>::value) {              // (of combine: the rows' own type)
        if (r.grad_weights)
            return r.weights ? row_sums<T, N, TO, true, false, true>(r, a, stream) : row_sums<T, N, TO, false, false, true>(r, a, stream);
        if (r.weights) return row_sums<T, N, TO, true, false, false>(r, a, stream);
    }
    return r.accumulate ? row_sums<T, N, TO, false, true, false>(r, a, stream) : row_sums<T, N, TO, false, false, false>(r, a, stream);
}

}  // namespace

static int64_t elements_of_piece(int32_t type, int64_t c)
{
    const int64_t n = type == FG_F32 ? 4 : 8;
    return c >= n ? n : 1;
}

// (up to 64 pieces of a row are rounded up to a power of two: the lanes of a row with products; few entries and rows need none: k_row_sums_few, whose pieces
// have four elements at least, or are one)
size_t row_sums_workspace_bytes(int32_t type, int64_t m, int64_t n_rows, int64_t c, bool products)
{
    if (!products && takes_few(m, n_rows, n_rows * ((c + 255) / 256))) return 0;
    const int64_t n = elements_of_piece(type, c);
    int64_t pieces = (c + n - 1) / n;
    if (pieces <= 64) pieces = lanes_for(pieces);
    return (size_t)(m / kChunk + m / (kChunk * kChunks)) * (size_t)(pieces * n) * sizeof(float);
}

bool sums_with_products(int32_t type, int64_t c)
{
    const int64_t n = elements_of_piece(type, c);
    return c % n == 0 && c <= 64 * n;
}

hipError_t launch_row_sums(const RowSums& r, hipStream_t stream)
{
    SumArgs a = {};
    a.index = r.index; a.order = r.order; a.bounds = r.bounds; a.weights = r.weights; a.grad_weights = r.grad_weights; a.walk = r.walk;
    a.m = (int32_t)r.m; a.n_rows = r.n_rows; a.by_fan = Divide((uint32_t)r.fan); a.scale = r.scale;
    if (r.out_type == FG_F32 && r.type != FG_F32) {
        // pieces of 16 bytes of the output, most of what moves where a table is large
        if (r.type == FG_BF16)
            return r.c >= kWide<float> ? row_sums_of<__bf16, kWide<float>, float>(r, a, stream) : row_sums_of<__bf16, 1, float>(r, a, stream);
        if (r.type == FG_F16)
            return r.c >= kWide<float> ? row_sums_of<_Float16, kWide<float>, float>(r, a, stream) : row_sums_of<_Float16, 1, float>(r, a, stream);
    }
    FG_BY_TYPE(r.type, r.c, (row_sums_of<T, N, T>(r, a, stream)))
}

}  // namespace fg
