// Rows by index: lookup, copies into an order by expert, weighted sums of rows, and the gradients of all of them.
//
// All of it moves rows; none computes enough to matter.  A lane handles 16 bytes of a row at a time, whatever the row's alignment (global loads
// and stores of 16 bytes need that of an element only), the last lane of a row the elements that are left.  Where every row is finished by
// lanes on their own (all but the products of the weights' gradient), lanes are dealt out over the 16-byte pieces of all rows in turn, so
// that none idles whatever a row's width; a lane's row is its piece's number divided by the pieces of a row.
// Sums are held in 32 bits and rounded once, in the order of the index: the same in every run.
#include "fg_rows.hpp"

namespace fg {

namespace {

constexpr int kBlock = 256;
constexpr int64_t kMostBlocks = 1 << 20;     // more work than that: blocks take several turns

template <typename T>
struct Piece {                               // 16 bytes of a row
    static constexpr int kN = 16 / sizeof(T);
    typedef T Vec __attribute__((ext_vector_type(kN), aligned(sizeof(T))));
    typedef float Wide __attribute__((ext_vector_type(kN)));
};

// The piece at p, of which n elements are there.  FULL: all.
template <typename T, bool FULL>
__device__ __forceinline__ typename Piece<T>::Vec load_piece(const T* __restrict__ p, int n)
{
    typedef typename Piece<T>::Vec Vec;
    if constexpr (FULL) return *reinterpret_cast<const Vec*>(p);
    Vec v = {};
#pragma unroll
    for (int i = 0; i < Piece<T>::kN - 1; ++i)
        if (i < n) v[i] = p[i];
    return v;
}
template <typename T, bool FULL>
__device__ __forceinline__ void store_piece(T* __restrict__ p, typename Piece<T>::Vec v, int n)
{
    typedef typename Piece<T>::Vec Vec;
    if constexpr (FULL) {
        *reinterpret_cast<Vec*>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < Piece<T>::kN - 1; ++i)
        if (i < n) p[i] = v[i];
}
template <typename T>
__device__ __forceinline__ typename Piece<T>::Wide wide(typename Piece<T>::Vec v)
{
    return __builtin_convertvector(v, typename Piece<T>::Wide);
}
template <typename T>
__device__ __forceinline__ typename Piece<T>::Vec narrow(typename Piece<T>::Wide v)
{
    return __builtin_convertvector(v, typename Piece<T>::Vec);
}

// FULL as a type: body(Full<true>{}) or body(Full<false>{})
template <bool F> struct Full { static constexpr bool value = F; };
template <typename T, typename Body>
__device__ __forceinline__ void by_fullness(int n, Body&& body)
{
    if (n >= Piece<T>::kN) body(Full<true>{}); else body(Full<false>{});
}

// The pieces of all rows in turn: piece number `first + lane` of a block's turn.
struct Deal {
    int64_t total;                           // rows x pieces of a row
    uint32_t pieces;
    Divide by_pieces;
    int32_t c;
};
struct At { int64_t row; int32_t col; int n; };
template <int N>
__device__ __forceinline__ At piece_at(const Deal& a, int64_t row0, uint32_t off0, uint32_t ahead)
{
    const uint32_t x = off0 + ahead, q = a.by_pieces(x);
    At at;
    at.row = row0 + q;
    at.col = (int32_t)(x - q * a.pieces) * N;
    at.n = a.c - at.col;
    return at;
}

template <int N>
Deal deal(int64_t rows, int64_t c)
{
    Deal a;
    a.pieces = (uint32_t)((c + N - 1) / N);
    a.total = rows * a.pieces;
    a.by_pieces = Divide(a.pieces);
    a.c = (int32_t)c;
    return a;
}
unsigned blocks_for(int64_t total, int64_t each)
{
    const int64_t b = (total + each - 1) / each;
    return (unsigned)(b < kMostBlocks ? b : kMostBlocks);
}

// ---- lookup ------------------------------------------------------------------------------------------------------------

template <typename T, int AHEAD>
__global__ __launch_bounds__(kBlock) void k_lookup(const T* __restrict__ table, int64_t table_stride, uint32_t n_rows, const int32_t* __restrict__ index,
                                                   float scale, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T> P;
    for (int64_t first = (int64_t)blockIdx.x * (kBlock * AHEAD); first < d.total; first += (int64_t)gridDim.x * (kBlock * AHEAD)) {
        const int64_t row0 = first / d.pieces;
        const uint32_t off0 = (uint32_t)(first - row0 * d.pieces);
        At at[AHEAD];
        int32_t name[AHEAD];
        typename P::Vec v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t ahead = u * kBlock + threadIdx.x;
            at[u] = piece_at<P::kN>(d, row0, off0, ahead);
            if (first + ahead >= d.total) at[u].n = 0;
            name[u] = at[u].n > 0 ? index[at[u].row] : -1;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            v[u] = typename P::Vec{};
            if ((uint32_t)name[u] < n_rows) {
                const T* p = table + (int64_t)name[u] * table_stride + at[u].col;
                by_fullness<T>(at[u].n, [&](auto full) { v[u] = load_piece<T, full.value>(p, at[u].n); });
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (at[u].n > 0) {
                T* p = out + at[u].row * out_stride + at[u].col;
                typename P::Wide x = wide<T>(v[u]) * scale;
                if ((uint32_t)name[u] >= n_rows) x = typename P::Wide{};           // also where the scale is not finite
                by_fullness<T>(at[u].n, [&](auto full) { store_piece<T, full.value>(p, narrow<T>(x), at[u].n); });
            }
    }
}

// ---- a token's row to its places ---------------------------------------------------------------------------------------

template <typename T>
__global__ __launch_bounds__(kBlock) void k_dispatch(const T* __restrict__ x, int64_t x_stride, const int32_t* __restrict__ place, int32_t k,
                                                     uint32_t n_rows, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T> P;
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = first / d.pieces;
        const At at = piece_at<P::kN>(d, row0, (uint32_t)(first - row0 * d.pieces), threadIdx.x);
        if (first + threadIdx.x >= d.total) continue;
        by_fullness<T>(at.n, [&](auto full) {
            const typename P::Vec v = load_piece<T, full.value>(x + at.row * x_stride + at.col, at.n);
            const int32_t* p = place + at.row * k;
            for (int32_t j = 0; j < k; ++j)
                if ((uint32_t)p[j] < n_rows) store_piece<T, full.value>(out + (int64_t)p[j] * out_stride + at.col, v, at.n);
        });
    }
}

// ---- weighted sums -----------------------------------------------------------------------------------------------------

constexpr int kAhead = 8;                    // rows whose pieces are under way at a time

template <typename T, bool WEIGHTED>
__global__ __launch_bounds__(kBlock) void k_combine(const T* __restrict__ rows, int64_t rows_stride, uint32_t n_rows, const int32_t* __restrict__ index,
                                                    const float* __restrict__ weights, int32_t k, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T> P;
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = first / d.pieces;
        const At at = piece_at<P::kN>(d, row0, (uint32_t)(first - row0 * d.pieces), threadIdx.x);
        if (first + threadIdx.x >= d.total) continue;
        by_fullness<T>(at.n, [&](auto full) {
            typename P::Wide sum = {};
            const int64_t base = at.row * k;
            for (int32_t j0 = 0; j0 < k; j0 += kAhead) {
                int32_t name[kAhead];
                float w[kAhead];
                typename P::Vec v[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    name[u] = j0 + u < k ? index[base + j0 + u] : -1;
                    w[u] = WEIGHTED && j0 + u < k ? weights[base + j0 + u] : 1.0f;
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    v[u] = typename P::Vec{};
                    if ((uint32_t)name[u] < n_rows) v[u] = load_piece<T, full.value>(rows + (int64_t)name[u] * rows_stride + at.col, at.n);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if ((uint32_t)name[u] < n_rows) {
                        const typename P::Wide x = wide<T>(v[u]);
#pragma unroll
                        for (int i = 0; i < P::kN; ++i) sum[i] = __builtin_fmaf(x[i], w[u], sum[i]);
                    }
            }
            store_piece<T, full.value>(out + at.row * out_stride + at.col, narrow<T>(sum), at.n);
        });
    }
}

// ---- gradients of weights, and of rows that are named once -------------------------------------------------------------

// `lanes` (a power of two, up to 64: a part of a wavefront; 256: the block) take a token: they walk along its row and those of up to eight
// of its k, so that the token's gradient is loaded once for the eight, whose products they add up at the end.
template <typename T, bool ROWS, bool WEIGHTED, bool WHOLE_BLOCK>
__global__ __launch_bounds__(kBlock) void k_combine_grad(const T* __restrict__ grad_out, int64_t grad_stride, int64_t t, int32_t c,
                                                         const T* __restrict__ rows, int64_t rows_stride, uint32_t n_rows,
                                                         const int32_t* __restrict__ index, const float* __restrict__ weights, int32_t k,
                                                         T* __restrict__ grad_rows, int64_t grad_rows_stride, float* __restrict__ grad_weights,
                                                         int lanes)
{
    typedef Piece<T> P;
    __shared__ float part[kBlock / 64][kAhead];
    const int lane = threadIdx.x & (lanes - 1);
    const int each = kBlock / lanes;
    const int64_t turns = (t + each - 1) / each;
    for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x) {
        const int64_t row = WHOLE_BLOCK ? turn : turn * each + threadIdx.x / lanes;
        const bool there = row < t;
        const int64_t base = row * k;
        for (int32_t j0 = 0; j0 < k; j0 += kAhead) {
            int32_t name[kAhead];
            float w[kAhead], dot[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const bool named = there && j0 + u < k;
                name[u] = named ? index[base + j0 + u] : -1;
                w[u] = WEIGHTED && named ? weights[base + j0 + u] : 1.0f;
                dot[u] = 0.0f;
            }
            for (int64_t col = (int64_t)lane * P::kN; there && col < c; col += (int64_t)lanes * P::kN) {
                const int n = c - (int32_t)col;
                by_fullness<T>(n, [&](auto full) {
                    const typename P::Wide g = wide<T>(load_piece<T, full.value>(grad_out + row * grad_stride + col, n));
                    typename P::Vec v[kAhead];
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        v[u] = typename P::Vec{};
                        if ((uint32_t)name[u] < n_rows && grad_weights)
                            v[u] = load_piece<T, full.value>(rows + (int64_t)name[u] * rows_stride + col, n);
                    }
#pragma unroll
                    for (int u = 0; u < kAhead; ++u)
                        if ((uint32_t)name[u] < n_rows) {
                            const typename P::Wide x = wide<T>(v[u]);
#pragma unroll
                            for (int i = 0; i < P::kN; ++i)
                                if (full.value || i < n) dot[u] = __builtin_fmaf(x[i], g[i], dot[u]);
                            if constexpr (ROWS)
                                store_piece<T, full.value>(grad_rows + (int64_t)name[u] * grad_rows_stride + col, narrow<T>(g * w[u]), n);
                        }
                });
            }
            if (!grad_weights) continue;
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                for (int o = (WHOLE_BLOCK ? 64 : lanes) >> 1; o > 0; o >>= 1) dot[u] += __shfl_xor(dot[u], o);
            if constexpr (WHOLE_BLOCK) {
                if ((threadIdx.x & 63) == 0)
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) part[threadIdx.x >> 6][u] = dot[u];
                __syncthreads();
                if (threadIdx.x == 0)
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) dot[u] = (part[0][u] + part[1][u]) + (part[2][u] + part[3][u]);
                __syncthreads();
            }
            if (lane == 0 && there)
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (j0 + u < k) grad_weights[base + j0 + u] = dot[u];
        }
    }
}

// ---- sums over the entries of a row ------------------------------------------------------------------------------------

constexpr int kChunk = 64;                   // entries of the sorted index that are summed beforehand where all name one row
constexpr int kSumAhead = 4;

struct SumArgs {
    const int32_t *index, *order, *bounds;
    const float* weights;
    int32_t m;
    int64_t n_rows;
    int32_t fan;
    Divide by_fan;
    float scale;
};

// Adds the entries [from, to) of the sorted index to sum.
template <typename T, bool WEIGHTED, bool FULL>
__device__ __forceinline__ void add_entries(typename Piece<T>::Wide& sum, const SumArgs& a, const T* __restrict__ grad, int64_t grad_stride, int32_t from,
                                            int32_t to, int32_t col, int n)
{
    typedef Piece<T> P;
    for (int32_t p0 = from; p0 < to; p0 += kSumAhead) {
        int32_t entry[kSumAhead];
        float w[kSumAhead];
        typename P::Vec v[kSumAhead];
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) entry[u] = p0 + u < to ? a.order[p0 + u] : -1;
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u) {
            v[u] = typename P::Vec{};
            w[u] = 1.0f;
            if ((uint32_t)entry[u] < (uint32_t)a.m) {
                const int64_t row = a.fan == 1 ? (uint32_t)entry[u] : a.by_fan((uint32_t)entry[u]);
                v[u] = load_piece<T, FULL>(grad + row * grad_stride + col, n);
                if (WEIGHTED) w[u] = a.weights[entry[u]];
            }
        }
#pragma unroll
        for (int u = 0; u < kSumAhead; ++u)
            if ((uint32_t)entry[u] < (uint32_t)a.m) {
                const typename P::Wide x = wide<T>(v[u]);
#pragma unroll
                for (int i = 0; i < P::kN; ++i) sum[i] = WEIGHTED ? __builtin_fmaf(x[i], w[u], sum[i]) : sum[i] + x[i];
            }
    }
}

// Rows with many entries: chunk q is summed here if all its entries name one row, so that such a row's sum is spread over many lanes.
template <typename T, bool WEIGHTED>
__global__ __launch_bounds__(kBlock) void k_row_parts(SumArgs a, const T* __restrict__ grad, int64_t grad_stride, float* __restrict__ partials, Deal d)
{
    typedef Piece<T> P;
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = first / d.pieces;
        const At at = piece_at<P::kN>(d, row0, (uint32_t)(first - row0 * d.pieces), threadIdx.x);
        if (first + threadIdx.x >= d.total) continue;
        const int32_t p0 = (int32_t)at.row * kChunk;
        const int32_t e0 = a.order[p0], e1 = a.order[p0 + kChunk - 1];
        if ((uint32_t)e0 >= (uint32_t)a.m || (uint32_t)e1 >= (uint32_t)a.m) continue;
        const int32_t name = a.index[e0];
        if (name != a.index[e1] || (uint32_t)name >= (uint32_t)a.n_rows) continue;
        by_fullness<T>(at.n, [&](auto full) {
            typename P::Wide sum = {};
            add_entries<T, WEIGHTED, full.value>(sum, a, grad, grad_stride, p0, p0 + kChunk, at.col, at.n);
            *reinterpret_cast<typename P::Wide*>(partials + at.row * ((int64_t)d.pieces * P::kN) + at.col) = sum;
        });
    }
}

template <typename T, typename TO, bool WEIGHTED, bool ACCUMULATE>
__global__ __launch_bounds__(kBlock) void k_row_sums(SumArgs a, const T* __restrict__ grad, int64_t grad_stride, const float* __restrict__ partials,
                                                     TO* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T> P;
    typedef TO OutVec __attribute__((ext_vector_type(P::kN), aligned(sizeof(TO))));
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = first / d.pieces;
        const At at = piece_at<P::kN>(d, row0, (uint32_t)(first - row0 * d.pieces), threadIdx.x);
        if (first + threadIdx.x >= d.total) continue;
        int32_t from = a.bounds[at.row], to = a.bounds[at.row + 1];
        from = from < 0 ? 0 : from;
        to = to > a.m ? a.m : to;
        if (ACCUMULATE && from >= to) continue;
        by_fullness<T>(at.n, [&](auto full) {
            typename P::Wide sum = {};
            const int32_t q0 = (from + kChunk - 1) / kChunk, q1 = to / kChunk;
            if (q0 < q1) {
                add_entries<T, WEIGHTED, full.value>(sum, a, grad, grad_stride, from, q0 * kChunk, at.col, at.n);
                const int64_t stride = (int64_t)d.pieces * P::kN;
                for (int32_t q = q0; q < q1; ++q) sum += *reinterpret_cast<const typename P::Wide*>(partials + q * stride + at.col);
                add_entries<T, WEIGHTED, full.value>(sum, a, grad, grad_stride, q1 * kChunk, to, at.col, at.n);
            } else {
                add_entries<T, WEIGHTED, full.value>(sum, a, grad, grad_stride, from, to, at.col, at.n);
            }
            sum *= a.scale;
            TO* p = out + at.row * out_stride + at.col;
            if constexpr (full.value) {
                OutVec* q = reinterpret_cast<OutVec*>(p);
                if (ACCUMULATE) sum += __builtin_convertvector(*q, typename P::Wide);
                *q = __builtin_convertvector(sum, OutVec);
            } else {
#pragma unroll
                for (int i = 0; i < P::kN - 1; ++i)
                    if (i < at.n) p[i] = (TO)(ACCUMULATE ? sum[i] + (float)p[i] : sum[i]);
            }
        });
    }
}

template <typename T, typename TO, bool WEIGHTED, bool ACCUMULATE>
hipError_t row_sums(const RowSums& r, const SumArgs& a, hipStream_t stream)
{
    const T* grad = (const T*)r.grad.at;
    if (const int64_t chunks = r.m / kChunk) {
        const Deal d = deal<Piece<T>::kN>(chunks, r.c);
        FG_LAUNCH((k_row_parts<T, WEIGHTED>), dim3(blocks_for(d.total, kBlock)), dim3(kBlock), 0, stream, a, grad, r.grad.stride, r.partials, d);
    }
    const Deal d = deal<Piece<T>::kN>(r.n_rows, r.c);
    FG_LAUNCH((k_row_sums<T, TO, WEIGHTED, ACCUMULATE>), dim3(blocks_for(d.total, kBlock)), dim3(kBlock), 0, stream, a, grad, r.grad.stride,
              (const float*)r.partials, (TO*)r.out.at, r.out.stride, d);
    return hipSuccess;
}

template <typename T, typename TO>
hipError_t row_sums_of(const RowSums& r, const SumArgs& a, hipStream_t stream)
{
    if (r.weights) return row_sums<T, TO, true, false>(r, a, stream);
    return r.accumulate ? row_sums<T, TO, false, true>(r, a, stream) : row_sums<T, TO, false, false>(r, a, stream);
}

template <typename T>
hipError_t lookup(RowsIn table, int64_t n_rows, int64_t c, const int32_t* index, int64_t m, float scale, RowsOut out, hipStream_t stream)
{
    constexpr int kFour = 4;
    const Deal d = deal<Piece<T>::kN>(m, c);
    if (d.total < 1024 * kBlock * kFour)
        FG_LAUNCH((k_lookup<T, 1>), dim3(blocks_for(d.total, kBlock)), dim3(kBlock), 0, stream, (const T*)table.at, table.stride, (uint32_t)n_rows, index,
                  scale, (T*)out.at, out.stride, d);
    else
        FG_LAUNCH((k_lookup<T, kFour>), dim3(blocks_for(d.total, kBlock * kFour)), dim3(kBlock), 0, stream, (const T*)table.at, table.stride,
                  (uint32_t)n_rows, index, scale, (T*)out.at, out.stride, d);
    return hipSuccess;
}

template <typename T>
hipError_t dispatch(RowsIn x, int64_t t, int64_t c, const int32_t* place, int32_t k, int64_t n_rows, RowsOut out, hipStream_t stream)
{
    const Deal d = deal<Piece<T>::kN>(t, c);
    FG_LAUNCH(k_dispatch<T>, dim3(blocks_for(d.total, kBlock)), dim3(kBlock), 0, stream, (const T*)x.at, x.stride, place, k, (uint32_t)n_rows, (T*)out.at,
              out.stride, d);
    return hipSuccess;
}

template <typename T>
hipError_t combine(RowsIn rows, int64_t n_rows, int64_t c, const int32_t* index, const float* weights, int64_t t, int32_t k, RowsOut out,
                   hipStream_t stream)
{
    const Deal d = deal<Piece<T>::kN>(t, c);
    const dim3 grid(blocks_for(d.total, kBlock));
    if (weights)
        FG_LAUNCH((k_combine<T, true>), grid, dim3(kBlock), 0, stream, (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)out.at,
                  out.stride, d);
    else
        FG_LAUNCH((k_combine<T, false>), grid, dim3(kBlock), 0, stream, (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)out.at,
                  out.stride, d);
    return hipSuccess;
}

template <typename T, bool ROWS, bool WEIGHTED>
hipError_t combine_grad(RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index, const float* weights, int32_t k,
                        RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    const int64_t pieces = (c + Piece<T>::kN - 1) / Piece<T>::kN;
    int lanes = 1;
    while (lanes < 64 && lanes < pieces) lanes *= 2;
    const bool whole = pieces > 64 && t < 2048;               // too few tokens for a wavefront each to fill the chip
    if (whole)
        FG_LAUNCH((k_combine_grad<T, ROWS, WEIGHTED, true>), dim3((unsigned)t), dim3(kBlock), 0, stream, (const T*)grad_out.at, grad_out.stride, t,
                  (int32_t)c, (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)grad_rows.at, grad_rows.stride, grad_weights, kBlock);
    else
        FG_LAUNCH((k_combine_grad<T, ROWS, WEIGHTED, false>), dim3(blocks_for(t, kBlock / lanes)), dim3(kBlock), 0, stream, (const T*)grad_out.at,
                  grad_out.stride, t, (int32_t)c, (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)grad_rows.at,
                  grad_rows.stride, grad_weights, lanes);
    return hipSuccess;
}

template <typename T>
hipError_t combine_grad_of(RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index, const float* weights, int32_t k,
                           RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    if (!grad_rows.at) return combine_grad<T, false, false>(grad_out, t, c, rows, n_rows, index, nullptr, k, grad_rows, grad_weights, stream);
    if (!weights) return combine_grad<T, true, false>(grad_out, t, c, rows, n_rows, index, weights, k, grad_rows, grad_weights, stream);
    return combine_grad<T, true, true>(grad_out, t, c, rows, n_rows, index, weights, k, grad_rows, grad_weights, stream);
}

}  // namespace

#define FG_BY_TYPE(type, call)                                  \
    switch (type) {                                             \
        case FG_F32: { typedef float T; return call; }          \
        case FG_BF16: { typedef __bf16 T; return call; }        \
        case FG_F16: { typedef _Float16 T; return call; }       \
        default: return hipErrorInvalidValue;                   \
    }

hipError_t launch_lookup(int32_t type, RowsIn table, int64_t n_rows, int64_t c, const int32_t* index, int64_t m, float scale, RowsOut out,
                         hipStream_t stream)
{
    FG_BY_TYPE(type, (lookup<T>(table, n_rows, c, index, m, scale, out, stream)))
}

hipError_t launch_dispatch(int32_t type, RowsIn x, int64_t t, int64_t c, const int32_t* place, int32_t k, int64_t n_rows, RowsOut out,
                           hipStream_t stream)
{
    FG_BY_TYPE(type, (dispatch<T>(x, t, c, place, k, n_rows, out, stream)))
}

hipError_t launch_combine(int32_t type, RowsIn rows, int64_t n_rows, int64_t c, const int32_t* index, const float* weights, int64_t t, int32_t k,
                          RowsOut out, hipStream_t stream)
{
    FG_BY_TYPE(type, (combine<T>(rows, n_rows, c, index, weights, t, k, out, stream)))
}

hipError_t launch_combine_grad(int32_t type, RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index,
                               const float* weights, int32_t k, RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    FG_BY_TYPE(type, (combine_grad_of<T>(grad_out, t, c, rows, n_rows, index, weights, k, grad_rows, grad_weights, stream)))
}

size_t row_sums_workspace_bytes(int32_t type, int64_t m, int64_t c)
{
    const int64_t n = type == FG_F32 ? 4 : 8;
    return (size_t)(m / kChunk) * (size_t)((c + n - 1) / n * n) * sizeof(float);
}

hipError_t launch_row_sums(const RowSums& r, hipStream_t stream)
{
    SumArgs a;
    a.index = r.index; a.order = r.order; a.bounds = r.bounds; a.weights = r.weights;
    a.m = (int32_t)r.m; a.n_rows = r.n_rows; a.fan = r.fan; a.by_fan = Divide((uint32_t)r.fan); a.scale = r.scale;
    if (r.out_type == FG_F32) {
        FG_BY_TYPE(r.type, (row_sums_of<T, float>(r, a, stream)))
    }
    FG_BY_TYPE(r.type, (row_sums_of<T, T>(r, a, stream)))
}

}  // namespace fg
