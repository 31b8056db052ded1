// Rows by index: lookup, copies into an order by expert, weighted sums of rows, and the gradients of all of them.
//
// All of it moves rows; none computes enough to matter.  A lane handles 16 bytes of a row at a time, whatever the row's alignment (global loads
// and stores of 16 bytes need that of an element only).  A row that is no multiple of 16 bytes ends with a piece that begins before its turn
// and covers some elements twice, with the same values; rows shorter than 16 bytes go element by element.  Where every row is finished by
// lanes on their own (all but the products of the weights' gradient), lanes are dealt out over the pieces of all rows in turn, so
// that none idles whatever a row's width; a lane's row is its piece's number divided by the pieces of a row.
// Sums are held in 32 bits and rounded once, in the order of the index: the same in every run.
#include <type_traits>
#include "fg_rows.hpp"

namespace fg {

namespace {

constexpr int kBlock = 256;
constexpr int64_t kFill = 256 * 2048;        // lanes that the chip holds at a time
constexpr int64_t kMostBlocks = 1 << 20;     // more work than that: blocks take several turns

// N elements of a row: 16 bytes, or one element
template <typename T> constexpr int kWide = 16 / sizeof(T);
template <typename T, int N>
struct Piece {
    typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    typedef float Wide __attribute__((ext_vector_type(N)));
    typedef uint32_t Words __attribute__((ext_vector_type(4)));
};
template <typename T, int N>
__device__ __forceinline__ typename Piece<T, N>::Vec load_piece(const T* __restrict__ p) { return *reinterpret_cast<const typename Piece<T, N>::Vec*>(p); }
template <typename T, int N>
__device__ __forceinline__ void store_piece(T* __restrict__ p, typename Piece<T, N>::Vec v) { *reinterpret_cast<typename Piece<T, N>::Vec*>(p) = v; }
template <typename T, int N>
__device__ __forceinline__ typename Piece<T, N>::Wide wide(typename Piece<T, N>::Vec v)
{
    return __builtin_convertvector(v, typename Piece<T, N>::Wide);
}
template <typename T, int N>
__device__ __forceinline__ typename Piece<T, N>::Vec narrow(typename Piece<T, N>::Wide v)
{
    return __builtin_convertvector(v, typename Piece<T, N>::Vec);
}
template <typename T, int N>
__device__ __forceinline__ typename Piece<T, N>::Vec only_if(bool yes, typename Piece<T, N>::Vec v)
{
    typedef Piece<T, N> P;
    if constexpr (N == 1) return yes ? v : typename P::Vec{};
    else {
        typename P::Words w = __builtin_bit_cast(typename P::Words, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = yes ? w[i] : 0u;
        return __builtin_bit_cast(typename P::Vec, w);
    }
}

// The pieces of all rows in turn.
struct Deal {
    int64_t total;                           // rows x pieces of a row
    uint64_t by_pieces_far;                  // ceil(2^64 / pieces): quotients of numbers below 2^31 pieces, for pieces <= 2^16 (FG_MAX_C)
    uint32_t pieces;
    Divide by_pieces;
    int32_t c;
    // the row of piece x; pieces == 1: by_pieces_far would not fit
    __device__ __forceinline__ int64_t row_of(int64_t x) const { return pieces == 1 ? x : (int64_t)__umul64hi((uint64_t)x, by_pieces_far); }
};
struct At {
    int64_t row;
    int32_t col;                             // where the piece begins
    int32_t skip;                            // elements at its beginning that are another's
};
template <int N>
__device__ __forceinline__ At piece_at(const Deal& a, int64_t row0, uint32_t off0, uint32_t ahead)
{
    const uint32_t x = off0 + ahead, q = a.by_pieces(x);
    At at;
    at.row = row0 + q;
    const int32_t col = (int32_t)(x - q * a.pieces) * N, last = a.c > N ? a.c - N : 0;
    at.col = col < last ? col : last;
    at.skip = col - at.col;
    return at;
}

Deal deal(int64_t rows, int64_t c, uint32_t pieces)
{
    Deal a;
    a.pieces = pieces;
    a.total = rows * a.pieces;
    a.by_pieces = Divide(a.pieces);
    a.by_pieces_far = a.pieces == 1 ? 0 : ~(uint64_t)0 / a.pieces + 1;      // (2^64 - 1 and 2^64 have the same quotient but where pieces divides 2^64: + 1 is right for both)
    a.c = (int32_t)c;
    return a;
}
template <typename T, int N>
Deal deal(int64_t rows, int64_t c) { return deal(rows, c, (uint32_t)((c + N - 1) / N)); }
unsigned blocks_for(int64_t total, int64_t each)
{
    const int64_t b = (total + each - 1) / each;
    return (unsigned)(b < kMostBlocks ? b : kMostBlocks);
}

// ---- lookup ------------------------------------------------------------------------------------------------------------

template <typename T, int N, int AHEAD>
__global__ __launch_bounds__(kBlock) void k_lookup(const T* __restrict__ table, int64_t table_stride, uint32_t n_rows, const int32_t* __restrict__ index,
                                                   float scale, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T, N> P;
    for (int64_t first = (int64_t)blockIdx.x * (kBlock * AHEAD); first < d.total; first += (int64_t)gridDim.x * (kBlock * AHEAD)) {
        const int64_t row0 = d.row_of(first);
        const uint32_t off0 = (uint32_t)(first - row0 * d.pieces);
        At at[AHEAD];
        int32_t name[AHEAD];
        typename P::Vec v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const uint32_t ahead = u * kBlock + threadIdx.x;
            at[u] = piece_at<N>(d, row0, off0, ahead);
            if (first + ahead >= d.total) at[u].row = -1;
            name[u] = at[u].row < 0 ? -1 : index[at[u].row];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            v[u] = typename P::Vec{};
            if ((uint32_t)name[u] < n_rows) v[u] = load_piece<T, N>(table + (int64_t)name[u] * table_stride + at[u].col);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (at[u].row >= 0) {
                typename P::Wide x = wide<T, N>(v[u]) * scale;
                if ((uint32_t)name[u] >= n_rows) x = typename P::Wide{};           // also where the scale is not finite
                store_piece<T, N>(out + at[u].row * out_stride + at[u].col, narrow<T, N>(x));
            }
    }
}

// ---- a token's row to its places ---------------------------------------------------------------------------------------

template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_dispatch(const T* __restrict__ x, int64_t x_stride, const int32_t* __restrict__ place, int32_t k,
                                                     uint32_t n_rows, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T, N> P;
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = d.row_of(first);
        const At at = piece_at<N>(d, row0, (uint32_t)(first - row0 * d.pieces), threadIdx.x);
        if (first + threadIdx.x >= d.total) continue;
        const typename P::Vec v = load_piece<T, N>(x + at.row * x_stride + at.col);
        const int32_t* p = place + at.row * k;
        for (int32_t j = 0; j < k; ++j)
            if ((uint32_t)p[j] < n_rows) store_piece<T, N>(out + (int64_t)p[j] * out_stride + at.col, v);
    }
}

// ---- entries, several at a time ----------------------------------------------------------------------------------------

// `U` words from p on, which needs the alignment of a word only; those from `there` on repeat the last.
template <int U, typename W>
__device__ __forceinline__ void load_words(const W* __restrict__ p, int there, W (&x)[U])
{
    typedef W Vec __attribute__((ext_vector_type(U == 1 ? 2 : U), aligned(4)));
    if (U > 1 && there >= U) {
        const Vec v = *reinterpret_cast<const Vec*>(p);
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = v[u];
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = p[u < there ? u : there - 1];
    }
}

// Calls body(U, first, there) over [0, n): eight at a time, the last of a list in one go as 8, 4 or 1 of which `there` are there, so that a short list
// costs one trip to memory and few loads that nobody asked for.
template <int N> struct Count { static constexpr int value = N; };
template <typename Body>
__device__ __forceinline__ void in_chunks(int32_t n, Body&& body)
{
    int32_t at = 0;
#pragma unroll 1
    for (; n - at > 4; at += 8) body(Count<8>{}, at, n - at < 8 ? n - at : 8);
    if (n - at > 1) body(Count<4>{}, at, n - at);
    else if (n - at == 1) body(Count<1>{}, at, 1);
}

// ---- weighted sums -----------------------------------------------------------------------------------------------------

// (n_rows > 0: an entry that names no row reads row 0 and adds zeros in its place, so that no load waits behind a branch)
template <typename T, int N, bool WEIGHTED>
__global__ __launch_bounds__(kBlock) void k_combine(const T* __restrict__ rows, int64_t rows_stride, uint32_t n_rows, const int32_t* __restrict__ index,
                                                    const float* __restrict__ weights, int32_t k, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T, N> P;
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = d.row_of(first);
        const At at = piece_at<N>(d, row0, (uint32_t)(first - row0 * d.pieces), threadIdx.x);
        if (first + threadIdx.x >= d.total) continue;
        typename P::Wide sum = {};
        const int64_t base = at.row * k;
        in_chunks(k, [&](auto count, int32_t j, int there) {
            constexpr int U = count.value;
            int32_t name[U];
            float w[U];
            typename P::Vec v[U];
            load_words<U>(index + base + j, there, name);
            if (WEIGHTED) load_words<U>(weights + base + j, there, w);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool named = u < there && (uint32_t)name[u] < n_rows;
                v[u] = load_piece<T, N>(rows + (named ? (int64_t)name[u] : 0) * rows_stride + at.col);
                if (WEIGHTED) w[u] = named ? w[u] : 0.0f;
                name[u] = named;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const typename P::Wide x = wide<T, N>(only_if<T, N>(name[u], v[u]));
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = WEIGHTED ? __builtin_fmaf(x[i], w[u], sum[i]) : sum[i] + x[i];
            }
        });
        store_piece<T, N>(out + at.row * out_stride + at.col, narrow<T, N>(sum));
    }
}

// ---- gradients of weights, and of rows that are named once -------------------------------------------------------------

// Adds eight values over `lanes` lanes of a wavefront (a power of two from 8 on; the lane's number among them is `lane`): at each of three steps a lane
// hands half of its values to the lane opposite and takes the other half, then the one that is left is added up.  Returns the sum of value
// eighth(lane, lanes).
__device__ __forceinline__ int eighth(int lane, int lanes) { return lane >> (__builtin_ctz(lanes) - 3); }
__device__ __forceinline__ float add_eight(float (&x)[8], int lane, int lanes)
{
    int o = lanes >> 1;
#pragma unroll
    for (int half = 4; half > 0; half >>= 1, o >>= 1) {
        const bool upper = lane & o;
#pragma unroll
        for (int u = 0; u < half; ++u) {
            const float keep = upper ? x[u + half] : x[u], give = upper ? x[u] : x[u + half];
            x[u] = keep + __shfl_xor(give, o);
        }
    }
    float sum = x[0];
    for (; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    return sum;
}

// `lanes` lanes (a power of two from 8 to 64, or 128 or 256: WAVES of them, which meet in LDS) take a token: they walk along its row and those of up
// to eight of its k, so that the token's gradient is loaded once for the eight.
template <typename T, int N, bool ROWS, bool WEIGHTED, int WAVES>
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
        const int64_t row = turn * each + (threadIdx.x >> log);
        const bool there = row < t;
        const int64_t base = there ? row * k : 0;
        for (int32_t j0 = 0; j0 < k; j0 += 8) {
            int32_t name[8];
            float w[8], dot[8];
            load_words<8>(index + base + j0, k - j0, name);
            if (WEIGHTED) load_words<8>(weights + base + j0, k - j0, w);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (j0 + u >= k || (uint32_t)name[u] >= n_rows) name[u] = -1;
                dot[u] = 0.0f;
            }
            for (int32_t turn_col = lane * N; there && turn_col < c; turn_col += lanes * N) {
                const int32_t col = turn_col > c - N ? c - N : turn_col, skip = turn_col - col;
                const typename P::Wide g = wide<T, N>(load_piece<T, N>(grad_out + row * grad_stride + col));
                if (dots) {
                    typename P::Vec v[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (u == 0 || j0 + u < k)
                            v[u] = load_piece<T, N>(rows + (name[u] < 0 ? 0 : (int64_t)name[u]) * rows_stride + col);
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (u == 0 || j0 + u < k) {
                            const typename P::Wide x = wide<T, N>(v[u]);
#pragma unroll
                            for (int i = 0; i < N; ++i)
                                if (i >= skip) dot[u] = __builtin_fmaf(x[i], g[i], dot[u]);
                        }
                }
                if constexpr (ROWS)
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (name[u] >= 0) {
                            float by = WEIGHTED ? w[u] : 1.0f;
                            if (WEIGHTED) asm volatile("" : "+v"(by));       // eight rows' products would otherwise be made ahead, in 64 registers
                            store_piece<T, N>(grad_rows + (int64_t)name[u] * grad_rows_stride + col, narrow<T, N>(WEIGHTED ? g * by : g));
                        }
            }
            if (!grad_weights) continue;
            // (products with row 0, of entries that name none, are dropped here, NaN and all)
#pragma unroll
            for (int u = 0; u < 8; ++u) dot[u] = name[u] < 0 ? 0.0f : dot[u];
            const int some = WAVES > 1 ? 64 : lanes;
            float sum = add_eight(dot, threadIdx.x & (some - 1), some);
            const int u = eighth(threadIdx.x & (some - 1), some);
            bool writes = (threadIdx.x & (some / 8 - 1)) == 0;
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
            if (writes && there && j0 + u < k) grad_weights[base + j0 + u] = sum;
        }
    }
}

// ---- sums over the entries of a row ------------------------------------------------------------------------------------

// Rows that are named often are summed in parts: `chunk` entries of the sorted index that all name one row, and kChunks such chunks, are summed
// beforehand, so that what one lane does for a row hardly grows with the row's entries.  chunk is kChunk, or where there are rows enough to
// fill the chip, four times the mean of a row's entries (a power of two): rows of a graph are named often, but all of them.
constexpr int kChunk = 32, kChunks = 32;
constexpr int64_t kParts2From = 16;          // chunks of chunks from which on it is looked whether there are any

struct SumArgs {
    const int32_t *index, *order, *bounds;
    const float* weights;
    float* grad_weights;     // DOTS
    int32_t m;
    int64_t n_rows;
    int32_t fan;
    Divide by_fan;
    float scale;
    int32_t shift;           // log2 of chunk
    float *parts, *parts2;   // sums of chunks, and of chunks of chunks (NULL: none)
};

// Adds the entries [from, to) of the sorted index to sum.  DOTS: their products with `row` (the piece of the row that they name) are added up over
// the `lanes` lanes that share it and written as their weights' gradients; `real`: this lane has a piece.
template <typename T, int N, bool WEIGHTED, bool DOTS>
__device__ __forceinline__ void add_entries(typename Piece<T, N>::Wide& sum, const SumArgs& a, const T* __restrict__ grad, int64_t grad_stride, int32_t from,
                                            int32_t to, int32_t col, int32_t c, const typename Piece<T, N>::Wide& row, bool real, int lanes)
{
    typedef Piece<T, N> P;
    in_chunks(to - from, [&](auto count, int32_t p, int there) {
        constexpr int U = count.value;
        int32_t entry[U];
        float w[U];
        typename P::Vec v[U];
        load_words<U>(a.order + from + p, there, entry);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if ((uint32_t)entry[u] >= (uint32_t)a.m) entry[u] = 0;         // (no order of fg_index_sort's: nothing outside is read)
            w[u] = WEIGHTED ? a.weights[entry[u]] : 1.0f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (fan == 1: the division by one)
            v[u] = load_piece<T, N>(grad + (int64_t)a.by_fan((uint32_t)entry[u]) * grad_stride + col);
        }
        float dot[8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const typename P::Wide x = wide<T, N>(only_if<T, N>(u < there && (!DOTS || real), v[u]));
            if (WEIGHTED) w[u] = u < there ? w[u] : 0.0f;
            float products = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                sum[i] = WEIGHTED ? __builtin_fmaf(x[i], w[u], sum[i]) : sum[i] + x[i];
                if (DOTS) products = __builtin_fmaf(x[i], row[i], products);
            }
            dot[u] = products;
        }
        if constexpr (DOTS) {
#pragma unroll
            for (int u = U; u < 8; ++u) dot[u] = 0.0f;
            const int lane = threadIdx.x & (lanes - 1), mine = eighth(lane, lanes);
            const float product = add_eight(dot, lane, lanes);
            if ((lane & (lanes / 8 - 1)) == 0 && mine < there) {
                const uint32_t e = (uint32_t)a.order[from + p + mine];
                if (e < (uint32_t)a.m) a.grad_weights[e] = product;
            }
        }
    });
}

template <typename T, int N>
__device__ __forceinline__ void add_parts(typename Piece<T, N>::Wide& sum, const float* __restrict__ parts, int64_t stride, int32_t from, int32_t to)
{
    typedef typename Piece<T, N>::Wide Wide;
    constexpr int U = 4;
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

template <typename T, int N, bool WEIGHTED, bool DOTS>
__global__ __launch_bounds__(kBlock) void k_row_parts(SumArgs a, const T* __restrict__ grad, int64_t grad_stride, const T* __restrict__ rows,
                                                      int64_t rows_stride, Deal d)
{
    typedef Piece<T, N> P;
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = d.row_of(first);
        const uint32_t off0 = (uint32_t)(first - row0 * d.pieces);
        const At at = piece_at<N>(d, row0, off0, threadIdx.x);
        if (first + threadIdx.x >= d.total) continue;
        const int32_t p = (int32_t)at.row << a.shift, n = 1 << a.shift;
        int32_t name;
        if (!one_row(a, p, n, name)) continue;
        float* part = a.parts + (first + threadIdx.x) * N;             // piece after piece: no piece of these overlaps another
        const bool real = at.skip < N;
        if constexpr (DOTS) {
            const typename P::Wide row = wide<T, N>(load_piece<T, N>(rows + (int64_t)name * rows_stride + at.col));
            typename P::Wide sum = {};
            add_entries<T, N, WEIGHTED, true>(sum, a, grad, grad_stride, p, p + n, at.col, d.c, row, real, (int)d.pieces);
            if (real) *reinterpret_cast<typename P::Wide*>(part) = sum;
        } else {
            typename P::Wide sum = {};
            add_entries<T, N, WEIGHTED, false>(sum, a, grad, grad_stride, p, p + n, at.col, d.c, sum, true, 0);
            *reinterpret_cast<typename P::Wide*>(part) = sum;
        }
    }
}

template <typename T, int N>
__global__ __launch_bounds__(kBlock) void k_row_parts_of_parts(SumArgs a, Deal d)
{
    typedef Piece<T, N> P;
    for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
        const int64_t row0 = d.row_of(first);
        const uint32_t x = (uint32_t)(first - row0 * d.pieces) + threadIdx.x, q = d.by_pieces(x);
        if (first + threadIdx.x >= d.total) continue;
        const int64_t r = row0 + q;
        int32_t name;
        if (!one_row(a, (int32_t)(r * kChunks) << a.shift, kChunks << a.shift, name)) continue;
        const int64_t stride = (int64_t)d.pieces * N;
        typename P::Wide sum = {};
        add_parts<T, N>(sum, a.parts + (x - q * d.pieces) * N, stride, (int32_t)r * kChunks, (int32_t)(r + 1) * kChunks);
        *reinterpret_cast<typename P::Wide*>(a.parts2 + (first + threadIdx.x) * N) = sum;
    }
}

// A row's entries: single ones up to the first whole chunk, chunks up to the first whole chunk of chunks, and so back.  `piece`: of the row.
template <typename T, int N, bool WEIGHTED, bool DOTS>
__device__ __forceinline__ void add_row(typename Piece<T, N>::Wide& sum, const SumArgs& a, const T* __restrict__ grad, int64_t grad_stride, int32_t from,
                                        int32_t to, int32_t col, int32_t c, uint32_t piece, uint32_t pieces, const typename Piece<T, N>::Wide& row, bool real)
{
    const int32_t q0 = (from + (1 << a.shift) - 1) >> a.shift, q1 = to >> a.shift;
    const bool parts = q0 < q1;
    // (the single entries before and after the chunks in one loop's code)
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        add_entries<T, N, WEIGHTED, DOTS>(sum, a, grad, grad_stride, side ? q1 << a.shift : from, side || !parts ? to : q0 << a.shift, col, c, row, real,
                                             (int)pieces);
        if (side || !parts) return;
        const int64_t stride = (int64_t)pieces * N;
        const float *at = a.parts + piece * N, *at2 = a.parts2 + piece * N;
        const int32_t r0 = a.parts2 ? (q0 + kChunks - 1) / kChunks : q1, r1 = a.parts2 ? q1 / kChunks : 0;
        if (r0 < r1) {
            add_parts<T, N>(sum, at, stride, q0, r0 * kChunks);
            add_parts<T, N>(sum, at2, stride, r0, r1);
            add_parts<T, N>(sum, at, stride, r1 * kChunks, q1);
        } else {
            add_parts<T, N>(sum, at, stride, q0, q1);
        }
    }
}

// Most rows of a large table have no entry and a store of zeros is all their work; a block takes `turns` runs of pieces and asks for the next run's
// bounds before it works on one.
constexpr int kTurns = 4;
template <typename T, int N, typename TO, bool WEIGHTED, bool ACCUMULATE, bool DOTS>
__global__ __launch_bounds__(kBlock, DOTS && sizeof(T) == 2 ? 3 : 4) void k_row_sums(SumArgs a, const T* __restrict__ grad, int64_t grad_stride, const T* __restrict__ rows,
                                                     int64_t rows_stride, TO* __restrict__ out, int64_t out_stride, Deal d, int turns)
{
    typedef Piece<T, N> P;
    typedef TO OutVec __attribute__((ext_vector_type(N), aligned(sizeof(TO))));
    for (int64_t first = (int64_t)blockIdx.x * (kBlock * turns); first < d.total; first += (int64_t)gridDim.x * (kBlock * turns)) {
        const int64_t row0 = d.row_of(first);
        const uint32_t off0 = (uint32_t)(first - row0 * d.pieces);
        At next = piece_at<N>(d, row0, off0, threadIdx.x);
        int32_t from_next = 0, to_next = 0;
        if (first + threadIdx.x < d.total) { from_next = a.bounds[next.row]; to_next = a.bounds[next.row + 1]; }
        for (int turn = 0; turn < turns; ++turn) {
            const uint32_t ahead = (uint32_t)turn * kBlock + threadIdx.x;
            if (first + ahead >= d.total) break;
            const At at = next;
            int32_t from = from_next, to = to_next;
            if (turn + 1 < turns && first + ahead + kBlock < d.total) {
                next = piece_at<N>(d, row0, off0, ahead + kBlock);
                from_next = a.bounds[next.row];
                to_next = a.bounds[next.row + 1];
            }
            from = from < 0 ? 0 : from;
            to = to > a.m ? a.m : to;
            if (ACCUMULATE && from >= to) continue;
            const uint32_t piece = (uint32_t)(at.col + at.skip) / N;
            const bool real = at.skip < N;
            TO* p = out + at.row * out_stride + at.col;
            typename P::Wide sum = {}, row = {};
            if (from < to) {
                if (DOTS) row = wide<T, N>(load_piece<T, N>(rows + at.row * rows_stride + at.col));
                add_row<T, N, WEIGHTED, DOTS>(sum, a, grad, grad_stride, from, to, at.col, d.c, piece, d.pieces, row, real);
            }
            sum *= a.scale;
            if (!ACCUMULATE || at.skip == 0) {
                OutVec* q = reinterpret_cast<OutVec*>(p);
                if (ACCUMULATE) sum += __builtin_convertvector(*q, typename P::Wide);
                if (!DOTS || real) *q = __builtin_convertvector(sum, OutVec);
            } else {
                // (added once: elements that the piece before covers are left to it)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i >= at.skip) p[i] = (TO)(sum[i] + (float)p[i]);
            }
        }
    }
}

// Weights' gradients of entries that name no row.
__global__ __launch_bounds__(kBlock) void k_no_rows(SumArgs a)
{
    int64_t p = a.bounds[a.n_rows];
    p = (p < 0 ? 0 : p) + (int64_t)blockIdx.x * kBlock + threadIdx.x;
    for (; p < a.m; p += (int64_t)gridDim.x * kBlock) {
        const uint32_t e = (uint32_t)a.order[p];
        if (e < (uint32_t)a.m) a.grad_weights[e] = 0.0f;
    }
}

// lanes that take a row's pieces where they have to meet: a power of two from 8 on
inline uint32_t lanes_for(int64_t pieces)
{
    uint32_t lanes = 8;
    while (lanes < pieces) lanes *= 2;
    return lanes;
}

template <typename T, int N, typename TO, bool WEIGHTED, bool ACCUMULATE, bool DOTS>
hipError_t row_sums(const RowSums& r, const SumArgs& a, hipStream_t stream)
{
    const T* grad = (const T*)r.grad.at;
    const T* rows = (const T*)r.rows.at;
    // with products a row's lanes are a power of two, so that they lie in one wavefront
    uint32_t pieces = (uint32_t)((r.c + N - 1) / N);
    if (DOTS) pieces = lanes_for(pieces);
    const Deal d = deal(r.n_rows, r.c, pieces);
    SumArgs b = a;
    int64_t chunk = kChunk;
    b.shift = 5;
    while (d.total >= kFill && chunk < 4 * (r.m / r.n_rows) && chunk < 65536) { chunk *= 2; ++b.shift; }
    b.parts = r.partials;
    b.parts2 = nullptr;
    const int64_t chunks = r.m / chunk, chunks2 = chunks / kChunks;
    if (chunks) {
        const Deal dp = deal(chunks, r.c, pieces);
        FG_LAUNCH((k_row_parts<T, N, WEIGHTED, DOTS>), dim3(blocks_for(dp.total, kBlock)), dim3(kBlock), 0, stream, b, grad, r.grad.stride, rows,
                  r.rows.stride, dp);
    }
    if (chunks2 >= kParts2From) {
        b.parts2 = r.partials + chunks * ((int64_t)pieces * N);
        const Deal dp = deal(chunks2, r.c, pieces);
        FG_LAUNCH((k_row_parts_of_parts<T, N>), dim3(blocks_for(dp.total, kBlock)), dim3(kBlock), 0, stream, b, dp);
    }
    const int turns = d.total >= (int64_t)kBlock * kTurns * 2048 ? kTurns : 1;
    FG_LAUNCH((k_row_sums<T, N, TO, WEIGHTED, ACCUMULATE, DOTS>), dim3(blocks_for(d.total, kBlock * turns)), dim3(kBlock), 0, stream, b, grad,
              r.grad.stride, rows, r.rows.stride, (TO*)r.out.at, r.out.stride, d, turns);
    if (DOTS) FG_LAUNCH(k_no_rows, dim3(blocks_for((r.m + 15) / 16, kBlock)), dim3(kBlock), 0, stream, b);
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

template <typename T, int N>
hipError_t lookup(RowsIn table, int64_t n_rows, int64_t c, const int32_t* index, int64_t m, float scale, RowsOut out, hipStream_t stream)
{
    constexpr int kFour = 4;
    const Deal d = deal<T, N>(m, c);
    if (d.total < 1024 * kBlock * kFour)
        FG_LAUNCH((k_lookup<T, N, 1>), dim3(blocks_for(d.total, kBlock)), dim3(kBlock), 0, stream, (const T*)table.at, table.stride, (uint32_t)n_rows, index,
                  scale, (T*)out.at, out.stride, d);
    else
        FG_LAUNCH((k_lookup<T, N, kFour>), dim3(blocks_for(d.total, kBlock * kFour)), dim3(kBlock), 0, stream, (const T*)table.at, table.stride,
                  (uint32_t)n_rows, index, scale, (T*)out.at, out.stride, d);
    return hipSuccess;
}

template <typename T, int N>
hipError_t dispatch(RowsIn x, int64_t t, int64_t c, const int32_t* place, int32_t k, int64_t n_rows, RowsOut out, hipStream_t stream)
{
    const Deal d = deal<T, N>(t, c);
    FG_LAUNCH((k_dispatch<T, N>), dim3(blocks_for(d.total, kBlock)), dim3(kBlock), 0, stream, (const T*)x.at, x.stride, place, k, (uint32_t)n_rows, (T*)out.at,
              out.stride, d);
    return hipSuccess;
}

template <typename T, int N>
hipError_t combine(RowsIn rows, int64_t n_rows, int64_t c, const int32_t* index, const float* weights, int64_t t, int32_t k, RowsOut out,
                   hipStream_t stream)
{
    if (n_rows == 0) return lookup<T, N>(rows, 0, c, index, t, 1.0f, out, stream);       // zeros
    const Deal d = deal<T, N>(t, c);
    const dim3 grid(blocks_for(d.total, kBlock));
    if (weights)
        FG_LAUNCH((k_combine<T, N, true>), grid, dim3(kBlock), 0, stream, (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)out.at,
                  out.stride, d);
    else
        FG_LAUNCH((k_combine<T, N, false>), grid, dim3(kBlock), 0, stream, (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)out.at,
                  out.stride, d);
    return hipSuccess;
}

template <typename T, int N, bool ROWS, bool WEIGHTED>
hipError_t combine_grad(RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index, const float* weights, int32_t k,
                        RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    const int64_t pieces = (c + N - 1) / N;
    // a wavefront or less for a token; more, so that a row is one trip to memory, while the chip has room for it
    int lanes = (int)lanes_for(pieces < 64 ? pieces : 64);
    while (lanes < kBlock && lanes < pieces && lanes * t <= kFill) lanes *= 2;
    const dim3 grid(blocks_for(t, kBlock / lanes));
#define FG_COMBINE_GRAD(WAVES)                                                                                                                  \
    FG_LAUNCH((k_combine_grad<T, N, ROWS, WEIGHTED, WAVES>), grid, dim3(kBlock), 0, stream, (const T*)grad_out.at, grad_out.stride, t, (int32_t)c, \
              (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)grad_rows.at, grad_rows.stride, grad_weights, lanes)
    if (lanes == 256) FG_COMBINE_GRAD(4);
    else if (lanes == 128) FG_COMBINE_GRAD(2);
    else FG_COMBINE_GRAD(1);
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

// by type and by width: rows of 16 bytes and more, or shorter ones
#define FG_BY_TYPE(type, c, call)                                                                                         \
    switch (type) {                                                                                                       \
        case FG_F32: FG_BY_WIDTH(float, c, call)                                                                          \
        case FG_BF16: FG_BY_WIDTH(__bf16, c, call)                                                                        \
        case FG_F16: FG_BY_WIDTH(_Float16, c, call)                                                                       \
        default: return hipErrorInvalidValue;                                                                             \
    }
#define FG_BY_WIDTH(type, c, call)                                                                                        \
    {                                                                                                                     \
        typedef type T;                                                                                                   \
        if ((c) >= kWide<T>) { constexpr int N = kWide<T>; return call; }                                                 \
        constexpr int N = 1;                                                                                              \
        return call;                                                                                                      \
    }

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
                          RowsOut out, hipStream_t stream)
{
    FG_BY_TYPE(type, c, (combine<T, N>(rows, n_rows, c, index, weights, t, k, out, stream)))
}

hipError_t launch_combine_grad(int32_t type, RowsIn grad_out, int64_t t, int64_t c, RowsIn rows, int64_t n_rows, const int32_t* index,
                               const float* weights, int32_t k, RowsOut grad_rows, float* grad_weights, hipStream_t stream)
{
    FG_BY_TYPE(type, c, (combine_grad_of<T, N>(grad_out, t, c, rows, n_rows, index, weights, k, grad_rows, grad_weights, stream)))
}

static int64_t elements_of_piece(int32_t type, int64_t c)
{
    const int64_t n = type == FG_F32 ? 4 : 8;
    return c >= n ? n : 1;
}

// (up to 64 pieces of a row are rounded up to a power of two: the lanes of a row with products)
size_t row_sums_workspace_bytes(int32_t type, int64_t m, int64_t c)
{
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
    SumArgs a;
    a.index = r.index; a.order = r.order; a.bounds = r.bounds; a.weights = r.weights; a.grad_weights = r.grad_weights;
    a.m = (int32_t)r.m; a.n_rows = r.n_rows; a.fan = r.fan; a.by_fan = Divide((uint32_t)r.fan); a.scale = r.scale;
    if (r.out_type == FG_F32) {
        FG_BY_TYPE(r.type, r.c, (row_sums_of<T, N, float>(r, a, stream)))
    }
    FG_BY_TYPE(r.type, r.c, (row_sums_of<T, N, T>(r, a, stream)))
}

}  // namespace fg
