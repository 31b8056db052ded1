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
constexpr int64_t kMostBlocks = 1 << 14;     // eight for every place on the chip; more work than that: blocks take several turns
constexpr int64_t kMostUneven = 1 << 20;     // the same where pieces differ in what they take: a block that is done makes room for the next
constexpr int64_t kFewWaves = 256 * 16;      // half of the wavefronts that the chip holds
constexpr int64_t kStream = 512 << 20;       // bytes that a call moves, twice the last-level cache, from which on most of its output has left that cache

// N elements of a row: 16 bytes, or one element
template <typename T> constexpr int kWide = 16 / sizeof(T);
template <typename T, int N>
struct Piece {
    typedef T Vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    typedef float Wide __attribute__((ext_vector_type(N)));
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    typedef uint32_t Words __attribute__((ext_vector_type(kWords < 1 ? 1 : kWords)));
};
// STREAM: past the caches, where nobody would find it again (kStream).  A template argument: of two accesses behind a test the compiler makes one
template <typename T, int N, bool STREAM = false>
__device__ __forceinline__ typename Piece<T, N>::Vec load_piece(const T* __restrict__ p)
{
    const auto* at = reinterpret_cast<const typename Piece<T, N>::Vec*>(p);
    if constexpr (STREAM) return __builtin_nontemporal_load(at);
    else return *at;
}
template <bool STREAM, typename V, typename T>
__device__ __forceinline__ void store_vec(T* __restrict__ p, V v)
{
    typedef V Loose __attribute__((aligned(sizeof(T))));
    if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<Loose*>(p));
    else *reinterpret_cast<Loose*>(p) = v;
}
template <typename T, int N, bool STREAM = false>
__device__ __forceinline__ void store_piece(T* __restrict__ p, typename Piece<T, N>::Vec v) { store_vec<STREAM>(p, v); }
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
        for (int i = 0; i < P::kWords; ++i) w[i] = yes ? w[i] : 0u;
        return __builtin_bit_cast(typename P::Vec, w);
    }
}

// ceil(2^64 / d), for quotients x / d of x < 2^31 d, d <= 2^16 (what M d exceeds 2^64 by, less than d, times x stays below it); d == 1: 0
struct DivideFar {
    uint64_t mul;
    DivideFar() = default;
    explicit DivideFar(uint32_t d) : mul(d == 1 ? 0 : ~(uint64_t)0 / d + 1) {}
    __device__ __forceinline__ int64_t operator()(int64_t x) const { return mul == 0 ? x : (int64_t)__umul64hi((uint64_t)x, mul); }
};

// How the pieces of all rows are dealt out.  One after the other over all lanes: no lane idles whatever a row's width, and every lane works out its
// row.  Or, where a row's pieces fill wavefronts to three quarters at least, ROWWISE: a wavefront for SEGS x 64 pieces of one row, so that what goes
// by the row (index, bounds, addresses, branches) is the scalar unit's and a wavefront has several kilobytes under way before it ends.
struct Deal {
    int64_t total;                           // rows x pieces of a row
    int64_t units;                           // rows x wavefronts of a row
    uint32_t pieces, waves;
    Divide by_pieces;
    DivideFar by_pieces_far, by_waves_far;
    int32_t c;
    int32_t segs;                            // 0: one after the other
};
template <int SEGS>
struct Span {
    int64_t row;
    uint32_t piece[SEGS];
    int32_t col[SEGS];                       // where the piece begins
    int32_t skip[SEGS];                      // elements at its beginning that are another's
    bool there[SEGS];                        // (where it isn't, col is the row's last piece)
};
template <int N, int SEGS>
__device__ __forceinline__ Span<SEGS> span_of(const Deal& d, int64_t row, uint32_t piece)
{
    Span<SEGS> at;
    at.row = row;
#pragma unroll
    for (int s = 0; s < SEGS; ++s) {
        at.piece[s] = piece + s * 64;
        const int32_t col = (int32_t)at.piece[s] * N, last = d.c > N ? d.c - N : 0;
        at.col[s] = col < last ? col : last;
        at.skip[s] = col - at.col[s];
        at.there[s] = at.piece[s] < d.pieces;
    }
    return at;
}
// SEGS == 0: one after the other
template <int N, int SEGS, typename Body>
__device__ __forceinline__ void each_span(const Deal& d, Body&& body)
{
    if constexpr (SEGS > 0) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        for (int64_t unit = (int64_t)blockIdx.x * (kBlock / 64) + wave; unit < d.units; unit += (int64_t)gridDim.x * (kBlock / 64)) {
            const int64_t row = d.by_waves_far(unit);
            body(span_of<N, SEGS>(d, row, (uint32_t)(unit - row * d.waves) * (64 * SEGS) + lane));
        }
    } else {
        for (int64_t first = (int64_t)blockIdx.x * kBlock; first < d.total; first += (int64_t)gridDim.x * kBlock) {
            const int64_t row0 = d.by_pieces_far(first);
            const uint32_t x = (uint32_t)(first - row0 * d.pieces) + threadIdx.x, q = d.by_pieces(x);
            if (first + threadIdx.x < d.total) body(span_of<N, 1>(d, row0 + q, x - q * d.pieces));
        }
    }
}

Deal deal(int64_t rows, int64_t c, uint32_t pieces, int most_segs)
{
    Deal d;
    d.pieces = pieces;
    d.total = rows * pieces;
    d.by_pieces = Divide(pieces);
    d.by_pieces_far = DivideFar(pieces);
    const uint32_t waves = (pieces + 63) / 64;
    d.segs = 4 * pieces >= 3 * 64 * waves ? 1 : 0;
    if (d.segs && most_segs >= 4 && (waves % 4 == 0 || waves >= 12)) d.segs = 4;
    else if (d.segs && most_segs >= 2 && (waves % 2 == 0 || waves >= 6)) d.segs = 2;
    // a few rows: a wavefront for each 64 pieces, so that more of the chip has a part
    if (d.segs && rows * waves < kFewWaves) d.segs = 1;
    d.waves = d.segs ? (waves + d.segs - 1) / d.segs : 1;
    d.by_waves_far = DivideFar(d.waves);
    d.units = rows * d.waves;
    d.c = (int32_t)c;
    return d;
}
template <typename T, int N>
Deal deal(int64_t rows, int64_t c, int most_segs) { return deal(rows, c, (uint32_t)((c + N - 1) / N), most_segs); }
dim3 blocks_for(int64_t total, int64_t each, int64_t most = kMostBlocks)
{
    const int64_t b = (total + each - 1) / each;
    return dim3((unsigned)(b < most ? b : most));
}
dim3 blocks_for(const Deal& d, int64_t most) { return d.segs ? blocks_for(d.units, kBlock / 64, most) : blocks_for(d.total, kBlock, most); }
// A launch of a kernel by how its pieces are dealt out (SEGS, the kernel's last template argument: up to MOST); N == 1: rows of up to seven elements, one after the other
#define FG_LAUNCH_DEAL(MOST, d, most, stream, kernel, ...)                                                                                  \
    do {                                                                                                                              \
        constexpr int fg_4 = N > 1 && MOST >= 4 ? 4 : 0, fg_2 = N > 1 && MOST >= 2 ? 2 : 0, fg_1 = N > 1 ? 1 : 0;                     \
        if (fg_4 && (d).segs == 4) FG_LAUNCH((kernel, fg_4>), blocks_for(d, most), dim3(kBlock), 0, stream, __VA_ARGS__);                   \
        else if (fg_2 && (d).segs == 2) FG_LAUNCH((kernel, fg_2>), blocks_for(d, most), dim3(kBlock), 0, stream, __VA_ARGS__);              \
        else if (fg_1 && (d).segs == 1) FG_LAUNCH((kernel, fg_1>), blocks_for(d, most), dim3(kBlock), 0, stream, __VA_ARGS__);              \
        else FG_LAUNCH((kernel, 0>), blocks_for((d).total, kBlock, most), dim3(kBlock), 0, stream, __VA_ARGS__);                            \
    } while (0)

// ---- lookup ------------------------------------------------------------------------------------------------------------

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

// Calls body(U, first, there) over [0, n): MOST (8, 4 or 2) at a time, the last of a list in one go as MOST, half of it or 1 of which `there` are
// there, so that a short list costs one trip to memory and few loads that nobody asked for.
template <int U> struct Count { static constexpr int value = U; };
template <int MOST, typename Body>
__device__ __forceinline__ void in_chunks(int32_t n, Body&& body)
{
    int32_t at = 0;
#pragma unroll 1
    for (; n - at > MOST / 2; at += MOST) body(Count<MOST>{}, at, n - at < MOST ? n - at : MOST);
    if (MOST > 2 && n - at > 1) body(Count<MOST / 2>{}, at, n - at);
    else if (n - at == 1) body(Count<1>{}, at, 1);
}

// ---- weighted sums -----------------------------------------------------------------------------------------------------

// (n_rows > 0: an entry that names no row reads row 0 and adds zeros in its place, so that no load waits behind a branch)
template <typename T, int N, bool WEIGHTED, bool STREAM, int SEGS>
__global__ __launch_bounds__(kBlock) void k_combine(const T* __restrict__ rows, int64_t rows_stride, uint32_t n_rows, const int32_t* __restrict__ index,
                                                    const float* __restrict__ weights, int32_t k, T* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T, N> P;
    constexpr int S = SEGS ? SEGS : 1;
    each_span<N, SEGS>(d, [&](const Span<S>& at) {
        typename P::Wide sum[S] = {};
        const int64_t base = at.row * k;
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
            if (at.there[s]) store_piece<T, N, STREAM>(out + at.row * out_stride + at.col[s], narrow<T, N>(sum[s]));
    });
}

// ---- gradients of weights, and of rows that are named once -------------------------------------------------------------

// Adds U values (8, 4, 2 or 1) over `lanes` lanes of a wavefront (a power of two from 8 on; the lane's number among them is `lane`): at each of log U steps
// a lane hands half of its values to the lane opposite and takes the other half, then the one that is left is added up.  Returns the sum of value
// share_of<U>(lane, lanes).
template <int U>
__device__ __forceinline__ int share_of(int lane, int lanes) { return lane >> (__builtin_ctz(lanes) - __builtin_ctz(U)); }
template <int U>
__device__ __forceinline__ float add_up(float (&x)[U], int lane, int lanes)
{
    int o = lanes >> 1;
#pragma unroll
    for (int half = U / 2; half > 0; half >>= 1, o >>= 1) {
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

// `lanes` lanes (8 to 32: WAVES == 0; 64, 128 or 256: WAVES wavefronts, which meet in LDS) take a token: they walk along its row and those of up
// to eight of its k, so that the token's gradient is loaded once for the eight.
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

// ---- sums over the entries of a row ------------------------------------------------------------------------------------

// Rows that are named often are summed in parts: `chunk` entries of the sorted index that all name one row, and kChunks such chunks, are summed
// by themselves and put together afterwards, so that what one lane does for a row hardly grows with the row's entries.  chunk is kChunk, or where
// there are rows enough to fill the chip, four times the mean of a row's entries (a power of two): rows of a graph are named often, but all of them.
//   k_row_sums   chunks of one row each, a row's first and last with its entries before and after them: their sums; rows without such a chunk
//   k_row_parts  chunks of chunks (where there are enough entries)
//   k_row_join   rows with a chunk: chunks up to the first whole chunk of chunks, those, and chunks again
// The long rows' entries are read while the many short ones are written.  Few entries and rows: k_row_sums_few alone, a launch instead of two or three.
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
    float scale;
    int32_t shift;           // log2 of chunk
    float *parts, *parts2;   // sums of chunks, and of chunks of chunks (NULL: none)
};

// Adds the entries [from, to) of the sorted index to sum.  DOTS: their products with `row` (the piece of the row that they name) are added up over
// the `lanes` lanes that share it and written as their weights' gradients; `real`: this lane has a piece.
template <typename T, int N, bool WEIGHTED, bool DOTS, int S>
__device__ __forceinline__ void add_entries(typename Piece<T, N>::Wide (&sum)[S], const SumArgs& a, const T* __restrict__ grad, int64_t grad_stride,
                                            int32_t from, int32_t to, const Span<S>& at, const typename Piece<T, N>::Wide& row, bool real, int lanes)
{
    typedef Piece<T, N> P;
    in_chunks<(16 / S < 8 ? 16 / S : 8)>(to - from, [&](auto count, int32_t p, int there) {
        constexpr int U = count.value;
        int32_t entry[U];
        float w[U];
        typename P::Vec v[U][S];
        load_words<U>(a.order + from + p, there, entry);
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
    from = from < 0 ? 0 : from;
    to = to > a.m ? a.m : to;
}
__device__ __forceinline__ int32_t first_chunk(const SumArgs& a, int32_t from) { return (int32_t)(((int64_t)from + (1 << a.shift) - 1) >> a.shift); }

template <typename T, int N, typename TO, bool ACCUMULATE, bool STREAM, int S>
__device__ __forceinline__ void store_sum(const SumArgs& a, typename Piece<T, N>::Wide (&sum)[S], TO* __restrict__ out, int64_t out_stride, int64_t row,
                                          const Span<S>& at)
{
    typedef TO OutVec __attribute__((ext_vector_type(N), aligned(sizeof(TO))));
    typedef typename Piece<T, N>::Wide Wide;
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (!at.there[s] || at.skip[s] >= N) continue;
        TO* p = out + row * out_stride + at.col[s];
        Wide x = sum[s] * a.scale;
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

template <typename T, int N, typename TO, bool WEIGHTED, bool ACCUMULATE, bool DOTS, bool STREAM, int SEGS>
__global__ __launch_bounds__(kBlock, DOTS && sizeof(T) == 2 ? 3 : 4) void k_row_sums(SumArgs a, const int32_t* __restrict__ index, const int32_t* __restrict__ order,
                                                                                     const int32_t* __restrict__ bounds, const float* __restrict__ weights,
                                                                                     const T* __restrict__ grad, int64_t grad_stride,
                                                                                     const T* __restrict__ rows, int64_t rows_stride,
                                                                                     TO* __restrict__ out, int64_t out_stride, Deal d)
{
    typedef Piece<T, N> P;
    constexpr int S = SEGS ? SEGS : 1;
    a.index = index; a.order = order; a.bounds = bounds; a.weights = weights;        // (arguments of their own: nothing stored changes them)
    each_span<N, SEGS>(d, [&](const Span<S>& at) {
        const bool real = !DOTS || at.skip[0] < N;
        if (at.row < a.chunks) {
            const int32_t q = (int32_t)at.row;
            int32_t name;
            if (!one_row(a, q << a.shift, 1 << a.shift, name)) return;
            int32_t from = a.bounds[name], to = a.bounds[name + 1];
            within(a, from, to);
            if (first_chunk(a, from) < q) from = q << a.shift;
            if (to >> a.shift > q + 1) to = (q + 1) << a.shift;
            typename P::Wide sum[S] = {}, row = {};
            if (DOTS) row = wide<T, N>(load_piece<T, N>(rows + (int64_t)name * rows_stride + at.col[0]));
            add_entries<T, N, WEIGHTED, DOTS, S>(sum, a, grad, grad_stride, from, to, at, row, real, (int)d.pieces);
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (real && at.there[s]) *reinterpret_cast<typename P::Wide*>(a.parts + (at.row * d.pieces + at.piece[s]) * N) = sum[s];
            return;
        }
        const int64_t name = at.row - a.chunks;
        int32_t from = a.bounds[name], to = a.bounds[name + 1];
        within(a, from, to);
        if (first_chunk(a, from) < to >> a.shift) return;                  // k_row_join
        if (ACCUMULATE && from >= to) return;
        typename P::Wide sum[S] = {}, row = {};
        if (DOTS && from < to) row = wide<T, N>(load_piece<T, N>(rows + name * rows_stride + at.col[0]));
        add_entries<T, N, WEIGHTED, DOTS, S>(sum, a, grad, grad_stride, from, to, at, row, real, (int)d.pieces);
        store_sum<T, N, TO, ACCUMULATE, STREAM, S>(a, sum, out, out_stride, name, at);
    });
}

// Few entries and rows: a wavefront for 64 pieces of a row; where a row has more than kAlone entries, the workgroup's wavefronts take a share of them each and meet in LDS.
constexpr int kFewBlock = 1024, kAlone = 32;
constexpr int64_t kFewEntries = 8192, kFewUnits = 32768;
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
        add_entries<T, N, WEIGHTED, false, 1>(sum, a, grad, grad_stride, from, to, at, none, true, 0);
        store_sum<T, N, TO, ACCUMULATE, false, 1>(a, sum, out, out_stride, row, at);
    }
    __syncthreads();
    for (int w = 0; w < kW; ++w) {
        const int32_t f = range[w][0], n = range[w][1] - f;
        if (n <= kAlone) continue;
        const int32_t share = (n + kW - 1) / kW, mine = wave * share < n ? wave * share : n, end = mine + share < n ? mine + share : n;
        int64_t of;
        const Span<1> there_at = span(w, of);
        Wide sum[1] = {}, none = {};
        add_entries<T, N, WEIGHTED, false, 1>(sum, a, grad, grad_stride, f + mine, f + end, there_at, none, true, 0);
        part[wave][lane] = sum[0];
        __syncthreads();
        if (wave == w) {
            sum[0] = part[0][lane];
#pragma unroll
            for (int i = 1; i < kW; ++i) sum[0] += part[i][lane];
            store_sum<T, N, TO, ACCUMULATE, false, 1>(a, sum, out, out_stride, row, at);
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
        store_sum<T, N, TO, ACCUMULATE, false, 1>(a, sum, out, out_stride, name, at);
    });
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
    SumArgs b = a;
    if constexpr (!DOTS) {
        Deal d = deal(r.n_rows, r.c, pieces, 1);
        d.waves = (pieces + 63) / 64;                        // a wavefront for 64 pieces whatever the width
        d.by_waves_far = DivideFar(d.waves);
        d.units = r.n_rows * d.waves;
        if (r.m <= kFewEntries && d.units <= kFewUnits) {
            FG_LAUNCH((k_row_sums_few<T, N, TO, WEIGHTED, ACCUMULATE>), blocks_for(d.units, kFewBlock / 64), dim3(kFewBlock), 0, stream, b, b.order, b.bounds,
                      b.weights, grad, r.grad.stride, (TO*)r.out.at, r.out.stride, d);
            return hipSuccess;
        }
    }
    int64_t chunk = kChunk;
    b.shift = 5;
    while (r.n_rows * pieces >= kFill && chunk < 4 * (r.m / r.n_rows) && chunk < 65536) { chunk *= 2; ++b.shift; }
    b.chunks = r.m / chunk;
    b.parts = r.partials;
    b.parts2 = nullptr;
    const Deal d = deal(b.chunks + r.n_rows, r.c, pieces, DOTS ? 1 : 2);
#define FG_SUMS(STREAM) k_row_sums<T, N, TO, WEIGHTED, ACCUMULATE, DOTS, STREAM
#define FG_SUMS_ARGS b, b.index, b.order, b.bounds, b.weights, grad, r.grad.stride, rows, r.rows.stride, (TO*)r.out.at, r.out.stride, d
    const bool past = !ACCUMULATE && !DOTS && (r.n_rows * (int64_t)sizeof(TO) + r.m / r.fan * (int64_t)sizeof(T)) * r.c >= kStream;
    if constexpr (DOTS) FG_LAUNCH_DEAL(1, d, kMostUneven, stream, FG_SUMS(false), FG_SUMS_ARGS);
    else if (!past) FG_LAUNCH_DEAL(2, d, kMostUneven, stream, FG_SUMS(false), FG_SUMS_ARGS);
    else FG_LAUNCH_DEAL(2, d, kMostUneven, stream, FG_SUMS(!ACCUMULATE), FG_SUMS_ARGS);
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

template <typename T, int N>
hipError_t lookup(RowsIn table, int64_t n_rows, int64_t c, const int32_t* index, int64_t m, float scale, RowsOut out, hipStream_t stream)
{
    const Deal d = deal<T, N>(m, c, 2);
#define FG_LOOKUP(STREAM) \
    FG_LAUNCH_DEAL(2, d, kMostBlocks, stream, FG_LOOKUP_OF(STREAM), (const T*)table.at, table.stride, (uint32_t)n_rows, index, scale, (T*)out.at, out.stride, d)
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
    FG_LAUNCH_DEAL(4, d, kMostBlocks, stream, FG_DISPATCH, (const T*)x.at, x.stride, place, k, (uint32_t)n_rows, (T*)out.at, out.stride, d);
#undef FG_DISPATCH
    return hipSuccess;
}

template <typename T, int N>
hipError_t combine(RowsIn rows, int64_t n_rows, int64_t c, const int32_t* index, const float* weights, int64_t t, int32_t k, RowsOut out,
                   hipStream_t stream)
{
    if (n_rows == 0) return lookup<T, N>(rows, 0, c, index, t, 1.0f, out, stream);       // zeros
    const Deal d = deal<T, N>(t, c, 2);
#define FG_COMBINE(WEIGHTED, STREAM) \
    FG_LAUNCH_DEAL(2, d, kMostBlocks, stream, FG_COMBINE_OF(WEIGHTED, STREAM), (const T*)rows.at, rows.stride, (uint32_t)n_rows, index, weights, k, (T*)out.at, out.stride, d)
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
    // a wavefront or less for a token; more, so that a row is one trip to memory, while the chip has room for it
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
    SumArgs a = {};
    a.index = r.index; a.order = r.order; a.bounds = r.bounds; a.weights = r.weights; a.grad_weights = r.grad_weights;
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
