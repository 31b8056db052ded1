// How rows are read, dealt out and written by the kernels that work on them (lookups, expert order, weighted sums, sums by index).
//
// All of them move rows; none computes enough to matter.  A lane handles 16 bytes of a row at a time, whatever the row's alignment (global loads
// and stores of 16 bytes need that of an element only).  A row that is no multiple of 16 bytes ends with a piece that begins before its turn
// and covers some elements twice, with the same values; rows shorter than 16 bytes go element by element.
//
// Rates to compare with, of this card: a copy of 4 GiB 4.8 TB/s, filling 1 GiB 6.9 TB/s, reading 1 GiB 6.0 TB/s.  The kernels below move what they
// cannot do without at 5 to 6.5 TB/s from 1 KiB a row on (200 MB each way), at 4 to 5 TB/s down to 64 bytes, below that at what random
// accesses to less than a line cost.
#pragma once
#include "fg_rows.hpp"

namespace fg {

namespace {

constexpr int kBlock = 256;
constexpr int64_t kFill = 256 * 2048;        // lanes that the chip holds at a time
// Eight workgroups for every place on the chip; more work than that: they take several turns.  Where pieces differ in what they take, a workgroup that is
// done makes room for the next instead (64k tokens' gradient, the commonest 4000 times: 313 us in turns, 300 so).
constexpr int64_t kMostBlocks = 1 << 14, kMostUneven = 1 << 20;
// Times that a row is named, on average, from which on rows are expected to be found in an XCD's L2 by those that name them too (by_xcd)
constexpr int64_t kShared = 4;
constexpr int64_t kFewWaves = 256 * 16;      // half of the wavefronts that the chip holds
// Bytes that a call moves, twice the last-level cache, from which on most of its output has left that cache when the call ends: it is stored past the
// caches (64k rows of 4 KiB looked up 75 -> 61 us; 32k sums of 8 rows of 4 KiB 236 -> 224, with the rows' loads 209; a gradient of 1 GiB 319 -> 297).
// Below, a kernel that reads the output next would pay for it (lookup and reader of 64 to 192 MB: 7 % slower).
constexpr int64_t kStream = 512 << 20;

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
// row.  Or, where a row's pieces fill wavefronts to three quarters at least, a wavefront for SEGS x 64 pieces of one row, so that what goes by the row
// (index, bounds, addresses, branches) is the scalar unit's and a wavefront moves enough to be worth its start.  SEGS measured, in us, for 1, 2, 4:
// 64k rows of 4 KiB looked up 65, 61, 70; 32k rows to 8 places 243, 244, 239; 32k sums of 8 rows 230, 224 (4: too many registers);
// a gradient of 131072 x 2048 float32 from 64k tokens 355, 297, 300, of 131072 x 4096 bf16 from 20k 200, 157, 200.
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
// SEGS == 0: one after the other.  `block` of `blocks` has a share.
template <int N, int SEGS, typename Body>
__device__ __forceinline__ void each_span(const Deal& d, int64_t block, int64_t blocks, Body&& body)
{
    if constexpr (SEGS > 0) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        for (int64_t unit = block * (kBlock / 64) + wave; unit < d.units; unit += blocks * (kBlock / 64)) {
            const int64_t row = d.by_waves_far(unit);
            body(span_of<N, SEGS>(d, row, (uint32_t)(unit - row * d.waves) * (64 * SEGS) + lane));
        }
    } else {
        for (int64_t first = block * kBlock; first < d.total; first += blocks * kBlock) {
            const int64_t row0 = d.by_pieces_far(first);
            const uint32_t x = (uint32_t)(first - row0 * d.pieces) + threadIdx.x, q = d.by_pieces(x);
            if (first + threadIdx.x < d.total) body(span_of<N, 1>(d, row0 + q, x - q * d.pieces));
        }
    }
}
template <int N, int SEGS, typename Body>
__device__ __forceinline__ void each_span(const Deal& d, Body&& body)
{
    each_span<N, SEGS>(d, (int64_t)blockIdx.x, (int64_t)gridDim.x, body);
}
// Workgroups go to the XCDs in turn; so counted, each XCD has one run of them, and rows that are near in the order meet in its L2.  blocks: a multiple of kXcds.
constexpr int64_t kXcds = 8;
__device__ __forceinline__ int64_t by_xcd(int64_t block, int64_t blocks) { return block % kXcds * (blocks / kXcds) + block / kXcds; }

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
unsigned to_xcds(dim3 grid) { return (unsigned)((grid.x + kXcds - 1) / kXcds * kXcds); }
dim3 blocks_for(const Deal& d, int64_t most) { return d.segs ? blocks_for(d.units, kBlock / 64, most) : blocks_for(d.total, kBlock, most); }
// A launch of a kernel by how its pieces are dealt out (SEGS, the kernel's last template argument: up to MOST); N == 1: rows of up to seven elements,
// one after the other
#define FG_LAUNCH_DEAL(MOST, d, grid, stream, kernel, ...)                                                              \
    do {                                                                                                                \
        constexpr int fg_4 = N > 1 && MOST >= 4 ? 4 : 0, fg_2 = N > 1 && MOST >= 2 ? 2 : 0, fg_1 = N > 1 ? 1 : 0;       \
        if (fg_4 && (d).segs == 4) FG_LAUNCH((kernel, fg_4>), dim3(grid), dim3(kBlock), 0, stream, __VA_ARGS__);        \
        else if (fg_2 && (d).segs == 2) FG_LAUNCH((kernel, fg_2>), dim3(grid), dim3(kBlock), 0, stream, __VA_ARGS__);   \
        else if (fg_1 && (d).segs == 1) FG_LAUNCH((kernel, fg_1>), dim3(grid), dim3(kBlock), 0, stream, __VA_ARGS__);   \
        else FG_LAUNCH((kernel, 0>), dim3(grid), dim3(kBlock), 0, stream, __VA_ARGS__);                                 \
    } while (0)

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

// ---- lanes that meet ---------------------------------------------------------------------------------------------------

// lanes that take a row's pieces where they have to meet: a power of two from 8 on
inline uint32_t lanes_for(int64_t pieces)
{
    uint32_t lanes = 8;
    while (lanes < pieces) lanes *= 2;
    return lanes;
}

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

}  // namespace fg
