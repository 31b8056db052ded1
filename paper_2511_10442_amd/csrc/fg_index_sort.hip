// Stable order of the entries of an index by the row that they name: order, place (its inverse) and bounds of the rows.
//
// A sort by digits from the lowest: every pass keeps the order that the one before made, so entries of one row stay as they came, and
// sums over them come out the same in every run.  An entry outside 0..n_rows-1 has the key n_rows, behind all rows.  A pass of a tile:
// 64 entries at a time a wavefront finds, with one ballot for every bit of the digit, which lanes have the same digit; the number of
// those before a lane is its rank, their count moves the wavefront's counter of that digit.
//
// A few entries are not sorted but counted: k_sort_few.  Up to 8192 of many rows one workgroup sorts in LDS, all digits in one launch.  Beyond, three
// launches a digit (counts of the tiles, their prefix, the entries to their places; where there are few counts, the last alone after the first digit's counts)
// and one for the bounds: 262144 entries of 64 rows 12 us, 65536 of 131072 31 (latency: a tile's chain of loads, ranks and stores is 5 to 7 us, however few
// there are), 4M of 100k 82, 32M of 1M 720.  A pass over 4M moves 48 to 64 MB in 23 to 26 us: stores of runs of 8 entries.
#include "fg_rows.hpp"

namespace fg {

namespace {

constexpr int kMaxBits = 10;                 // of a digit: a million rows in two passes
constexpr int kSmallBlock = 1024;
// Entries that one workgroup sorts in LDS, where a row has two digits or more.  us a call in this one launch / in the four for more, of 2000, 60000 and 1M
// rows: 4097 entries 14.6 / 16.9, 16.4 / 18.5, 22 / 31; 6000 16.7 / 17.2, 18.6 / 18.7, 24 / 35; 8192 19.6 / 17.6, 21.9 / 18.9, 28 / 35.  Up to 60000 rows they meet
// at some 6000 entries; from there to 8192 the one launch, which needs no workspace, loses 2 to 3 us and gains 7 and more where rows are many.  (With one digit
// two launches are always less: 8192 of 256 rows 14.6 / 7.9.)
constexpr int64_t kSmallM = 8192;
// Entries that are counted, by 4 and by 16 lanes a question, and how many questions (entries and bounds) and looks at a key at most.  us counted by 4 /
// counted by 16 / sorted in LDS: 64 entries of 8 rows 1.7 / 2.1 / 3.0, 300 of 50000 4.2 / 5.3 / 7.0, 100 of 200000 5.5 / 8.6 / 7.9, 1000 of 5003 7.2 / 4.0 / 7.2, 1024 of 20000
// 7.2 / 5.5 / 7.5, 1000 of 60000 7.7 / 8.3 / 7.6, 4096 of 10000 21 / 8.4 / 12.4, of 16000 21 / 12.0 / 12.5.  (8192 of 256 by 16 13.1, in LDS 14.6.)
constexpr int64_t kFewM = 512, kFewQuestions = 1 << 18, kSomeM = 4096, kSomeQuestions = 1 << 15, kSomeLooks = 1 << 26;
// Rows whose bounds a workgroup writes; for more, more workgroups sort the same entries (1000 entries of 5003 rows, before they were
// counted: one workgroup and a search of the bounds in a launch of its own 8.8 us, five 6.6).
constexpr int64_t kSmallRows = 1024, kSmallBlocks = 256;
constexpr int kBlock = 256;
constexpr unsigned kXcds = 8;
// A tile: few entries, so that there are many, up to a million; then runs that are worth storing (4M entries of 100k rows, us, by threads x entries
// of a tile: 256 x 8 101, 256 x 16 108, 512 x 4 96, 512 x 8 84, 512 x 16 101, 1024 x 4 90, 1024 x 8 92).
constexpr int kItems = 4;
constexpr int64_t kMediumM = 1 << 20;
constexpr int kLargeBlock = 512, kLargeItems = 8;
// Tiles and counts of a pass (tiles x digits) up to which every tile adds them up for itself and counts the next pass's digits as it goes, so that the launches
// between two passes are saved (us with them / without, by tiles of as many entries, also where rows follow Zipf's law: 8200 entries of 5000 rows 26 / 19,
// 32768 of 131072 31 / 24, 65536 of 64 11.2 / 8.5, 131072 of 2000 31 / 24; 65536 of 131072, 2^15 counts, 32 / 30; 131072 of 131072, 2^16, 35 / 41;
// 196 tiles, 200000 entries of 8 rows, 11.1 / 8.8, 489, 500000 of 16, 13.5 / 15.2).
constexpr int kJoinedBits = 15;
constexpr int64_t kJoinedCounts = 1 << kJoinedBits, kJoinedTiles = 256;
constexpr int kJoinedBlock = kBlock * kItems;

struct Plan { int bits, passes; bool joined, large; int64_t tiles; };

inline Plan plan_for(int64_t m, int64_t n_rows)
{
    Plan p;
    int bits = 1;
    while (((int64_t)1 << bits) <= n_rows) ++bits;       // keys 0..n_rows
    p.passes = (bits + kMaxBits - 1) / kMaxBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.large = m > kMediumM;
    const int64_t tile = p.large ? kLargeBlock * kLargeItems : kBlock * kItems;
    p.tiles = (m + tile - 1) / tile;
    p.joined = !p.large && p.tiles <= kJoinedTiles && p.tiles << p.bits <= kJoinedCounts;
    return p;
}

inline size_t up(size_t x) { return (x + 255) / 256 * 256; }

struct Layout { size_t counts, totals, key_a, order_a, key_b, order_b, total; };

inline Layout layout_for(int64_t m, const Plan& p)
{
    Layout l;
    const size_t words = up((size_t)m * 4);
    l.counts = 0;
    l.totals = up(((size_t)1 << p.bits) * (size_t)p.tiles * 4) * (p.joined ? p.passes : 1);       // (joined: of every pass)
    l.key_a = l.totals + up(((size_t)1 << p.bits) * 4);
    l.order_a = l.key_a + (p.passes > 1 ? words : 0);
    l.key_b = l.order_a + (p.passes > 1 ? words : 0);
    l.order_b = l.key_b + (p.passes > 1 ? words : 0);
    l.total = l.order_b + (p.passes > 2 ? words : 0);
    return l;
}

inline bool takes_few(int64_t m, int64_t n_rows) { return m <= kFewM && m + n_rows < kFewQuestions; }
inline bool takes_some(int64_t m, int64_t n_rows) { return m <= kSomeM && m + n_rows < kSomeQuestions && m * (m + n_rows) < kSomeLooks; }
inline bool takes_small_sort(int64_t m, const Plan& p) { return m <= kSmallM && p.passes > 1; }

__device__ __forceinline__ uint32_t key_of(int32_t name, uint32_t n_rows) { return (uint32_t)name < n_rows ? (uint32_t)name : n_rows; }

// Lanes of the wavefront whose digit is this lane's.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, bool there)
{
    uint64_t peers = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1u;
        const uint64_t ones = __ballot(one);
        peers &= one ? ones : ~ones;
    }
    return peers;
}

// Rank of this lane's entry among the wavefront's entries of its digit so far, whose counters are moved on.
__device__ __forceinline__ uint32_t rank_in_wave(volatile uint32_t* counter, uint32_t digit, int bits, bool there)
{
    const uint64_t peers = same_digit(digit, bits, there);
    const uint32_t lane = __lane_id();
    const uint32_t before = __popcll(peers & ((1ull << lane) - 1));
    uint32_t rank = 0;
    if (there) rank = counter[digit] + before;
    __builtin_amdgcn_wave_barrier();                     // every lane has read before one of them writes
    if (there && before == 0) counter[digit] = rank + __popcll(peers);
    __builtin_amdgcn_wave_barrier();
    return rank;
}

// Neighbouring tiles are workgroups of one XCD, whose L2 joins what they write next to each other; the grid is a multiple of kXcds.
__device__ __forceinline__ int64_t tile_of_block() { return (int64_t)(blockIdx.x % kXcds) * (gridDim.x / kXcds) + blockIdx.x / kXcds; }

// Exclusive prefix over the block's threads; `sums` has one word for each wavefront.
template <int WAVES, typename W>
__device__ __forceinline__ W block_prefix(W x, W* sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    W run = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const W y = __shfl_up(run, o);
        if (lane >= o) run += y;
    }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    W before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) before += w < wave ? sums[w] : 0;
    __syncthreads();
    return before + run - x;
}

// ---- a few entries, counted ----------------------------------------------------------------------------------------------

// An entry's place is the number of entries before it, a row's bound that of the entries of rows before it: LANES lanes a question look at every key, which has
// the entry's number in its `low` lowest bits (up to 512 entries and 2^18 rows, 4096 and 2^15: 27 bits), in LDS.  No step waits for another but the first load.
constexpr int kFewBlock = 1024;
template <int LANES>
__global__ __launch_bounds__(kFewBlock) void k_sort_few(const int32_t* __restrict__ index, int32_t m, uint32_t n_rows, int low, int32_t* __restrict__ order,
                                                        int32_t* __restrict__ place, int32_t* __restrict__ bounds)
{
    typedef uint32_t Four __attribute__((ext_vector_type(4)));
    extern __shared__ Four fours[];                      // as many as LANES divides
    uint32_t* keys = (uint32_t*)fours;
    const int tid = threadIdx.x, sub = tid % LANES, n = (m + 4 * LANES - 1) / (4 * LANES) * LANES;
    for (int e = tid; e < 4 * n; e += kFewBlock) keys[e] = e < m ? key_of(index[e], n_rows) << low | e : ~0u;
    __syncthreads();
    const int64_t q = (int64_t)blockIdx.x * (kFewBlock / LANES) + tid / LANES;
    if (q > m + (int64_t)n_rows) return;
    const uint32_t what = q < m ? keys[q] : (uint32_t)(q - m) << low;
    uint32_t before = 0;
#pragma unroll 4
    for (int i = sub; i < n; i += LANES) {
        const Four k = fours[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) before += k[j] < what;
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) before += __shfl_xor(before, o);
    if (sub != 0) return;
    if (q >= m) bounds[q - m] = (int32_t)before;
    else {
        order[before] = (int32_t)q;
        if (place) place[q] = what >> low < n_rows ? (int32_t)before : -1;
    }
}

template <int LANES>
hipError_t count_few(const int32_t* index, int64_t m, int64_t n_rows, int32_t* order, int32_t* place, int32_t* bounds, hipStream_t stream)
{
    int low = 0;
    while (((int64_t)1 << low) < m) ++low;
    const int64_t each = kFewBlock / LANES, blocks = (m + n_rows + each) / each;
    const size_t lds = (size_t)(m + 4 * LANES - 1) / (4 * LANES) * (4 * LANES) * sizeof(uint32_t);
    FG_LAUNCH((k_sort_few<LANES>), dim3((unsigned)blocks), dim3(kFewBlock), lds, stream, index, (int32_t)m, (uint32_t)n_rows, low, order, place, bounds);
    return hipSuccess;
}

// ---- one workgroup -----------------------------------------------------------------------------------------------------

// (of a large table every workgroup sorts all entries: the search of its share of the bounds finds them in LDS, and nothing is launched after it)
template <int ITEMS>
__global__ __launch_bounds__(kSmallBlock) void k_sort_small(const int32_t* __restrict__ index, int32_t m, uint32_t n_rows, int bits, int passes,
                                                            int32_t* __restrict__ order, int32_t* __restrict__ place, int32_t* __restrict__ bounds)
{
    constexpr int BLOCK = kSmallBlock, kW = BLOCK / 64;
    static_assert(1 << kMaxBits <= BLOCK, "a lane has one digit at most");
    __shared__ uint32_t keys[ITEMS * BLOCK], from[ITEMS * BLOCK];
    __shared__ uint32_t counter[kW][1 << kMaxBits];
    __shared__ uint32_t sums[kW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int digits = 1 << bits;
    uint32_t key[ITEMS], at[ITEMS];
    // (a wavefront's entries are one run of ITEMS x 64, taken 64 at a time: their order is that of the ranks)
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int e = (wave * ITEMS + i) * 64 + lane;
        at[i] = e;
        key[i] = e < m ? key_of(index[e], n_rows) : 0;
    }
    for (int pass = 0; pass < passes; ++pass) {
        for (int d = lane; d < digits; d += 64) counter[wave][d] = 0;
        __builtin_amdgcn_wave_barrier();
        uint32_t rank[ITEMS];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int e = (wave * ITEMS + i) * 64 + lane;
            rank[i] = rank_in_wave(counter[wave], (key[i] >> (pass * bits)) & (digits - 1), bits, e < m);
        }
        __syncthreads();
        // (a wavefront's counters of one digit are read at once and written at once)
        uint32_t n[kW], count = 0;
#pragma unroll
        for (int w = 0; w < kW; ++w) n[w] = tid < digits ? counter[w][tid] : 0;
#pragma unroll
        for (int w = 0; w < kW; ++w) count += n[w];
        uint32_t start = block_prefix<kW>(count, sums);
        if (tid < digits)
#pragma unroll
            for (int w = 0; w < kW; ++w) {
                counter[w][tid] = start;
                start += n[w];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int e = (wave * ITEMS + i) * 64 + lane;
            if (e < m) {
                const uint32_t to = counter[wave][(key[i] >> (pass * bits)) & (digits - 1)] + rank[i];
                keys[to] = key[i];
                from[to] = at[i];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int e = (wave * ITEMS + i) * 64 + lane;
            if (e < m) {
                key[i] = keys[e];
                at[i] = from[e];
            }
        }
    }
    if (blockIdx.x == 0)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int e = (wave * ITEMS + i) * 64 + lane;
            if (e < m) {
                order[e] = at[i];
                if (place) place[at[i]] = key[i] < n_rows ? e : -1;
            }
        }
    for (int64_t v = (int64_t)blockIdx.x * BLOCK + tid; v <= n_rows; v += (int64_t)gridDim.x * BLOCK) {
        int lo = 0, hi = m;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (keys[mid] < (uint32_t)v) lo = mid + 1; else hi = mid;
        }
        bounds[v] = lo;
    }
}

// bounds[v]: entries whose key is below v.  Fifteen places are looked at a time, which cost one trip to memory.
__global__ __launch_bounds__(kBlock) void k_sort_bounds(const uint32_t* __restrict__ keys, int32_t m, int64_t n_rows, int32_t* __restrict__ bounds)
{
    const int64_t v = (int64_t)blockIdx.x * kBlock + threadIdx.x;
    if (v > n_rows) return;
    constexpr int kWays = 16;
    int64_t lo = 0, hi = m;
    while (lo < hi) {
        const int64_t step = (hi - lo + kWays - 1) / kWays;
        uint32_t key[kWays - 1];
#pragma unroll
        for (int i = 0; i < kWays - 1; ++i) {
            const int64_t at = lo + (i + 1) * step - 1;
            key[i] = keys[at < hi ? at : hi - 1];
        }
        int below = 0;
#pragma unroll
        for (int i = 0; i < kWays - 1; ++i) below += lo + (i + 1) * step - 1 < hi && key[i] < (uint32_t)v;
        lo += below * step;
        if (below < kWays - 1 && hi > lo + step - 1) hi = lo + step - 1;     // (the place looked at behind the last run would be hi itself)
    }
    bounds[v] = (int32_t)lo;
}

// ---- many workgroups, one digit a pass ---------------------------------------------------------------------------------

// JOIN: the counts of a tile lie together, and those of the `later` passes, `later_counts` words on each, which k_sort_scatter makes, begin at zero.
template <int BLOCK, int ITEMS, bool JOIN>
__global__ __launch_bounds__(BLOCK) void k_sort_count(const uint32_t* __restrict__ keys, int64_t m, uint32_t n_rows, int shift, int bits, int64_t tiles,
                                                      uint32_t* __restrict__ counts, int64_t later_counts, int later)
{
    typedef uint32_t Four __attribute__((ext_vector_type(4), aligned(4)));
    __shared__ uint32_t counter[1 << kMaxBits];
    const int digits = 1 << bits;
    const int64_t tile = tile_of_block();
    if (tile >= tiles) return;
    for (int d = threadIdx.x; d < digits; d += BLOCK) counter[d] = 0;
    __syncthreads();
    const int64_t first = tile * (BLOCK * ITEMS);
    auto add = [&](uint32_t key) { atomicAdd(&counter[(key_of((int32_t)key, n_rows) >> shift) & (digits - 1)], 1u); };
    const int64_t end = first + BLOCK * ITEMS < m ? first + BLOCK * ITEMS : m;
    if (ITEMS >= 4 && first + BLOCK * ITEMS <= m) {
        Four v[ITEMS < 4 ? 1 : ITEMS / 4];
#pragma unroll
        for (int i = 0; i < ITEMS / 4; ++i) v[i] = *reinterpret_cast<const Four*>(keys + first + (i * BLOCK + threadIdx.x) * 4);
#pragma unroll
        for (int i = 0; i < ITEMS / 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) add(v[i][j]);
    } else {
        for (int64_t e = first + threadIdx.x; e < end; e += BLOCK) add(keys[e]);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += BLOCK) {
        counts[JOIN ? tile * digits + d : (int64_t)d * tiles + tile] = counter[d];
        if (JOIN)
            for (int p = 1; p <= later; ++p) counts[p * later_counts + tile * digits + d] = 0;
    }
}

// One workgroup a digit: exclusive prefix over the tiles, and the sum.
__global__ __launch_bounds__(kBlock) void k_sort_scan(uint32_t* __restrict__ counts, int64_t tiles, uint32_t* __restrict__ totals)
{
    constexpr int kWaves = kBlock / 64;
    __shared__ uint32_t sums[kWaves];
    __shared__ uint32_t carry;
    uint32_t* row = counts + (int64_t)blockIdx.x * tiles;
    uint32_t before = 0;
    for (int64_t t0 = 0; t0 < tiles; t0 += kBlock) {
        const int64_t t = t0 + threadIdx.x;
        const uint32_t n = t < tiles ? row[t] : 0;
        const uint32_t start = block_prefix<kWaves>(n, sums);
        if (t < tiles) row[t] = before + start;
        if (threadIdx.x == kBlock - 1) carry = start + n;
        __syncthreads();
        before += carry;
        __syncthreads();
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// A tile is put in order in LDS first, so that its entries of one digit leave as one run; runs of neighbouring tiles lie next to each other.  (4M
// entries: every lane storing its own 75 us a pass, runs 38, with more wavefronts a workgroup 25.)
// FIRST: keys are the index itself and entries are numbered as they come.  LAST: place is written, with one pass in all the bounds too.
// JOIN: counts [tile][digit] are added up here, and those of the pass that follows made (`next`).
template <int BLOCK, int ITEMS, bool JOIN>
constexpr size_t scatter_lds(int digits) { return ((size_t)digits * (BLOCK / 64 + (JOIN ? 3 : 1)) + 2 * BLOCK * ITEMS) * 4; }

template <int BLOCK, int ITEMS, bool JOIN, bool FIRST, bool LAST>
__global__ __launch_bounds__(BLOCK) void k_sort_scatter(const uint32_t* __restrict__ keys, const int32_t* __restrict__ from, int64_t m, uint32_t n_rows,
                                                        int shift, int bits, int64_t tiles, const uint32_t* __restrict__ counts,
                                                        const uint32_t* __restrict__ totals, uint32_t* __restrict__ keys_out,
                                                        int32_t* __restrict__ order, int32_t* __restrict__ place, int32_t* __restrict__ bounds,
                                                        uint32_t* __restrict__ next)
{
    constexpr int kTile = BLOCK * ITEMS, kWaves = BLOCK / 64, kOwn = (1 << kMaxBits) / BLOCK;
    extern __shared__ uint32_t lds[];                    // scatter_lds()
    __shared__ uint64_t sums[kWaves];
    const int digits = 1 << bits;
    uint32_t* sorted = lds;
    int32_t* entries = (int32_t*)(lds + kTile);
    uint32_t* away = lds + 2 * kTile;                    // of a digit: from its place in the tile to its place in the order
    uint32_t* counters = away + digits;                  // [wave][digit]
    const int64_t tile = tile_of_block();
    if (tile >= tiles) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t* counter = counters + wave * digits;
    const int64_t first = tile * kTile + wave * (64 * ITEMS);
    uint32_t key[ITEMS], rank[ITEMS];
    int32_t entry[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t e = first + i * 64 + lane;
        key[i] = e < m ? (FIRST ? key_of((int32_t)keys[e], n_rows) : keys[e]) : 0;
        entry[i] = FIRST || e >= m ? (int32_t)e : from[e];
    }
    uint32_t total[kOwn], already[kOwn];                 // of this lane's digits: in the index, in the tiles before
    uint32_t* joined = counters + kWaves * digits;       // JOIN: [digit] total, [digit] already
    if constexpr (JOIN) {
        static_assert(kOwn == 1, "a lane has one digit at most");
        if (tid < digits) joined[tid] = joined[digits + tid] = 0;
        __syncthreads();
        const int groups = BLOCK >> bits, d = tid & (digits - 1);
        uint32_t sum = 0, sum_before = 0;
        for (int t0 = tid >> bits; t0 < tiles; t0 += groups * 8) {
            uint32_t n[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) n[u] = counts[(t0 + u * groups < tiles ? t0 + u * groups : 0) * digits + d];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                sum += t0 + u * groups < tiles ? n[u] : 0;
                sum_before += t0 + u * groups < tile ? n[u] : 0;
            }
        }
        if (sum) atomicAdd(&joined[d], sum);
        if (sum_before) atomicAdd(&joined[digits + d], sum_before);
    } else {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int d = i * BLOCK + tid;
            total[i] = d < digits ? totals[d] : 0;
            already[i] = d < digits ? counts[(int64_t)d * tiles + tile] : 0;
        }
    }
    for (int d = lane; d < digits; d += 64) counter[d] = 0;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        rank[i] = rank_in_wave(counter, (key[i] >> shift) & (digits - 1), bits, first + i * 64 + lane < m);
    __syncthreads();
    if constexpr (JOIN) {
        total[0] = tid < digits ? joined[tid] : 0;
        already[0] = tid < digits ? joined[digits + tid] : 0;
    }
    uint64_t before = 0;                                 // of the whole order in the upper half, of the tile in the lower
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
        if (i * BLOCK >= digits) break;
        const int d = i * BLOCK + tid;
        uint32_t here = 0;
        if (d < digits)
            for (int w = 0; w < kWaves; ++w) here += counters[w * digits + d];
        const uint64_t both = (uint64_t)total[i] << 32 | here;
        const uint64_t start = before + block_prefix<kWaves>(both, sums);
        if (d < digits) {
            const uint32_t all = (uint32_t)(start >> 32);
            uint32_t to = (uint32_t)start;
            if (bounds && tile == 0 && d <= (int64_t)n_rows) bounds[d] = (int32_t)all;
            away[d] = all + already[i] - to;
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t n = counters[w * digits + d];
                counters[w * digits + d] = to;
                to += n;
            }
        }
        if (tid == BLOCK - 1) sums[0] = start + both;
        __syncthreads();
        before = sums[0];
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (first + i * 64 + lane < m) {
            const uint32_t to = counter[(key[i] >> shift) & (digits - 1)] + rank[i];
            sorted[to] = key[i];
            entries[to] = entry[i];
        }
    __syncthreads();
    const int64_t left = m - tile * kTile;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int p = i * BLOCK + tid;
        if (p < left) {
            const uint32_t k = sorted[p], to = away[(k >> shift) & (digits - 1)] + p;
            order[to] = entries[p];
            if (keys_out) keys_out[to] = k;
            if (LAST && place) place[entries[p]] = k < n_rows ? (int32_t)to : -1;
            if (JOIN && !LAST) {
                // (one addition for the entries of a wavefront that are counted together: those of a row that is named often)
                const uint32_t at = (to / kTile) * digits + ((k >> (shift + bits)) & (digits - 1));
                const uint64_t peers = same_digit(at, kJoinedBits, true);
                if ((peers & ((1ull << lane) - 1)) == 0) atomicAdd(&next[at], (uint32_t)__popcll(peers));
            }
        }
    }
}

template <int BLOCK, int ITEMS, bool JOIN, bool FIRST, bool LAST, typename... Args>
hipError_t scatter(unsigned blocks, int bits, hipStream_t stream, Args... args)
{
    const size_t lds = scatter_lds<BLOCK, ITEMS, JOIN>(1 << bits);
    // (beyond 64 KiB a kernel has to be told)
    if (lds > 65536)
        FG_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(&k_sort_scatter<BLOCK, ITEMS, JOIN, FIRST, LAST>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    FG_LAUNCH((k_sort_scatter<BLOCK, ITEMS, JOIN, FIRST, LAST>), dim3(blocks), dim3(BLOCK), lds, stream, args...);
    return hipSuccess;
}

template <int BLOCK, int ITEMS, bool JOIN>
hipError_t many(const int32_t* index, int64_t m, int64_t n_rows, const Plan& p, int32_t* order, int32_t* place, int32_t* bounds, char* ws,
                hipStream_t stream)
{
    const Layout l = layout_for(m, p);
    uint32_t *counts = (uint32_t*)(ws + l.counts), *totals = (uint32_t*)(ws + l.totals);
    uint32_t* key_to[2] = {(uint32_t*)(ws + l.key_a), (uint32_t*)(ws + l.key_b)};
    int32_t* order_to[2] = {(int32_t*)(ws + l.order_a), (int32_t*)(ws + l.order_b)};
    const uint32_t* keys = (const uint32_t*)index;
    const int32_t* from = nullptr;
    const unsigned spread = (unsigned)((p.tiles + kXcds - 1) / kXcds * kXcds);
    const int64_t later_counts = (int64_t)(l.totals / p.passes / sizeof(uint32_t));      // (joined)
    for (int pass = 0; pass < p.passes; ++pass) {
        const bool first = pass == 0, last = pass == p.passes - 1;
        const int shift = pass * p.bits;
        uint32_t* keys_out = p.passes > 1 ? key_to[pass & 1] : nullptr;
        int32_t* out = last ? order : order_to[pass & 1];
        int32_t* starts = p.passes == 1 ? bounds : nullptr;
        if (first || !JOIN)
            FG_LAUNCH((k_sort_count<BLOCK, ITEMS, JOIN>), dim3(spread), dim3(BLOCK), 0, stream, keys, m, (uint32_t)n_rows, shift, p.bits, p.tiles, counts,
                      later_counts, p.passes - 1);
        if (!JOIN) FG_LAUNCH(k_sort_scan, dim3(1u << p.bits), dim3(kBlock), 0, stream, counts, p.tiles, totals);
#define FG_SCATTER(FIRST, LAST)                                                                                                          \
    FG_TRY((scatter<BLOCK, ITEMS, JOIN, FIRST, LAST>(spread, p.bits, stream, keys, from, m, (uint32_t)n_rows, shift, p.bits, p.tiles,    \
                                                     (const uint32_t*)counts, (const uint32_t*)totals, keys_out, out, place, starts,     \
                                                     JOIN ? counts + later_counts : nullptr)))
        if (first && last) FG_SCATTER(true, true);
        else if (first) FG_SCATTER(true, false);
        else if (last) FG_SCATTER(false, true);
        else FG_SCATTER(false, false);
#undef FG_SCATTER
        keys = keys_out;
        from = out;
        if (JOIN) counts += later_counts;
    }
    if (p.passes > 1)
        FG_LAUNCH(k_sort_bounds, dim3((unsigned)(n_rows / kBlock + 1)), dim3(kBlock), 0, stream, keys, (int32_t)m, n_rows, bounds);
    return hipSuccess;
}

template <int ITEMS>
hipError_t small(const int32_t* index, int64_t m, int64_t n_rows, const Plan& p, int32_t* order, int32_t* place, int32_t* bounds, hipStream_t stream)
{
    const int64_t blocks = (n_rows + kSmallRows) / kSmallRows;
    FG_LAUNCH((k_sort_small<ITEMS>), dim3((unsigned)(blocks < kSmallBlocks ? blocks : kSmallBlocks)), dim3(kSmallBlock), 0, stream, index, (int32_t)m,
              (uint32_t)n_rows, p.bits, p.passes, order, place, bounds);
    return hipSuccess;
}

}  // namespace

size_t index_sort_workspace_bytes(int64_t m, int64_t n_rows)
{
    const Plan p = plan_for(m, n_rows);
    return takes_few(m, n_rows) || takes_some(m, n_rows) || takes_small_sort(m, p) ? 0 : layout_for(m, p).total;
}

hipError_t launch_index_sort(const int32_t* index, int64_t m, int64_t n_rows, int32_t* order, int32_t* place, int32_t* bounds, void* workspace,
                             hipStream_t stream)
{
    const Plan p = plan_for(m, n_rows);
    if (takes_few(m, n_rows)) return count_few<4>(index, m, n_rows, order, place, bounds, stream);
    if (takes_some(m, n_rows)) return count_few<16>(index, m, n_rows, order, place, bounds, stream);
    if (takes_small_sort(m, p)) {
        if (m <= kSmallBlock) return small<1>(index, m, n_rows, p, order, place, bounds, stream);
        if (m <= 4 * kSmallBlock) return small<4>(index, m, n_rows, p, order, place, bounds, stream);
        return small<8>(index, m, n_rows, p, order, place, bounds, stream);
    }
    if (p.joined) return many<kJoinedBlock, 1, true>(index, m, n_rows, p, order, place, bounds, (char*)workspace, stream);
    if (!p.large) return many<kBlock, kItems, false>(index, m, n_rows, p, order, place, bounds, (char*)workspace, stream);
    return many<kLargeBlock, kLargeItems, false>(index, m, n_rows, p, order, place, bounds, (char*)workspace, stream);
}

}  // namespace fg
