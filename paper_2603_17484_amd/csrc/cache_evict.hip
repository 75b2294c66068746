// Eviction from a paged KV cache: of the first `rows` rows of a sequence every KV head keeps the `keep` of greatest weight (of equal ones
// the first; NaN is less than everything).  Kept rows before row `keep` stay where they are; the i-th row that leaves before it is the
// place of the i-th kept row behind it.  As many leave before as are kept behind, no place is read and written both, and so the moves are
// independent of one another, in place, and no more bytes move than have to.  The order of rows does not matter to the attention over them:
// their positions are in the keys.
//
// Which rows stay is a radix selection over the weights' bits, ordered as whole numbers: the histogram of their highest bits says in which bin
// the last row that stays lies, that of the bits below among the rows of this bin where in it, and so on.  Then the lists: places that become free, and
// rows that move there, both ascending.
//   evict_select_kernel  up to 8192 rows: a workgroup per KV head of a sequence, the weights in its registers, 11, 11 and 10 bits; where there are
//                        many, it makes the moves too
//   evict_first_kernel, evict_second_kernel, evict_list_kernel
//                        more: a workgroup per 8192 rows (or 1/64).  The first leaves the histogram of its rows' highest 11 bits; each of the second adds up
//                        those of its KV head and lists its rows in the bin found; each of the third takes all of these into shared memory,
//                        so that it knows by itself which rows stay and what comes before its own on the lists (no atomics on memory, nothing to clear)
//   evict_move_kernel    the moves: K, V, exponents, weights
//
// Selection is bound by chains of launches and of dependent loads, moves by their bytes.  Half of 114688 rows of 4 KV heads in bf16 (120 MB) 61 us: 7, 9 and 15 of
// selection, 28 of moves (4.2 TB/s; a copy of 4 GiB: 4.8).  A quarter of 1792 to 3584 rows of 32 x 8 KV heads in e4m3 (74 MB) 33.
#include "paged.hpp"

namespace l2a {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kFewThreads = 256;                 // of up to 2048 rows each of many pairs
constexpr int kPer = 8;                          // rows of a thread
constexpr int kBlock = kSelectThreads * kPer;
constexpr int kMostSegments = 64;                // workgroups of a KV head of a sequence
constexpr int kBins = 2 * kSelectThreads;        // 11 bits; the last 10 leave half of them empty
// Rows of a bin in shared memory.  A bin is a quarter of a power of two: half of 114688 log-normal weights (a tenth of them zero) with sigma 2, 1 and 0.5 leave 3300, 6200 and 10900 rows in
// it.  Where they
// do not fit, the last kernel goes through their list in memory three times, us of selection for these 33, 34 and 37, for 262144 rows 43, 43 and 49, for 2^20 75, 87 and 105.  What takes
// long are equal weights at the border, whose counts are one word: all zero 252, 529 and 2030.
constexpr int kCandidates = 6144;

struct Counts {
    int bin, left;     // the bin of the first bits in which the last row that stays lies, and the how-manieth in it that is
    int listed;        // rows of the segment in it
    int greater[2];    // rows that stay for their first bits, before the keep-th row and behind
};

struct EvictArgs {
    Geom gm;
    Pages c;
    const int32_t *rows, *keep;
    int max_rows;
    const float* weight_in;
    float* weight;
    int32_t* kept;    // [B, Hkv, max_rows], optional
    // workspace
    int32_t* moves;   // [B * Hkv]: how many
    int32_t *to, *from;  // [B * Hkv][max_rows / 2]
    // of calls with more than kBlock rows
    int segments, segment;  // of a KV head of a sequence; rows of each, whole blocks
    int stride;       // of keys: segments x segment
    uint32_t* keys;   // [B * Hkv][stride] order of the weights
    int32_t* bins;    // [B * Hkv][segments][kBins]
    Counts* counts;   // [B * Hkv][segments]
    u32x2* listed;    // [B * Hkv][stride] a segment's rows in the bin of the first bits: order, row
};

__device__ __forceinline__ int rows_of(const EvictArgs& a, int b) { return plan::clamp(a.rows[b], 0, min(a.max_rows, a.c.capacity())); }
// Whole numbers in the order of the weights.  Zeros are alike, NaN comes first.
__device__ __forceinline__ uint32_t order(float w) {
    const uint32_t x = __float_as_uint(w + 0.f);
    if (w != w) return 0u;
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}
__device__ __forceinline__ int page_at(const EvictArgs& a, int b, int row) { return a.c.table[(size_t)b * a.c.max_pages + (row >> a.c.page_log2)]; }

struct Sizes {
    int pair, b, hk, n, m;
};
__device__ __forceinline__ Sizes sizes_of(const EvictArgs& a, int pair) {
    Sizes z;
    z.pair = pair, z.b = pair / a.gm.Hkv, z.hk = pair - z.b * a.gm.Hkv;
    z.n = rows_of(a, z.b), z.m = plan::clamp(a.keep[z.b], 0, z.n);
    return z;
}
// The pair's lists in the workspace.
__device__ __forceinline__ int32_t* to_of(const EvictArgs& a, const Sizes& z) { return a.to + (size_t)z.pair * (a.max_rows / 2); }
__device__ __forceinline__ int32_t* from_of(const EvictArgs& a, const Sizes& z) { return a.from + (size_t)z.pair * (a.max_rows / 2); }
// Row i0 + T j + thread of a block (of T threads) as order; 0 past the end.  Where the weights do not stay in place, those before the keep-th go to theirs (the moves
// write over those that leave).  page_of(row): its page.
template <int T, typename Page>
__device__ __forceinline__ void load_block(const EvictArgs& a, const Sizes& z, int i0, uint32_t (&x)[kPer], Page&& page_of) {
    float w[kPer];
    size_t row[kPer];
    bool real[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * T + (int)threadIdx.x, page = i < z.n ? page_of(i) : 0;
        real[j] = (unsigned)page < (unsigned)a.c.pages;
        row[j] = pool_row(a.c, a.gm.Hkv, plan::clamp(page, 0, a.c.pages - 1), z.hk, i);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) w[j] = i0 + j * T + (int)threadIdx.x < z.n ? a.weight_in[row[j]] : 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * T + (int)threadIdx.x;
        x[j] = i < z.n ? order(w[j]) : 0u;
        if (a.weight != a.weight_in && i < z.m && real[j]) a.weight[row[j]] = w[j];
    }
}
// The same of a block whose order was left in memory (segments are whole blocks).
template <int T>
__device__ __forceinline__ void load_keys(const EvictArgs& a, const Sizes& z, int i0, uint32_t (&x)[kPer]) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = a.keys[(size_t)z.pair * a.stride + i0 + j * T + (int)threadIdx.x];
}

template <int T>
struct Shared {
    int sums[T / 64], chosen[2], counts[2][kPer][T / 64];
};
// Bins from the highest number down, EACH a thread in the order of threads; mine: how many rows this thread's have, `highest` its first.  The bin in
// which the left-th row lies, and the how-manieth in it that is.  (Before it is called again there has to be a barrier.)
template <int EACH, int T>
__device__ __forceinline__ void choose(Shared<T>& sh, const int (&mine)[EACH], int highest, int& bin, int& left) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) sum += mine[e];
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int below = __shfl_up(upto, o);
        if (lane >= o) upto += below;
    }
    if (lane == 63) sh.sums[wave] = upto;
    __syncthreads();
    int before = upto - sum;
#pragma unroll
    for (int w = 0; w < T / 64; ++w)
        if (w < wave) before += sh.sums[w];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        if (before < left && left <= before + mine[e]) sh.chosen[0] = highest - e, sh.chosen[1] = left - before;
        before += mine[e];
    }
    __syncthreads();
    bin = sh.chosen[0], left = sh.chosen[1];
}
// Places of flags among all of a block, in the order of rows: of this thread's j-th, how many lie before it; and how many there are.  Two kinds of flags
// at once, the second's numbers in the upper halves (a block has fewer than 2^16 rows).  turn: 0 and 1 by turns.
template <int T>
__device__ __forceinline__ int places(Shared<T>& sh, int turn, const bool (&flag)[kPer], const bool (&other)[kPer], int (&at)[kPer]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned long long before = (1ull << lane) - 1ull;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const unsigned long long set = __ballot(flag[j]), more = __ballot(other[j]);
        at[j] = __popcll(set & before) + (__popcll(more & before) << 16);
        if (lane == 0) sh.counts[turn][j][wave] = __popcll(set) + (__popcll(more) << 16);
    }
    __syncthreads();
    // every wavefront adds up all counts: a lane those of two
    constexpr int kWavesOf = T / 64, kCounts = kPer * kWavesOf;
    static_assert(kCounts <= 128, "two counts a lane");
    const int* const counts = &sh.counts[turn][0][0];
    const int c0 = 2 * lane < kCounts ? counts[2 * lane] : 0, c1 = 2 * lane < kCounts ? counts[2 * lane + 1] : 0;
    int upto = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int below = __shfl_up(upto, o);
        if (lane >= o) upto += below;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = j * kWavesOf + wave;
        at[j] += __shfl(upto - c0 - c1, i >> 1) + (i & 1 ? __shfl(c0, i >> 1) : 0);
    }
    return __shfl(upto, 63);
}
// What the rows of a block before it had: equal ones, places that become free, rows that move.
struct Before {
    int equal, holes, movers;
};
// The lists of a block, its rows x in registers: all greater than `found` stay, and the first `left` of those equal to it.
template <int T, typename Index>
__device__ __forceinline__ void list_block(const EvictArgs& a, Shared<T>& sh, const Sizes& z, int i0, const uint32_t (&x)[kPer], uint32_t found, int left, Before& past,
                                           Index* to, Index* from) {
    int32_t* const kept = a.kept ? a.kept + (size_t)z.pair * a.max_rows : nullptr;
    bool flag[kPer], other[kPer], stays[kPer];
    int at[kPer];
    const bool all = z.m == z.n;
#pragma unroll
    for (int j = 0; j < kPer; ++j) flag[j] = !all && x[j] == found && i0 + j * T + (int)threadIdx.x < z.n, other[j] = false;
    const int equal = places(sh, 0, flag, other, at);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * T + (int)threadIdx.x;
        stays[j] = i < z.n && (all || x[j] > found || (flag[j] && past.equal + at[j] < left));
        flag[j] = i < z.m && !stays[j], other[j] = i >= z.m && stays[j];
    }
    const int both = places(sh, 1, flag, other, at), holes = both & 0xffff, movers = both >> 16;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * T + (int)threadIdx.x;
        if (flag[j]) to[past.holes + (at[j] & 0xffff)] = (Index)i;
        if (other[j]) from[past.movers + (at[j] >> 16)] = (Index)i;
        if (kept && i < z.m && stays[j]) kept[i] = i;
    }
    past = Before{past.equal + equal, past.holes + holes, past.movers + movers};
}

// The moves of a pair, from the first-th group of lanes' on: a group per move, 16 bytes a lane, K's and V's beside one another; kAhead moves of a
// group on their way together.
constexpr int kAhead = 4;
template <int BITS, typename Index, typename Page>
__device__ __forceinline__ void move_rows(const EvictArgs& a, const Sizes& z, int count, int first, int groups, const Index* to_list, const Index* from_list, Page&& page_of) {
    constexpr int kLanes = 2 * BITS, kRowBytes = kD * BITS / 8;
    const int lane = threadIdx.x % kLanes, c = lane % (kLanes / 2);
    char* const pool = (lane < kLanes / 2 ? a.c.k : a.c.v) + c * 16;
    unsigned char* const scales = lane < kLanes / 2 ? a.c.ks : a.c.vs;
    for (int i0 = first * kAhead; i0 < count; i0 += groups * kAhead) {
        int to[kAhead], from[kAhead];
        size_t dst[kAhead], src[kAhead];
        bool on[kAhead];
        u32x4 x[kAhead];
        uint32_t e[kAhead];
        float w[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) to[j] = to_list[min(i0 + j, count - 1)], from[j] = from_list[min(i0 + j, count - 1)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int p = page_of(to[j]), q = page_of(from[j]);
            on[j] = i0 + j < count && (unsigned)p < (unsigned)a.c.pages && (unsigned)q < (unsigned)a.c.pages;  // page numbers outside the pool are never followed
            dst[j] = on[j] ? pool_row(a.c, a.gm.Hkv, p, z.hk, to[j]) : 0, src[j] = on[j] ? pool_row(a.c, a.gm.Hkv, q, z.hk, from[j]) : 0;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (on[j]) {
                x[j] = *reinterpret_cast<const u32x4*>(pool + src[j] * kRowBytes);
                if (BITS < 16 && c == 0) e[j] = *reinterpret_cast<const uint32_t*>(scales + src[j] * kRowScales);
                if (lane == 1) w[j] = a.weight_in[src[j]];
            }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (on[j]) {
                *reinterpret_cast<u32x4*>(pool + dst[j] * kRowBytes) = x[j];
                if (BITS < 16 && c == 0) *reinterpret_cast<uint32_t*>(scales + dst[j] * kRowScales) = e[j];
                if (lane == 1) a.weight[dst[j]] = w[j];
            }
            if (lane == 2 && a.kept && i0 + j < count) a.kept[(size_t)z.pair * a.max_rows + to[j]] = from[j];
        }
    }
}
template <int BITS>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(EvictArgs a) {
    constexpr int kGroups = kThreads / (2 * BITS);
    const Sizes z = sizes_of(a, blockIdx.y);
    move_rows<BITS>(a, z, a.moves[z.pair], blockIdx.x * kGroups + (int)threadIdx.x / (2 * BITS), gridDim.x * kGroups, to_of(a, z), from_of(a, z),
                    [&](int row) { return page_at(a, z.b, row); });
}

// MOVE: BITS of the elements, or 0: the moves are another kernel's.  Page numbers, and where it makes the moves its lists, stay in shared memory: nothing it
// moves waits for more than its own row.
template <int MOVE, int T>
__global__ __launch_bounds__(T) void evict_select_kernel(EvictArgs a) {
    constexpr int kPages = T * kPer / 16, kList = MOVE ? T * kPer / 2 : 1;
    __shared__ Shared<T> sh;
    __shared__ int bins[kBins], pages[kPages];
    __shared__ uint16_t to[kList], from[kList];
    const Sizes z = sizes_of(a, blockIdx.x);
    for (int i = threadIdx.x; i < kBins; i += T) bins[i] = 0;
    for (int i = threadIdx.x; i < min(kPages, a.c.max_pages); i += T) pages[i] = a.c.table[(size_t)z.b * a.c.max_pages + i];
    auto page_of = [&](int row) { return pages[row >> a.c.page_log2]; };
    if (z.m == 0) {
        if (threadIdx.x == 0) a.moves[z.pair] = 0;
        return;
    }
    __syncthreads();
    uint32_t x[kPer], found = 0;
    load_block<T>(a, z, 0, x, page_of);
    int left = z.m;
    constexpr int kEach = kBins / T;  // bins of a thread
    const int highest = kBins - 1 - kEach * (int)threadIdx.x;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        if (z.m == z.n) break;
        constexpr int kShift[3] = {21, 10, 0};
        const int shift = kShift[pass], above = pass ? kShift[pass - 1] : 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (j * T + (int)threadIdx.x < z.n && (pass == 0 || (x[j] >> above) == (found >> above))) atomicAdd(&bins[(x[j] >> shift) & (pass == 2 ? kBins / 2 - 1 : kBins - 1)], 1);
        __syncthreads();
        int mine[kEach], bin;
#pragma unroll
        for (int e = 0; e < kEach; ++e) mine[e] = bins[highest - e], bins[highest - e] = 0;  // (for the next pass)
        choose(sh, mine, highest, bin, left);
        found |= (uint32_t)bin << shift;
    }
    Before past{0, 0, 0};
    if constexpr (MOVE) {
        list_block(a, sh, z, 0, x, found, left, past, to, from);
        __syncthreads();  // (the lists, and weights that did not stay in place)
        move_rows<MOVE>(a, z, past.holes, threadIdx.x / (2 * MOVE), T / (2 * MOVE), to, from, page_of);
    } else {
        list_block(a, sh, z, 0, x, found, left, past, to_of(a, z), from_of(a, z));
        if (threadIdx.x == 0) a.moves[z.pair] = past.holes;
    }
}

// The workgroup's segment of its pair: rows i0 .. i1 - 1.
struct Segment {
    int i0, i1;
};
__device__ __forceinline__ Segment segment_of(const EvictArgs& a, const Sizes& z) {
    const long long i0 = (long long)blockIdx.x * a.segment;
    return Segment{i0 < z.n ? (int)i0 : z.n, i0 + a.segment < z.n ? (int)(i0 + a.segment) : z.n};
}

__global__ __launch_bounds__(kSelectThreads) void evict_first_kernel(EvictArgs a) {
    __shared__ int bins[kBins];
    const Sizes z = sizes_of(a, blockIdx.y);
    const Segment g = segment_of(a, z);
    if (g.i0 >= g.i1) return;
    for (int i = threadIdx.x; i < kBins; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i0 = g.i0; i0 < g.i1; i0 += kBlock) {
        uint32_t x[kPer];
        load_block<kSelectThreads>(a, z, i0, x, [&](int row) { return page_at(a, z.b, row); });
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int i = i0 + j * kSelectThreads + (int)threadIdx.x;
            a.keys[(size_t)z.pair * a.stride + i] = x[j];  // (a segment is whole blocks)
            if (i < z.n) atomicAdd(&bins[x[j] >> 21], 1);
        }
    }
    __syncthreads();
    int32_t* const out = a.bins + ((size_t)z.pair * a.segments + blockIdx.x) * kBins;
    for (int i = threadIdx.x; i < kBins; i += kSelectThreads) out[i] = bins[i];
}

__global__ __launch_bounds__(kSelectThreads) void evict_second_kernel(EvictArgs a) {
    __shared__ Shared<kSelectThreads> sh;
    __shared__ int count, greater[2];
    const Sizes z = sizes_of(a, blockIdx.y);
    const Segment g = segment_of(a, z);
    if (g.i0 >= g.i1 || z.m == 0 || z.m == z.n) return;
    if (threadIdx.x == 0) count = greater[0] = greater[1] = 0;
    const int highest = kBins - 1 - 2 * (int)threadIdx.x, of = (z.n + a.segment - 1) / a.segment;
    int sums[2] = {0, 0}, bin, left = z.m, mine[2] = {0, 0};
#pragma unroll 8
    for (int s = 0; s < of; ++s) {
        const int32_t* const p = a.bins + ((size_t)z.pair * a.segments + s) * kBins;
        sums[0] += p[highest], sums[1] += p[highest - 1];
    }
    choose(sh, sums, highest, bin, left);
    u32x2* const listed = a.listed + (size_t)z.pair * a.stride + g.i0;
    const int lane = threadIdx.x & 63;
    for (int i0 = g.i0; i0 < g.i1; i0 += kBlock) {
        uint32_t x[kPer];
        load_keys<kSelectThreads>(a, z, i0, x);
        unsigned long long set[kPer];
        int all = 0, at = 0;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int i = i0 + j * kSelectThreads + (int)threadIdx.x;
            const bool more = i < z.n && (int)(x[j] >> 21) > bin;
            mine[0] += more && i < z.m, mine[1] += more && i >= z.m;
            set[j] = __ballot(i < z.n && (int)(x[j] >> 21) == bin);
            all += __popcll(set[j]);
        }
        if (lane == 0) at = atomicAdd(&count, all);
        at = __shfl(at, 0);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {  // (in any order)
            if (set[j] >> lane & 1) listed[at + __popcll(set[j] & ((1ull << lane) - 1ull))] = u32x2{x[j], (uint32_t)(i0 + j * kSelectThreads + (int)threadIdx.x)};
            at += __popcll(set[j]);
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) mine[e] += __shfl_xor(mine[e], o);
        if (lane == 0) atomicAdd(&greater[e], mine[e]);
    }
    __syncthreads();
    if (threadIdx.x == 0) a.counts[(size_t)z.pair * a.segments + blockIdx.x] = Counts{bin, left, count, {greater[0], greater[1]}};
}

__global__ __launch_bounds__(kSelectThreads) void evict_list_kernel(EvictArgs a) {
    __shared__ Shared<kSelectThreads> sh;
    __shared__ int bins[kBins], ends[kMostSegments], past_counts[4];
    __shared__ u32x2 candidates[kCandidates];
    const Sizes z = sizes_of(a, blockIdx.y);
    const Segment g = segment_of(a, z);
    if (z.m == 0 || g.i0 >= g.i1) {
        if (blockIdx.x == 0 && threadIdx.x == 0) a.moves[z.pair] = 0;
        return;
    }
    const int of = (z.n + a.segment - 1) / a.segment, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t own[kPer];
    load_keys<kSelectThreads>(a, z, g.i0, own);  // (on their way until the lists)
    uint32_t found = 0;
    int left = 0;
    Before past{0, 0, 0};
    if (z.m < z.n) {
        const Counts* const counts = a.counts + (size_t)z.pair * a.segments;
        left = counts[0].left;
        found = (uint32_t)counts[0].bin << 21;
        if (wave == 0) {  // a lane a segment
            const bool on = lane < of, before = lane < (int)blockIdx.x;
            int upto = on ? counts[lane].listed : 0, greater[2] = {before ? counts[lane].greater[0] : 0, before ? counts[lane].greater[1] : 0};
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int below = __shfl_up(upto, o);
                if (lane >= o) upto += below;
                greater[0] += __shfl_xor(greater[0], o), greater[1] += __shfl_xor(greater[1], o);
            }
            if (on) ends[lane] = upto;
            if (lane < 2) past_counts[lane] = greater[lane], past_counts[2 + lane] = 0;
        }
        __syncthreads();
        const int in = ends[of - 1];
        // the rows in the bin, a wavefront a segment: f(order and row, place among all)
        auto all = [&](auto&& f) __attribute__((always_inline)) {
            constexpr int kAhead = 4;
            for (int s = wave; s < of; s += kSelectThreads / 64) {
                const u32x2* const listed = a.listed + (size_t)z.pair * a.stride + (size_t)s * a.segment;
                const int first = s ? ends[s - 1] : 0, n = ends[s] - first;
                for (int k0 = lane; k0 < n; k0 += 64 * kAhead) {
                    u32x2 x[kAhead];
#pragma unroll
                    for (int j = 0; j < kAhead; ++j) x[j] = listed[min(k0 + 64 * j, n - 1)];
#pragma unroll
                    for (int j = 0; j < kAhead; ++j)
                        if (k0 + 64 * j < n) f(x[j], first + k0 + 64 * j);
                }
            }
        };
        const int highest = kBins - 1 - 2 * (int)threadIdx.x;
        const bool fits = in <= kCandidates;
        bins[highest] = bins[highest - 1] = 0;
        if (fits) all([&](const u32x2& x, int at) __attribute__((always_inline)) { candidates[at] = x; });
        __syncthreads();
        auto some = [&](auto&& f) __attribute__((always_inline)) {
            if (fits) {
                for (int at = threadIdx.x; at < in; at += kSelectThreads) f(candidates[at][0], (int)candidates[at][1]);
            } else {
                all([&](const u32x2& x, int) __attribute__((always_inline)) { f(x[0], (int)x[1]); });
            }
        };
#pragma unroll
        for (int pass = 0; pass < 2; ++pass) {
            const int above = pass ? 10 : 21, shift = pass ? 0 : 10;
            some([&](uint32_t x, int) __attribute__((always_inline)) {
                if ((x >> above) == (found >> above)) atomicAdd(&bins[(x >> shift) & ((1u << (above - shift)) - 1u)], 1);
            });
            __syncthreads();
            const int here[2] = {bins[highest], bins[highest - 1]};
            bins[highest] = bins[highest - 1] = 0;  // (for the next pass)
            int bin;
            choose(sh, here, highest, bin, left);
            found |= (uint32_t)bin << shift;
        }
        int greater[2] = {0, 0}, equal[2] = {0, 0};  // of the segments before, before the keep-th row and behind
        some([&](uint32_t x, int i) __attribute__((always_inline)) {
            if (i >= g.i0) return;
            if (x > found) greater[0] += i < z.m, greater[1] += i >= z.m;
            if (x == found) equal[0] += i < z.m, equal[1] += i >= z.m;
        });
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            int x = e < 2 ? greater[e] : equal[e - 2];
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
            if (lane == 0 && x) atomicAdd(&past_counts[e], x);
        }
        __syncthreads();
        const int e0 = min(left, past_counts[2]), e1 = min(left - e0, past_counts[3]);  // equal ones that stay
        past.equal = past_counts[2] + past_counts[3];
        past.holes = min(z.m, g.i0) - past_counts[0] - e0;
        past.movers = past_counts[1] + e1;
    }
    for (int i0 = g.i0; i0 < g.i1; i0 += kBlock) {
        if (i0 > g.i0) load_keys<kSelectThreads>(a, z, i0, own);
        list_block(a, sh, z, i0, own, found, left, past, to_of(a, z), from_of(a, z));
    }
    if ((int)blockIdx.x == of - 1 && threadIdx.x == 0) a.moves[z.pair] = past.holes;
}

constexpr int kMoveWorkgroups = 16384;
// KV heads of sequences from which on each one's moves are made by the workgroup that selects its rows, us for those of another kernel: 256 of 3000 rows in
// e4m3, 3/4 kept, 27 for 34; 1024 of 500 in e2m1 47 for 58; 256 of 8000 in bf16 142 for 130.  Fewer: 128 of 8000 106 for 63, 4 of 3000 24 for 16.
constexpr int kAlone = 256;
// And from which on, where they have up to 2048 rows, by one of 256 threads, of which a CU holds more, us for those of 1024 threads: 1024 of 1792 in e4m3 73 for 96, of 500 in
// e2m1 19.5 for 47, of 100 14.5 for 45; 512 of 2000 in e4m3 34 for 46.  256 of 2000 27.2 for 25.5.
constexpr int kMany = 512;
static_assert(kMany >= kAlone, "who selects with few threads makes the moves too, and leaves no list for another kernel");

size_t lay_out(EvictArgs& a, char* base) {
    size_t at = 0;
    auto take = [&](auto*& p, size_t count) {
        p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += (count * sizeof(*p) + 255) / 256 * 256;
    };
    const size_t pairs = (size_t)a.gm.B * a.gm.Hkv;
    take(a.moves, pairs);
    take(a.to, pairs * (a.max_rows / 2));
    take(a.from, pairs * (a.max_rows / 2));
    if (a.max_rows <= kBlock) return at;
    a.segment = (a.max_rows + kMostSegments * kBlock - 1) / (kMostSegments * kBlock) * kBlock;
    a.segments = (a.max_rows + a.segment - 1) / a.segment;
    a.stride = a.segments * a.segment;
    take(a.keys, pairs * a.stride);
    take(a.bins, pairs * a.segments * kBins);
    take(a.counts, pairs * a.segments);
    take(a.listed, pairs * a.stride);
    return at;
}

}  // namespace

size_t evict_workspace(const Geom& g, int max_rows) {
    EvictArgs a{};
    a.gm = g, a.max_rows = max_rows;
    return lay_out(a, nullptr);
}

int cache_evict(const Geom& g, const Pages& c, const int32_t* rows, const int32_t* keep, int max_rows, const float* weight_in, float* weight,
                int32_t* kept, void* workspace, hipStream_t st) {
    EvictArgs a{g, c, rows, keep, max_rows, weight_in, weight, kept};
    lay_out(a, (char*)workspace);
    const int pairs = g.B * g.Hkv;
    auto launch = [&](auto bits) {
        constexpr int BITS = decltype(bits)::value;
        const bool alone = max_rows <= kBlock && pairs >= kAlone;
        if (max_rows <= kBlock) {
            KernelTimer kt("evict_select", st);
            if (pairs >= kMany && max_rows <= kFewThreads * kPer) hipLaunchKernelGGL((evict_select_kernel<BITS, kFewThreads>), dim3(pairs), dim3(kFewThreads), 0, st, a);
            else if (alone) hipLaunchKernelGGL((evict_select_kernel<BITS, kSelectThreads>), dim3(pairs), dim3(kSelectThreads), 0, st, a);
            else hipLaunchKernelGGL((evict_select_kernel<0, kSelectThreads>), dim3(pairs), dim3(kSelectThreads), 0, st, a);
        } else {
            const dim3 grid(a.segments, pairs);
            KernelTimer kt("evict_select", st);
            hipLaunchKernelGGL(evict_first_kernel, grid, dim3(kSelectThreads), 0, st, a);
            hipLaunchKernelGGL(evict_second_kernel, grid, dim3(kSelectThreads), 0, st, a);
            hipLaunchKernelGGL(evict_list_kernel, grid, dim3(kSelectThreads), 0, st, a);
        }
        if (!alone && max_rows > 1) {
            KernelTimer kt("evict_move", st);
            constexpr int kEach = kThreads / (2 * BITS) * kAhead;  // moves of a workgroup
            const int most = (max_rows / 2 + kEach - 1) / kEach, share = (kMoveWorkgroups + pairs - 1) / pairs;
            hipLaunchKernelGGL(evict_move_kernel<BITS>, dim3(most < share ? most : share, pairs), dim3(kThreads), 0, st, a);
        }
    };
    if (c.bits == 16) launch(std::integral_constant<int, 16>{});
    else if (c.bits == 8) launch(std::integral_constant<int, 8>{});
    else launch(std::integral_constant<int, 4>{});
    return launch_status();
}

}  // namespace l2a
