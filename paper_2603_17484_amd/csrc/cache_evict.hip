// Eviction from a paged KV cache: of the first `rows` rows of a sequence every KV head keeps the `keep` of greatest weight (of equal ones
// the first; NaN is less than everything).  Kept rows before row `keep` stay where they are; the i-th row that leaves before it is the
// place of the i-th kept row behind it.  As many leave before as are kept behind, no place is read and written both, and so the moves are
// independent of one another, in place, and no more bytes move than have to.  The order of rows does not matter to the attention over them:
// their positions are in the keys.
//
// Which rows stay is a radix selection over the weights' bits, ordered as whole numbers: the histogram of their highest bits says in which bin
// the last row that stays lies, that of the bits below among the rows of this bin where in it, and so on.  Then the lists: places that become free, and
// rows that move there, both ascending.
//   evict_select_kernel  up to 8192 rows: a workgroup per KV head of a sequence, the weights in its registers, 11, 11 and 10 bits
//   evict_first_kernel, evict_second_kernel, evict_third_kernel, evict_list_kernel
//                        more: a workgroup per 8192 rows (or 1/64); each leaves its own histogram, and each workgroup of the next
//                        kernel adds up those of its KV head (no atomics on memory, nothing to clear)
//   evict_move_kernel    the moves: K, V, exponents, weights
#include "paged.hpp"

namespace l2a {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kPer = 8;                          // rows of a thread
constexpr int kBlock = kSelectThreads * kPer;
constexpr int kMostSegments = 64;                // workgroups of a KV head of a sequence
constexpr int kBins1 = 2048, kBins3 = 1024;      // 11, 11 and 10 bits

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
    uint32_t* keys;   // [B * Hkv][max_rows] order of the weights
    int32_t *bins1, *bins2;  // [B * Hkv][segments][kBins1]
    int32_t* bins3;   // [B * Hkv][segments][2][kBins3]: of rows before the keep-th and behind
    int32_t* above;   // [B * Hkv][segments][2]: rows whose upper 22 bits say that they stay, before and behind
    int32_t* chosen;  // [B * Hkv][4]: the bin of the first bits and the how-manieth in it, of the first two
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
// Row i0 + 1024 j + thread of a block as order; 0 past the end.  Where the weights do not stay in place, those before the keep-th go to theirs (the moves
// write over those that leave).
__device__ __forceinline__ void load_block(const EvictArgs& a, const Sizes& z, int i0, uint32_t (&x)[kPer]) {
    float w[kPer];
    size_t row[kPer];
    bool real[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * kSelectThreads + (int)threadIdx.x, page = i < z.n ? page_at(a, z.b, i) : 0;
        real[j] = (unsigned)page < (unsigned)a.c.pages;
        row[j] = pool_row(a.c, a.gm.Hkv, plan::clamp(page, 0, a.c.pages - 1), z.hk, i);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) w[j] = i0 + j * kSelectThreads + (int)threadIdx.x < z.n ? a.weight_in[row[j]] : 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * kSelectThreads + (int)threadIdx.x;
        x[j] = i < z.n ? order(w[j]) : 0u;
        if (a.weight != a.weight_in && i < z.m && real[j]) a.weight[row[j]] = w[j];
    }
}
__device__ __forceinline__ void load_keys(const EvictArgs& a, const Sizes& z, int i0, uint32_t (&x)[kPer]) {
    const uint32_t* const keys = a.keys + (size_t)z.pair * a.max_rows;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * kSelectThreads + (int)threadIdx.x;
        x[j] = i < z.n ? keys[i] : 0u;
    }
}

struct Shared {
    int sums[kSelectThreads / 64], chosen[2], counts[kPer][kSelectThreads / 64];
};
// Bins from the highest number down, EACH a thread in the order of threads; mine: how many rows this thread's have, `highest` its first.  The bin in
// which the left-th row lies, and the how-manieth in it that is.
template <int EACH>
__device__ __forceinline__ void choose(Shared& sh, const int (&mine)[EACH], int highest, int& bin, int& left) {
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
    for (int w = 0; w < kSelectThreads / 64; ++w)
        if (w < wave) before += sh.sums[w];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        if (before < left && left <= before + mine[e]) sh.chosen[0] = highest - e, sh.chosen[1] = left - before;
        before += mine[e];
    }
    __syncthreads();
    bin = sh.chosen[0], left = sh.chosen[1];
    __syncthreads();
}
// Places of flags among all of a block, in the order of rows: of this thread's j-th, how many lie before it; and how many there are.  Two kinds of flags
// at once, the second's numbers in the upper halves (a block has fewer than 2^16 rows).
__device__ __forceinline__ int places(Shared& sh, const bool (&flag)[kPer], const bool (&other)[kPer], int (&at)[kPer]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned long long before = (1ull << lane) - 1ull;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const unsigned long long set = __ballot(flag[j]), more = __ballot(other[j]);
        at[j] = __popcll(set & before) + (__popcll(more & before) << 16);
        if (lane == 0) sh.counts[j][wave] = __popcll(set) + (__popcll(more) << 16);
    }
    __syncthreads();
    // every wavefront adds up all counts: a lane those of two
    constexpr int kWavesOf = kSelectThreads / 64, kCounts = kPer * kWavesOf;
    static_assert(kCounts == 128, "two counts a lane");
    const int* const counts = &sh.counts[0][0];
    const int c0 = counts[2 * lane], c1 = counts[2 * lane + 1];
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
    const int total = __shfl(upto, 63);
    __syncthreads();
    return total;
}
// What the rows of a block before it had: equal ones, places that become free, rows that move.
struct Before {
    int equal, holes, movers;
};
// The lists of a block, its rows x in registers: all greater than `found` stay, and the first `left` of those equal to it.
__device__ __forceinline__ void list_block(const EvictArgs& a, Shared& sh, const Sizes& z, int i0, const uint32_t (&x)[kPer], uint32_t found, int left, Before& past) {
    int32_t *to = a.to + (size_t)z.pair * (a.max_rows / 2), *from = a.from + (size_t)z.pair * (a.max_rows / 2);
    int32_t* const kept = a.kept ? a.kept + (size_t)z.pair * a.max_rows : nullptr;
    bool flag[kPer], other[kPer], stays[kPer];
    int at[kPer];
    const bool all = z.m == z.n;
#pragma unroll
    for (int j = 0; j < kPer; ++j) flag[j] = !all && x[j] == found && i0 + j * kSelectThreads + (int)threadIdx.x < z.n, other[j] = false;
    const int equal = places(sh, flag, other, at);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * kSelectThreads + (int)threadIdx.x;
        stays[j] = i < z.n && (all || x[j] > found || (flag[j] && past.equal + at[j] < left));
        flag[j] = i < z.m && !stays[j], other[j] = i >= z.m && stays[j];
    }
    const int both = places(sh, flag, other, at), holes = both & 0xffff, movers = both >> 16;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int i = i0 + j * kSelectThreads + (int)threadIdx.x;
        if (flag[j]) to[past.holes + (at[j] & 0xffff)] = i;
        if (other[j]) from[past.movers + (at[j] >> 16)] = i;
        if (kept && i < z.m && stays[j]) kept[i] = i;
    }
    past = Before{past.equal + equal, past.holes + holes, past.movers + movers};
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
    __shared__ Shared sh;
    __shared__ int bins[kBins1];
    const Sizes z = sizes_of(a, blockIdx.x);
    if (z.m == 0) {
        if (threadIdx.x == 0) a.moves[z.pair] = 0;
        return;
    }
    uint32_t x[kPer], found = 0;
    load_block(a, z, 0, x);
    int left = z.m;
    const int highest = kBins1 - 1 - 2 * (int)threadIdx.x;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        if (z.m == z.n) break;
        constexpr int kShift[3] = {21, 10, 0};
        const int shift = kShift[pass], above = pass ? kShift[pass - 1] : 0;
        bins[highest] = bins[highest - 1] = 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (j * kSelectThreads + (int)threadIdx.x < z.n && (pass == 0 || (x[j] >> above) == (found >> above))) atomicAdd(&bins[(x[j] >> shift) & (pass == 2 ? kBins3 - 1 : kBins1 - 1)], 1);
        __syncthreads();
        const int mine[2] = {bins[highest], bins[highest - 1]};
        int bin;
        choose<2>(sh, mine, highest, bin, left);
        found |= (uint32_t)bin << shift;
    }
    Before past{0, 0, 0};
    list_block(a, sh, z, 0, x, found, left, past);
    if (threadIdx.x == 0) a.moves[z.pair] = past.holes;
}

// The workgroup's segment of its pair: rows i0 .. i1 - 1.
struct Segment {
    int i0, i1;
};
__device__ __forceinline__ Segment segment_of(const EvictArgs& a, const Sizes& z) {
    const long long i0 = (long long)blockIdx.x * a.segment;
    Segment g;
    g.i0 = i0 < z.n ? (int)i0 : z.n, g.i1 = i0 + a.segment < z.n ? (int)(i0 + a.segment) : z.n;
    return g;
}
__device__ __forceinline__ int32_t* bins_at(const EvictArgs& a, int32_t* bins, int pair, int segment) { return bins + ((size_t)pair * a.segments + segment) * kBins1; }
// Segments that have rows.
__device__ __forceinline__ int segments_of(const EvictArgs& a, const Sizes& z) { return (z.n + a.segment - 1) / a.segment; }
// The bin of a pair's histograms, all segments together, in which the left-th row lies.
__device__ __forceinline__ int choose_bin(const EvictArgs& a, Shared& sh, const Sizes& z, int32_t* bins, int& left) {
    int mine[2] = {0, 0};
    const int highest = kBins1 - 1 - 2 * (int)threadIdx.x, of = segments_of(a, z);
#pragma unroll 8
    for (int g = 0; g < of; ++g) {
        const int32_t* const p = bins_at(a, bins, z.pair, g);
        mine[0] += p[highest], mine[1] += p[highest - 1];
    }
    int bin;
    choose<2>(sh, mine, highest, bin, left);
    return bin;
}
static_assert(kBins1 == 2 * kSelectThreads && 2 * kBins3 == kBins1, "bins of a thread");

// The highest 11 bits, and the order of all rows for the kernels behind.
__global__ __launch_bounds__(kSelectThreads) void evict_first_kernel(EvictArgs a) {
    __shared__ int bins[kBins1];
    const Sizes z = sizes_of(a, blockIdx.y);
    const Segment g = segment_of(a, z);
    if (g.i0 >= g.i1) return;
    for (int i = threadIdx.x; i < kBins1; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i0 = g.i0; i0 < g.i1; i0 += kBlock) {
        uint32_t x[kPer];
        load_block(a, z, i0, x);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int i = i0 + j * kSelectThreads + (int)threadIdx.x;
            if (i < z.n) {
                a.keys[(size_t)z.pair * a.max_rows + i] = x[j];
                atomicAdd(&bins[x[j] >> 21], 1);
            }
        }
    }
    __syncthreads();
    int32_t* const out = bins_at(a, a.bins1, z.pair, blockIdx.x);
    for (int i = threadIdx.x; i < kBins1; i += kSelectThreads) out[i] = bins[i];
}
// The next 11 bits of rows in the bin found.  (Its number is left for the kernels behind, by the first workgroup.)
__global__ __launch_bounds__(kSelectThreads) void evict_second_kernel(EvictArgs a) {
    __shared__ Shared sh;
    __shared__ int bins[kBins1];
    const Sizes z = sizes_of(a, blockIdx.y);
    const Segment g = segment_of(a, z);
    if (g.i0 >= g.i1 || z.m == 0 || z.m == z.n) return;
    for (int i = threadIdx.x; i < kBins1; i += kSelectThreads) bins[i] = 0;
    int left = z.m;
    const uint32_t first = (uint32_t)choose_bin(a, sh, z, a.bins1, left);
    if (blockIdx.x == 0 && threadIdx.x == 0) a.chosen[z.pair * 4] = (int)first, a.chosen[z.pair * 4 + 1] = left;
    for (int i0 = g.i0; i0 < g.i1; i0 += kBlock) {
        uint32_t x[kPer];
        load_keys(a, z, i0, x);
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (i0 + j * kSelectThreads + (int)threadIdx.x < z.n && (x[j] >> 21) == first) atomicAdd(&bins[(x[j] >> 10) & (kBins1 - 1)], 1);
    }
    __syncthreads();
    int32_t* const out = bins_at(a, a.bins2, z.pair, blockIdx.x);
    for (int i = threadIdx.x; i < kBins1; i += kSelectThreads) out[i] = bins[i];
}
// The last 10, rows before the keep-th and behind apart, and how many of either stay for their higher bits.
__global__ __launch_bounds__(kSelectThreads) void evict_third_kernel(EvictArgs a) {
    __shared__ Shared sh;
    __shared__ int bins[2 * kBins3], above[2];
    const Sizes z = sizes_of(a, blockIdx.y);
    const Segment g = segment_of(a, z);
    if (g.i0 >= g.i1 || z.m == 0 || z.m == z.n) return;
    for (int i = threadIdx.x; i < 2 * kBins3; i += kSelectThreads) bins[i] = 0;
    if (threadIdx.x < 2) above[threadIdx.x] = 0;
    int left = a.chosen[z.pair * 4 + 1];
    const uint32_t upper = (uint32_t)a.chosen[z.pair * 4] << 11 | (uint32_t)choose_bin(a, sh, z, a.bins2, left);
    if (blockIdx.x == 0 && threadIdx.x == 0) a.chosen[z.pair * 4 + 2] = (int)upper, a.chosen[z.pair * 4 + 3] = left;
    int mine[2] = {0, 0};
    for (int i0 = g.i0; i0 < g.i1; i0 += kBlock) {
        uint32_t x[kPer];
        load_keys(a, z, i0, x);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int i = i0 + j * kSelectThreads + (int)threadIdx.x, behind = i >= z.m;
            if (i >= z.n) continue;
            if ((x[j] >> 10) == upper) atomicAdd(&bins[behind * kBins3 + (int)(x[j] & (kBins3 - 1))], 1);
            if ((x[j] >> 10) > upper) mine[0] += !behind, mine[1] += behind;
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) mine[e] += __shfl_xor(mine[e], o);
        if ((threadIdx.x & 63) == 0) atomicAdd(&above[e], mine[e]);
    }
    __syncthreads();
    int32_t* const out = bins_at(a, a.bins3, z.pair, blockIdx.x);
    for (int i = threadIdx.x; i < 2 * kBins3; i += kSelectThreads) out[i] = bins[i];
    if (threadIdx.x < 2) a.above[((size_t)z.pair * a.segments + blockIdx.x) * 2 + threadIdx.x] = above[threadIdx.x];
}
// The lists.  What the segments before have of them follows from their histograms.
__global__ __launch_bounds__(kSelectThreads) void evict_list_kernel(EvictArgs a) {
    __shared__ Shared sh;
    __shared__ int greater[kMostSegments][2], equal[kMostSegments][2];  // of each segment, before the keep-th row and behind
    const Sizes z = sizes_of(a, blockIdx.y);
    const Segment g = segment_of(a, z);
    const int of = segments_of(a, z);
    if (z.m == 0 || g.i0 >= g.i1) {
        if (blockIdx.x == 0 && threadIdx.x == 0) a.moves[z.pair] = 0;
        return;
    }
    uint32_t found = 0;
    int left = 0;
    Before past{0, 0, 0};
    if (z.m < z.n) {
        const uint32_t upper = (uint32_t)a.chosen[z.pair * 4 + 2];
        left = a.chosen[z.pair * 4 + 3];
        const int bin = kBins3 - 1 - (int)threadIdx.x;  // this thread's
        int mine[1] = {0};
#pragma unroll 8
        for (int s = 0; s < of; ++s) {
            const int32_t* const p = bins_at(a, a.bins3, z.pair, s);
            mine[0] += p[bin] + p[kBins3 + bin];
        }
        int lowest;
        choose<1>(sh, mine, bin, lowest, left);
        found = upper << 10 | (uint32_t)lowest;
        // a wavefront for each half of a segment before this one
        const int lane = threadIdx.x & 63;
        for (int i = threadIdx.x >> 6; i < 2 * (int)blockIdx.x; i += kSelectThreads / 64) {
            const int32_t* const p = bins_at(a, a.bins3, z.pair, i >> 1) + (i & 1) * kBins3;
            int more = lane == 0 ? a.above[((size_t)z.pair * a.segments + (i >> 1)) * 2 + (i & 1)] : 0;
#pragma unroll
            for (int e = 0; e < kBins3 / 64; ++e) more += e * 64 + lane > lowest ? p[e * 64 + lane] : 0;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) more += __shfl_xor(more, o);
            if (lane == 0) greater[i >> 1][i & 1] = more, equal[i >> 1][i & 1] = p[lowest];
        }
        __syncthreads();
        for (int s = 0; s < (int)blockIdx.x; ++s) {
            const int i0 = s * a.segment, i1 = i0 + a.segment, before = plan::clamp(z.m, i0, i1) - i0;  // rows of it before the keep-th
            const int e0 = plan::clamp(left - past.equal, 0, equal[s][0]), e1 = plan::clamp(left - past.equal - equal[s][0], 0, equal[s][1]);
            past.holes += before - greater[s][0] - e0;
            past.movers += greater[s][1] + e1;
            past.equal += equal[s][0] + equal[s][1];
        }
    }
    for (int i0 = g.i0; i0 < g.i1; i0 += kBlock) {
        uint32_t x[kPer];
        load_keys(a, z, i0, x);
        list_block(a, sh, z, i0, x, found, left, past);
    }
    if ((int)blockIdx.x == of - 1 && threadIdx.x == 0) a.moves[z.pair] = past.holes;
}

// A group of lanes per move, 16 bytes a lane, K's and V's beside one another; kAhead moves of a group on their way together.
template <int BITS>
__global__ __launch_bounds__(kThreads) void evict_move_kernel(EvictArgs a) {
    constexpr int kLanes = 2 * BITS, kGroups = kThreads / kLanes, kAhead = 4, kRowBytes = kD * BITS / 8;
    const int pair = blockIdx.y, b = pair / a.gm.Hkv, hk = pair - b * a.gm.Hkv;
    const int count = a.moves[pair], lane = threadIdx.x % kLanes, c = lane % (kLanes / 2);
    const size_t list = (size_t)pair * (a.max_rows / 2);
    char* const pool = (lane < kLanes / 2 ? a.c.k : a.c.v) + c * 16;
    unsigned char* const scales = lane < kLanes / 2 ? a.c.ks : a.c.vs;
    for (int i0 = (blockIdx.x * kGroups + (int)threadIdx.x / kLanes) * kAhead; i0 < count; i0 += gridDim.x * kGroups * kAhead) {
        int to[kAhead], from[kAhead];
        size_t dst[kAhead], src[kAhead];
        bool on[kAhead];
        u32x4 x[kAhead];
        uint32_t e[kAhead];
        float w[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) to[j] = a.to[list + min(i0 + j, count - 1)], from[j] = a.from[list + min(i0 + j, count - 1)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int p = page_at(a, b, to[j]), q = page_at(a, b, from[j]);
            on[j] = i0 + j < count && (unsigned)p < (unsigned)a.c.pages && (unsigned)q < (unsigned)a.c.pages;  // page numbers outside the pool are never followed
            dst[j] = on[j] ? pool_row(a.c, a.gm.Hkv, p, hk, to[j]) : 0, src[j] = on[j] ? pool_row(a.c, a.gm.Hkv, q, hk, from[j]) : 0;
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
            if (lane == 2 && a.kept && i0 + j < count) a.kept[(size_t)pair * a.max_rows + to[j]] = from[j];
        }
    }
}

constexpr int kMoveWorkgroups = 16384;

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
    take(a.keys, pairs * a.max_rows);
    take(a.bins1, pairs * a.segments * kBins1);
    take(a.bins2, pairs * a.segments * kBins1);
    take(a.bins3, pairs * a.segments * kBins1);
    take(a.above, pairs * a.segments * 2);
    take(a.chosen, pairs * 4);
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
    if (max_rows <= kBlock) {
        KernelTimer kt("evict_select", st);
        hipLaunchKernelGGL(evict_select_kernel, dim3(pairs), dim3(kSelectThreads), 0, st, a);
    } else {
        const dim3 grid(a.segments, pairs);
        KernelTimer kt("evict_select", st);
        hipLaunchKernelGGL(evict_first_kernel, grid, dim3(kSelectThreads), 0, st, a);
        hipLaunchKernelGGL(evict_second_kernel, grid, dim3(kSelectThreads), 0, st, a);
        hipLaunchKernelGGL(evict_third_kernel, grid, dim3(kSelectThreads), 0, st, a);
        hipLaunchKernelGGL(evict_list_kernel, grid, dim3(kSelectThreads), 0, st, a);
    }
    if (max_rows > 1) {
        KernelTimer kt("evict_move", st);
        auto launch = [&](auto bits) {
            constexpr int BITS = decltype(bits)::value;
            constexpr int kEach = kThreads / (2 * BITS) * 4;  // moves of a workgroup
            const int most = (max_rows / 2 + kEach - 1) / kEach, share = (kMoveWorkgroups + pairs - 1) / pairs;
            hipLaunchKernelGGL(evict_move_kernel<BITS>, dim3(most < share ? most : share, pairs), dim3(kThreads), 0, st, a);
        };
        if (c.bits == 16) launch(std::integral_constant<int, 16>{});
        else if (c.bits == 8) launch(std::integral_constant<int, 8>{});
        else launch(std::integral_constant<int, 4>{});
    }
    return launch_status();
}

}  // namespace l2a
