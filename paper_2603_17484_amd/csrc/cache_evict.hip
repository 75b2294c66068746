// Eviction from a paged KV cache: of the first `rows` rows of a sequence every KV head keeps the `keep` of greatest weight (of equal ones
// the first; NaN is less than everything).  Kept rows before row `keep` stay where they are; the i-th row that leaves before it is the
// place of the i-th kept row behind it.  As many leave before as are kept behind, no place is read and written both, and so the moves are
// independent of one another, in place, and no more bytes move than have to.  The order of rows does not matter to the attention over them:
// their positions are in the keys.
//
//   evict_select_kernel  a workgroup per KV head of a sequence: the weight of the last row that stays, by radix selection (8 bits a
//                        pass over the weights' bits, ordered as whole numbers), and the lists of places and of rows that move there
//   evict_move_kernel    the moves: K, V, exponents, weights
#include "paged.hpp"

namespace l2a {
namespace {

constexpr int kSelectThreads = 1024;
constexpr int kBins = 256;

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
};

__device__ __forceinline__ int rows_of(const EvictArgs& a, int b) { return plan::clamp(a.rows[b], 0, min(a.max_rows, a.c.capacity())); }
// Whole numbers in the order of the weights.  Zeros are alike, NaN comes first.
__device__ __forceinline__ uint32_t order(float w) {
    const uint32_t x = __float_as_uint(w + 0.f);
    if (w != w) return 0u;
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}
__device__ __forceinline__ int page_at(const EvictArgs& a, int b, int row) { return a.c.table[(size_t)b * a.c.max_pages + (row >> a.c.page_log2)]; }
__device__ __forceinline__ size_t row_at(const EvictArgs& a, int b, int hk, int row) {
    return pool_row(a.c, a.gm.Hkv, plan::clamp(page_at(a, b, row), 0, a.c.pages - 1), hk, row);
}

// Sum of x over the threads before this one, and over all.
__device__ __forceinline__ void scan(int x, int* sums, int& before, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int below = __shfl_up(upto, o);
        if (lane >= o) upto += below;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    before = upto - x, total = 0;
#pragma unroll
    for (int w = 0; w < kSelectThreads / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
}

__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
    __shared__ int bins[kBins], sums[kSelectThreads / 64], chosen[2];
    const int pair = blockIdx.x, b = pair / a.gm.Hkv, hk = pair - b * a.gm.Hkv;
    const int n = rows_of(a, b), m = plan::clamp(a.keep[b], 0, n);
    // the m-th greatest: from the highest 8 bits on, which value they have, and the how-manieth of those with it that is
    uint32_t found = 0;
    int left = m;
    if (m > 0 && m < n) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < kBins) bins[threadIdx.x] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += kSelectThreads) {
                const uint32_t x = order(a.weight_in[row_at(a, b, hk, i)]);
                if (shift == 24 || (x >> (shift + 8)) == (found >> (shift + 8))) atomicAdd(&bins[(x >> shift) & 255], 1);
            }
            __syncthreads();
            // thread t: the bins above t
            const int mine = threadIdx.x < kBins ? bins[kBins - 1 - threadIdx.x] : 0;
            int before, total;
            scan(mine, sums, before, total);
            if (threadIdx.x < kBins && before < left && left <= before + mine) chosen[0] = kBins - 1 - (int)threadIdx.x, chosen[1] = left - before;
            __syncthreads();
            found |= (uint32_t)chosen[0] << shift, left = chosen[1];
            __syncthreads();
        }
    }
    // `left` rows with the weight found stay, the first ones, and all with a greater one
    int32_t *to = a.to + (size_t)pair * (a.max_rows / 2), *from = a.from + (size_t)pair * (a.max_rows / 2);
    int32_t* const kept = a.kept ? a.kept + (size_t)pair * a.max_rows : nullptr;
    int equal = 0, holes = 0, movers = 0;
    for (int i0 = 0; i0 < n && m > 0; i0 += kSelectThreads) {
        const int i = i0 + (int)threadIdx.x;
        float w = 0.f;
        size_t at = 0;
        if (i < n) at = row_at(a, b, hk, i), w = a.weight_in[at];
        const uint32_t x = order(w);
        int before, total;
        const bool tie = i < n && m < n && x == found;
        scan(tie, sums, before, total);
        const bool stays = i < n && (m == n || x > found || (tie && equal + before < left));
        equal += total;
        const bool hole = i < m && !stays, mover = i >= m && stays;
        scan((hole ? 1 : 0) + (mover ? 0x10000 : 0), sums, before, total);
        if (hole) to[holes + (before & 0xffff)] = i;
        if (mover) from[movers + (before >> 16)] = i;
        holes += total & 0xffff, movers += total >> 16;
        if (i < m && stays) {
            if (a.weight != a.weight_in && (unsigned)page_at(a, b, i) < (unsigned)a.c.pages) a.weight[at] = w;
            if (kept) kept[i] = i;
        }
    }
    if (threadIdx.x == 0) a.moves[pair] = holes;
}

// A group of lanes per move: 16 lanes K, 16 lanes V.
__global__ __launch_bounds__(kThreads) void evict_move_kernel(EvictArgs a) {
    const int pair = blockIdx.y, b = pair / a.gm.Hkv, hk = pair - b * a.gm.Hkv;
    const int count = a.moves[pair], lane = threadIdx.x & 31, row_bytes = kD * a.c.bits / 8;
    const size_t list = (size_t)pair * (a.max_rows / 2);
    char* const pool = lane < 16 ? a.c.k : a.c.v;
    unsigned char* const scales = lane < 16 ? a.c.ks : a.c.vs;
    const int c = lane & 15;
    for (int i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i < count; i += gridDim.x * (kThreads / 32)) {
        const int to = a.to[list + i], from = a.from[list + i];
        if (lane == 0 && a.kept) a.kept[(size_t)pair * a.max_rows + to] = from;
        // page numbers outside the pool are never followed
        if ((unsigned)page_at(a, b, to) >= (unsigned)a.c.pages || (unsigned)page_at(a, b, from) >= (unsigned)a.c.pages) continue;
        const size_t dst = row_at(a, b, hk, to), src = row_at(a, b, hk, from);
        if (c * 16 < row_bytes) *reinterpret_cast<u32x4*>(pool + dst * row_bytes + c * 16) = *reinterpret_cast<const u32x4*>(pool + src * row_bytes + c * 16);
        if (a.c.bits < 16 && c == 0) *reinterpret_cast<uint32_t*>(scales + dst * kRowScales) = *reinterpret_cast<const uint32_t*>(scales + src * kRowScales);
        if (lane == 0) a.weight[dst] = a.weight_in[src];
    }
}

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
    {
        KernelTimer kt("evict_select", st);
        hipLaunchKernelGGL(evict_select_kernel, dim3(pairs), dim3(kSelectThreads), 0, st, a);
    }
    {
        KernelTimer kt("evict_move", st);
        const int most = (max_rows / 2 + kThreads / 32 - 1) / (kThreads / 32), share = (4096 + pairs - 1) / pairs;
        if (most) hipLaunchKernelGGL(evict_move_kernel, dim3(most < share ? most : share, pairs), dim3(kThreads), 0, st, a);
    }
    return launch_status();
}

}  // namespace l2a
