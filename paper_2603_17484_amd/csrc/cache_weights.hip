// The attention weights that cached rows receive from the new tokens of a call:
//   w_j <- decay w_j + sum over the group's heads and the tokens t >= j with a finite log-sum-exp of exp(scale <q_t, k_j> - lse_t),
// rows of the new tokens themselves beginning at zero.  With the log-sum-exps that the attention left, weights need neither V nor a maximum, and
// every key's sum is its own: no key's infinity or NaN enters another's.
//
// Few rows (decoding): bound by the keys' bytes.  A wavefront holds a sequence's rows as an operand of the matrix instructions (A) and takes a
// stretch of the keys, 32 at a time as the other operand (B: a lane owns a key), whose loads are on their way while the 32 before are at
// work.  S = Q K^T leaves a lane with 16 rows' scores of its key, whose exponentials it adds up.  (Loads under a condition, in the loop: 172 us for 170 in bf16, one
// behind 32K 10.6 for 10.0.)
//
// Many rows: bound by the matrix cores and the exponentials.  The rows that count are packed first.  Then a workgroup holds 256 keys in
// registers, 64 a wavefront, and their tiles of 32 rows come through shared memory, once for all four wavefronts.  All work laid end to end is a line; every
// workgroup takes an equal stretch of it, and what it does not finish of a chunk of keys meets the rest in a last kernel.
//
// Nothing is added by atomics: the order of every sum is fixed.
//
// Measured (us): 64 tokens behind 8K of 32 / 8 heads in bf16 (831 MB) 170, 4.9 TB/s (a copy of 4 GiB: 4.8), in e4m3 93, in e2m1 57; one behind 32K 10, of which 6 are
// the call's; 2048 behind 32K of 28 / 4 heads, half of them routed (248 GFLOP), 250 a call (0.99 PFLOP/s; 8192 x 8192 matrices
// 1.22); traced kernel by kernel 10 packing, 257 to 265 the products, 5 joining.
#include "paged.hpp"
#include "tiles.hpp"

namespace l2a {
namespace {

using plan::Seq;

constexpr int kSub = 32;    // keys of an operand
constexpr int kRows = 32;   // rows of a tile
constexpr int kWaves = 4;

// A tile's numbers: -lse log2 e of its rows, then their positions (padding: -inf, -1).
struct Numbers {
    float bias[kRows];
    int limit[kRows];
};
// A chunk's keys times a pair's rows, on the line of all work; one that a workgroup begins and does not end.
struct Open {
    long long start, per;  // where it begins; stretches of the line
    int tiles, pair, chunk, pad;
};

struct WeightsArgs {
    Geom gm;  // gm.T = packed tokens
    Pages c;
    const __bf16* q;  // [T, Hq, D]
    const int32_t *seq_start, *pos;
    const float* lse;  // [Hq, T]
    int max_new;
    float decay;
    const float* weight_in;  // optional
    float* weight;
    // workspace of long calls
    int cap;           // rows of a KV head of all sequences, whole tiles
    int32_t* listed;   // [B * Hkv] rows
    int32_t* before;   // [B * Hkv][chunks] listed rows before each chunk of keys that begins with a new token's
    int chunks;
    __bf16* packed;    // [Hkv][cap][D]
    Numbers* numbers;  // [Hkv][cap / kRows]
    Open* open;        // [workgroups]
    float* slots;      // [workgroups][2][kChunk]
    int workgroups;
};

// ---------------------------------------------------------------------------------------
// few rows
// ---------------------------------------------------------------------------------------
constexpr int kMostSeqs = 1024;  // of a launch: their lengths are summed in shared memory

// Key blocks of all sequences up to and with each, in ends; -> of all.
template <typename F>
__device__ __forceinline__ int sum_up(int n, int* ends, int* sums, F&& count) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int total = 0;
    for (int s0 = 0; s0 < n; s0 += 64 * kWaves) {
        const int i = s0 + (int)threadIdx.x;
        int upto = i < n ? count(i) : 0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int below = __shfl_up(upto, o);
            if (lane >= o) upto += below;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) upto += sums[w];
        }
        if (i < n) ends[i] = total + upto;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += sums[w];
    }
    __syncthreads();
    return total;
}
// The first of n ascending ends that lies behind x.
__device__ __forceinline__ int behind(const int* ends, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int page_of(const WeightsArgs& a, int b, int key) { return a.c.table[(size_t)b * a.c.max_pages + (key >> a.c.page_log2)]; }

// A wavefront's part of a KV head of a sequence: `count` blocks of 32 keys from block0 on.
struct Part {
    Seq s;
    int b, hk, block0, count;
};
template <int BITS>
__device__ __forceinline__ void few_part(const WeightsArgs& a, const Part& part) {
    const Geom& gm = a.gm;
    const Seq s = part.s;
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, G = gm.G, b = part.b, hk = part.hk, block0 = part.block0, count = part.count;
    const int last = s.pos + s.n - 1, rows = s.n * G;
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    // the rows: an operand, and what their scores are told apart by
    const int r = min(n, rows - 1), tok = r / G;
    const __bf16* const qp = a.q + ((size_t)(s.start + tok) * gm.Hq + hk * G + r - tok * G) * kD;
    bf16x8 q[8];
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = *reinterpret_cast<const bf16x8*>(qp + slot_channel<BITS>(ks, h));
    const float lse = a.lse[(size_t)(hk * G + r - tok * G) * gm.T + s.start + tok];
    const bool counts = n < rows && fabsf(lse) < INFINITY;
    const float my_bias = counts ? -lse * kLog2e : 0.f;
    const int my_limit = counts ? s.pos + tok : -1;
    float bias[16];
    int limit[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) bias[e] = __shfl(my_bias, c_row(e, h)), limit[e] = __shfl(my_limit, c_row(e, h));
    auto key_at = [&](int j) { return (block0 + j) * kSub + n; };
    auto page_at = [&](int j) { return page_of(a, b, min(key_at(min(j, count - 1)), last)); };
    auto row_at = [&](int j, int page) { return pool_row(a.c, gm.Hkv, plan::clamp(page, 0, a.c.pages - 1), hk, min(key_at(j), last)); };
    int page = page_at(0), coming = page_at(1);
    size_t row = row_at(0, page);
    RawKeys<BITS> raw;
    raw.load(a.c, row, h);
    const float* const old_weights = a.weight_in ? a.weight_in : a.weight;
    auto old_at = [&](size_t at) { return old_weights[a.weight_in ? at : 0]; };
    float old = old_at(row);
    // (The last block by itself, and no load under a condition: what is on its way is then known, and waited for no earlier than it is needed.)
    auto step = [&](auto next, int j) __attribute__((always_inline)) {
        bf16x8 k[8];
        raw.get(h, k);
        const size_t row_here = row;
        const int page_here = page;
        const float old_here = old;
        if constexpr (decltype(next)::value) {
            page = coming, row = row_at(j + 1, coming);
            raw.load(a.c, row, h);
            old = old_at(row);
            coming = page_at(j + 2);
        }
        f32x16 sc = zero16;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) sc = mfma32(q[ks], k[ks], sc);
        const int key = key_at(j);
        float sum = 0.f, more = 0.f;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float x = fast_exp2(fmaf(sc[e], gm.scale_log2, bias[e])), y = fast_exp2(fmaf(sc[e + 1], gm.scale_log2, bias[e + 1]));
            sum += key <= limit[e] ? x : 0.f;
            more += key <= limit[e + 1] ? y : 0.f;
        }
        sum += more;
        sum += __shfl_xor(sum, 32);
        if (h == 0 && key <= last && (unsigned)page_here < (unsigned)a.c.pages) a.weight[row_here] = a.weight_in && key < s.pos ? fmaf(a.decay, old_here, sum) : sum;
    };
    for (int j = 0; j < count - 1; ++j) step(std::true_type{}, j);
    step(std::false_type{}, count - 1);
}

// Up to 16 rows of a cache of 8 or 4 bits, in tiles of 16 x 16, which do half of what 32 rows do in fewer registers.  (64 tokens behind 8K of 32 / 8 heads in e4m3 93 us for
// 105, in e2m1 57 for 67.)  Lane (n, g) holds key n of either 16
// (and row n), channels 32 g .., which have one exponent; S = Q K^T leaves it with rows 4 g .. 4 g + 3.
template <int BITS>
struct Raw16 {
    u32x4 x[BITS / 4];
    uint32_t exponent;
    __device__ __forceinline__ void load(const Pages& c, size_t row, int g) {
        const char* const p = c.k + row * (kD * BITS / 8) + g * (4 * BITS);
#pragma unroll
        for (int i = 0; i < BITS / 4; ++i) x[i] = *reinterpret_cast<const u32x4*>(p + i * 16);
        exponent = c.ks[row * kRowScales + g];
    }
    __device__ __forceinline__ void get(bf16x8 (&k)[4]) const {
        constexpr int kSlots = 16 / BITS;  // slots of a load
#pragma unroll
        for (int i = 0; i < BITS / 4; ++i) {
            u32x4 y[kSlots];
            dequantise<BITS>(x[i], exponent_value(exponent), y);
#pragma unroll
            for (int j = 0; j < kSlots; ++j) k[i * kSlots + j] = __builtin_bit_cast(bf16x8, y[j]);
        }
    }
};
template <int BITS>
__device__ __forceinline__ void sixteen_part(const WeightsArgs& a, const Part& part) {
    const Geom& gm = a.gm;
    const Seq s = part.s;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, G = gm.G, b = part.b, hk = part.hk, last = s.pos + s.n - 1, rows = s.n * G;
    const bool second = g & 1;  // the own key, whose weight lanes below 32 write: of the second 16
    auto own_of = [second](auto x, auto y) { return second ? y : x; };
    const int r = min(n, rows - 1), tok = r / G;
    const __bf16* const qp = a.q + ((size_t)(s.start + tok) * gm.Hq + hk * G + r - tok * G) * kD + g * 32;
    bf16x8 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const bf16x8*>(qp + 8 * i);
    const float lse = a.lse[(size_t)(hk * G + r - tok * G) * gm.T + s.start + tok];
    const bool counts = n < rows && fabsf(lse) < INFINITY;
    const float my_bias = counts ? -lse * kLog2e : 0.f;
    const int my_limit = counts ? s.pos + tok : -1;
    float bias[4];
    int limit[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[e] = __shfl(my_bias, 4 * g + e), limit[e] = __shfl(my_limit, 4 * g + e);
    struct Keys {
        size_t row0, row1;
        int page0, page1;
    };
    auto key_at = [&](int j, int p) { return (part.block0 + j) * kSub + 16 * p + n; };
    auto in_reach = [&](int j, int p) { return min(key_at(min(j, part.count - 1), p), last); };
    auto find_pages = [&](int j, Keys& at) { at.page0 = page_of(a, b, in_reach(j, 0)), at.page1 = page_of(a, b, in_reach(j, 1)); };
    auto row_at = [&](int page, int key) { return pool_row(a.c, gm.Hkv, plan::clamp(page, 0, a.c.pages - 1), hk, key); };
    auto find_rows = [&](int j, Keys& at) { at.row0 = row_at(at.page0, in_reach(j, 0)), at.row1 = row_at(at.page1, in_reach(j, 1)); };
    Keys here, coming;
    Raw16<BITS> raw[2];
    float old;
    const float* const old_weights = a.weight_in ? a.weight_in : a.weight;
    auto load = [&]() {
        raw[0].load(a.c, here.row0, g), raw[1].load(a.c, here.row1, g);
        old = old_weights[a.weight_in ? own_of(here.row0, here.row1) : 0];
    };
    find_pages(0, here), find_pages(1, coming);
    find_rows(0, here);
    load();
    // (The last block by itself, and no load under a condition: what is on its way is then known, and waited for no earlier than it is needed.)
    auto step = [&](auto more, int j) __attribute__((always_inline)) {
        bf16x8 k[2][4];
        raw[0].get(k[0]), raw[1].get(k[1]);
        const float old_here = old;
        const Keys own = here;
        if constexpr (decltype(more)::value) {
            here = coming;
            find_rows(j + 1, here);
            find_pages(j + 2, coming);
            load();
        }
        f32x4 sc[2];
        mfma16_vgpr_pair<true>(sc[0], sc[1], q, k[0], q, k[1]);
        float sum[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int key = key_at(j, p);
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = fast_exp2(fmaf(sc[p][e], gm.scale_log2, bias[e]));
                x[e] = key <= limit[e] ? y : 0.f;
            }
            sum[p] = (x[0] + x[1]) + (x[2] + x[3]);
        }
        float all = own_of(sum[0], sum[1]) + __shfl_xor(own_of(sum[1], sum[0]), 16);
        all += __shfl_xor(all, 32);
        const int key = key_at(j, second), page = own_of(own.page0, own.page1);
        if (g < 2 && key <= last && (unsigned)page < (unsigned)a.c.pages)
            a.weight[own_of(own.row0, own.row1)] = a.weight_in && key < s.pos ? fmaf(a.decay, old_here, all) : all;
    };
    for (int j = 0; j < part.count - 1; ++j) step(std::true_type{}, j);
    step(std::false_type{}, part.count - 1);
}

// ROWS: how many a KV head of a sequence has at most, 16 or 32.
template <int BITS, int ROWS>
__global__ __launch_bounds__(64 * kWaves, 2) void weights_few_kernel(WeightsArgs a, int b0) {
    __shared__ int ends[kMostSeqs], sums[kWaves];
    const Geom& gm = a.gm;
    const int seqs = min(gm.B - b0, kMostSeqs);
    const int blocks = sum_up(seqs, ends, sums, [&](int i) {
        const Seq s = seq_at(gm, a.c, a.seq_start, a.pos, b0 + i, a.max_new);
        return s.n ? (s.pos + s.n + kSub - 1) / kSub : 0;
    });
    // a stretch of all blocks, sequence by sequence and KV head by KV head
    const long long units = (long long)blocks * gm.Hkv, waves = (long long)gridDim.x * kWaves, w = (long long)blockIdx.x * kWaves + same(threadIdx.x >> 6);
    const int per = (int)((units + waves - 1) / waves);
    long long u = w * per;
    const long long end = u + per < units ? u + per : units;
    if (u >= end) return;
    int i = behind(ends, seqs, (int)(u / gm.Hkv));
    for (; u < end; ++i) {
        // sequence i's part of the stretch
        const int first = i ? ends[i - 1] : 0, its = ends[i] - first, b = b0 + i;
        if (its == 0) continue;
        Seq s = seq_at(gm, a.c, a.seq_start, a.pos, b, a.max_new);
        s = Seq{same(s.start), same(s.n), same(s.pos)};
        while (u < end && u < (long long)ends[i] * gm.Hkv) {
            const int local = same((int)(u - (long long)first * gm.Hkv)), hk = local / its, block0 = local - hk * its;
            const Part part{s, b, hk, block0, same((int)(end - u < its - block0 ? end - u : its - block0))};
            if constexpr (ROWS == 16) sixteen_part<BITS>(a, part);
            else few_part<BITS>(a, part);
            u += part.count;
        }
    }
}

// ---------------------------------------------------------------------------------------
// many rows
// ---------------------------------------------------------------------------------------
constexpr int kChunk = 64 * kWaves;  // keys of a workgroup
constexpr int kPackTokens = 64;      // of a workgroup of the packing kernel
constexpr int kPackThreads = 1024;   // one for each of their rows

// Where a sequence's packed rows begin: whole tiles, one more for each sequence before.
__device__ __forceinline__ int packed_at(const WeightsArgs& a, const Seq& s, int b) { return s.start * a.gm.G / kRows * kRows + b * kRows; }

// Packs the rows with a finite log-sum-exp: a workgroup 64 tokens of a KV head of a sequence, which counts those before them first.
// (Sequence b's workgroups are numbered from start / 64 + b on.)
__global__ __launch_bounds__(kPackThreads) void weights_pack_kernel(WeightsArgs a) {
    __shared__ int sums[kPackThreads / 64], codes[kPackThreads];
    const Geom& gm = a.gm;
    const int hk = blockIdx.y, G = gm.G;
    auto number = [&](int b) { return plan::clamp(a.seq_start[b], 0, gm.T) / kPackTokens + b; };
    int b = 0;
    for (int hi = gm.B - 1; b < hi;) {  // the last one that begins here or before
        const int mid = (b + hi + 1) >> 1;
        if (number(mid) <= (int)blockIdx.x) b = mid;
        else hi = mid - 1;
    }
    const int pair = b * gm.Hkv + hk;
    const Seq s = seq_at(gm, a.c, a.seq_start, a.pos, b, a.max_new);
    const long long from = (long long)((int)blockIdx.x - number(b)) * kPackTokens;
    if (from < 0 || from >= s.n) return;
    const int t0 = (int)from, t1 = min(t0 + kPackTokens, s.n);
    const float* const lse = a.lse + (size_t)hk * G * gm.T + s.start;
    auto counts = [&](int t, int g) { return fabsf(lse[(size_t)g * gm.T + t]) < INFINITY; };
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto all = [&](int x) {  // of all threads
        for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o);
        __syncthreads();
        if (lane == 0) sums[wave] = x;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < kPackThreads / 64; ++w) total += sums[w];
        return total;
    };
    int earlier = 0;
    for (int t = threadIdx.x; t < t0; t += kPackThreads) {
#pragma unroll
        for (int g = 0; g < 16; ++g) earlier += counts(t, min(g, G - 1)) && g < G;  // loads that do not wait for one another
    }
    const int first = all(earlier);
    // a thread per row, in order
    const int t = t0 + (int)threadIdx.x / G, g = (int)threadIdx.x % G;
    const bool on = t < t1 && (int)threadIdx.x < kPackTokens * G, mine = on && counts(t, g);
    const unsigned long long set = __ballot(mine);
    __syncthreads();
    if (lane == 0) sums[wave] = __popcll(set);
    __syncthreads();
    int at = __popcll(set & ((1ull << lane) - 1ull)), here = 0;
    for (int w = 0; w < kPackThreads / 64; ++w) {
        if (w < wave) at += sums[w];
        here += sums[w];
    }
    const size_t base = (size_t)hk * a.cap + packed_at(a, s, b);
    Numbers* const numbers = a.numbers + base / kRows;
    if (mine) {
        codes[at] = t * G + g;
        const int r = first + at;
        numbers[r / kRows].bias[r % kRows] = -lse[(size_t)g * gm.T + t] * kLog2e, numbers[r / kRows].limit[r % kRows] = s.pos + t;
    }
    // chunks of keys whose first key is a new token's: the rows before it
    if (on && g == 0 && (s.pos + t) % kChunk == 0) a.before[(size_t)pair * a.chunks + (s.pos + t) / kChunk - (s.pos + kChunk - 1) / kChunk] = first + at;
    int end = first + here;
    if (t1 == s.n) {  // the last tile is filled up
        const int r = end + (int)threadIdx.x;
        if (r < (end + kRows - 1) / kRows * kRows) numbers[r / kRows].bias[r % kRows] = -INFINITY, numbers[r / kRows].limit[r % kRows] = -1;
        if (threadIdx.x == 0) a.listed[pair] = end;
        end = (end + kRows - 1) / kRows * kRows;
    }
    __syncthreads();
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int i = threadIdx.x >> 4; i < end - first; i += kPackThreads / 16) {
        const int c = threadIdx.x & 15, code = i < here ? codes[i] : 0, tok = code / G;
        const u32x4* const q = reinterpret_cast<const u32x4*>(a.q + ((size_t)(s.start + tok) * gm.Hq + hk * G + code - tok * G) * kD) + c;
        reinterpret_cast<u32x4*>(a.packed + (base + first + i) * kD)[c] = i < here ? *q : zero;
    }
}

// What a chunk takes on the line besides its tiles: loading (and converting) its keys, in tiles.
template <int BITS>
constexpr int kStart = 2 + BITS / 4;

// Tiles before boundary x of a chunk that begins at `start`.  Boundaries next to an end of a chunk move there.
template <int BITS>
__device__ __forceinline__ int tiles_before(long long x, long long start, int tiles) {
    const long long at = x - start - kStart<BITS>;
    return at <= 1 ? 0 : at >= tiles - 1 ? tiles : (int)at;
}
struct PairWork {
    int chunks, plain, tiles;  // chunks of keys; those before the first that begins with a new token's key; tiles of rows
};
__device__ __forceinline__ PairWork pair_work(const WeightsArgs& a, int pair, const Seq& s) {
    PairWork p;
    p.chunks = s.n ? (s.pos + s.n + kChunk - 1) / kChunk : 0;
    p.plain = min((s.pos + kChunk - 1) / kChunk, p.chunks);
    p.tiles = s.n ? (plan::clamp(a.listed[pair], 0, s.n * a.gm.G) + kRows - 1) / kRows : 0;
    return p;
}
// The first tile with a row that sees a key of chunk j.
__device__ __forceinline__ int first_tile(const WeightsArgs& a, int pair, const PairWork& p, int j) {
    return j < p.plain ? 0 : plan::clamp(a.before[(size_t)pair * a.chunks + j - p.plain] / kRows, 0, p.tiles);
}

constexpr int kMostPairs = 1024;  // of a launch
constexpr int kFour = 1024 + 16;  // 4 rows of 256 bytes in shared memory, and 16: see attn_extend_bf16.hip
constexpr int kTileBytes = kRows / 4 * kFour;
constexpr int kRing = 3;

template <int BITS>
__global__ __launch_bounds__(64 * kWaves, 3) void weights_many_kernel(WeightsArgs a, int pair0) {
    __shared__ __attribute__((aligned(16))) char ring[kRing * kTileBytes];
    __shared__ __attribute__((aligned(16))) Numbers number_ring[kRing];
    __shared__ long long ends[kMostPairs];
    __shared__ long long sums[kWaves];
    const Geom& gm = a.gm;
    const int pairs = min(gm.B * gm.Hkv - pair0, kMostPairs), lane = threadIdx.x & 63, wave = same(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
    auto seq = [&](int pair) { return seq_at(gm, a.c, a.seq_start, a.pos, pair / gm.Hkv, a.max_new); };
    long long total = 0;
    for (int p0 = 0; p0 < pairs; p0 += 64 * kWaves) {  // the line
        const int i = p0 + (int)threadIdx.x;
        long long upto = 0;
        if (i < pairs) {
            const PairWork p = pair_work(a, pair0 + i, seq(pair0 + i));
            upto = (long long)p.plain * (p.tiles + kStart<BITS>);
            for (int j = p.plain; j < p.chunks; ++j) upto += p.tiles - first_tile(a, pair0 + i, p, j) + kStart<BITS>;
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const long long below = __shfl_up(upto, o);
            if (lane >= o) upto += below;
        }
        __syncthreads();
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) upto += sums[w];
        }
        if (i < pairs) ends[i] = total + upto;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += sums[w];
    }
    __syncthreads();
    const int w = (int)(blockIdx.x & 7) * (a.workgroups >> 3) + (int)(blockIdx.x >> 3);  // neighbours on one XCD
    if (threadIdx.x == 0) a.open[w].pair = -1;
    const long long per = (total + a.workgroups - 1) / a.workgroups, x0 = w * per, x1 = x0 + per < total ? x0 + per : total;
    if (x0 >= x1) return;
    const lds_cptr tile_at = (lds_cptr)(uintptr_t)(lds_offset(ring) + (n >> 2) * kFour + (n & 3) * 64);
    const unsigned ring_at = lds_offset(ring) + wave * 2 * kFour, numbers_at = lds_offset(number_ring);
    int i = 0;
    {
        int hi = pairs - 1;
        while (i < hi) {
            const int mid = (i + hi) >> 1;
            if (ends[mid] > x0) hi = mid;
            else i = mid + 1;
        }
    }
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (i = same(i); i < pairs; ++i) {
        long long start = i ? ends[i - 1] : 0;
        if (start >= x1) break;
        const int pair = pair0 + i, b = pair / gm.Hkv, hk = pair - b * gm.Hkv;
        Seq s = seq(pair);
        s = Seq{same(s.start), same(s.n), same(s.pos)};
        PairWork pw = pair_work(a, pair, s);
        pw.tiles = same(pw.tiles);
        const int last = s.pos + s.n - 1;
        const size_t base = (size_t)hk * a.cap + packed_at(a, s, b);
        int j = 0;
        if (x0 > start) {  // whole chunks before this stretch
            const long long each = pw.tiles + kStart<BITS>, skip = (x0 - start) / each;
            j = skip < pw.plain ? (int)skip : pw.plain;
            start += j * each;
        }
        for (j = same(j); j < pw.chunks; ++j) {
            const int t_first = same(first_tile(a, pair, pw, j)), tiles = pw.tiles - t_first;
            const long long begin = start, end = start + tiles + kStart<BITS>;
            if (begin >= x1) break;
            start = end;
            if (end <= x0) continue;
            const int from = x0 <= begin ? 0 : tiles_before<BITS>(x0, begin, tiles), to = x1 >= end ? tiles : tiles_before<BITS>(x1, begin, tiles);
            if (from >= to && !(tiles == 0 && x0 <= begin)) continue;
            // ---- the chunk's keys, 64 a wavefront, while the first tiles come
            const int key0 = j * kChunk;
            auto issue = [&](int t) {  // tile t of the piece
                const size_t row = base + (size_t)(t_first + from + t) * kRows;
                const char* const q = (const char*)(a.packed + row * kD) + wave * 2048;
                const unsigned slot = t % kRing, off = ((lane >> 2) & 3) * 256 + (lane >> 4) * 64 + (lane & 3) * 16;
#pragma unroll
                for (int e = 0; e < 2; ++e) dma16_so(q + e * 1024, off, ring_at + slot * kTileBytes + e * kFour);
                dma4_so(a.numbers + row / kRows, lane * 4, numbers_at + slot * (unsigned)sizeof(Numbers));
            };
            const int count = to - from;
            bf16x8 k[2][8];
            size_t rows[2];
            bool real[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const int key = key0 + wave * 64 + kb * 32 + n, mine = min(key, last), page = page_of(a, b, mine);
                rows[kb] = pool_row(a.c, gm.Hkv, plan::clamp(page, 0, a.c.pages - 1), hk, mine);
                real[kb] = key <= last && (unsigned)page < (unsigned)a.c.pages;
                RawKeys<BITS> raw;
                raw.load(a.c, rows[kb], h);
                raw.get(h, k[kb]);
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) asm volatile("" : "+v"(k[kb][ks]));  // waited for here, and so not in the loop, behind its loads
            }
            __syncthreads();  // the ring is free
            if (count > 0) issue(0);
            if (count > 1) issue(1);
            float sum[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
            // (The weights of a tile between the matrix instructions of the next, slot by slot, take as long: the chip's clock falls with what it does at once.)
            for (int t = 0; t < count; ++t) {
                if (t + 1 < count) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
                else dma_wait();
                __syncthreads();
                if (t + 2 < count) issue(t + 2);
                const int slot = t % kRing;
                const lds_cptr at = tile_at + slot * kTileBytes;
                bf16x8 q[8];
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    const int c = slot_channel<BITS>(ks, h) / 8;
                    q[ks] = *(const __attribute__((address_space(3))) bf16x8*)(at + (c >> 2) * 256 + (c & 3) * 16);
                }
                const Numbers& nr = number_ring[slot];
                float bias[16];
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(nr.bias + c_row(e, h));
                    bias[e] = x[0], bias[e + 1] = x[1], bias[e + 2] = x[2], bias[e + 3] = x[3];
                }
                const bool whole = min(nr.limit[0], nr.limit[kRows - 1]) >= key0 + kChunk - 1;  // (ascending but for padding)
                f32x16 sc[2] = {zero16, zero16};
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) sc[kb] = mfma32(q[ks], k[kb][ks], sc[kb]);
                if (same(whole)) {
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int e = 0; e < 16; ++e) sum[kb][e & 3] += fast_exp2(fmaf(sc[kb][e], gm.scale_log2, bias[e]));
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int limit = nr.limit[c_row(e, h)];
#pragma unroll
                        for (int kb = 0; kb < 2; ++kb) {
                            const float x = fast_exp2(fmaf(sc[kb][e], gm.scale_log2, bias[e]));
                            sum[kb][e & 3] += key0 + wave * 64 + kb * 32 + n <= limit ? x : 0.f;
                        }
                    }
                }
            }
            // ---- out
            const bool begins = from == 0, finishes = to == tiles;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                float x = (sum[kb][0] + sum[kb][1]) + (sum[kb][2] + sum[kb][3]);
                x += __shfl_xor(x, 32);
                const int in = wave * 64 + kb * 32 + n;
                if (h != 0) continue;
                if (!begins || !finishes) {
                    a.slots[((size_t)w * 2 + (begins ? 1 : 0)) * kChunk + in] = x;
                } else if (real[kb]) {
                    if (a.weight_in && key0 + in < s.pos) x = fmaf(a.decay, a.weight_in[rows[kb]], x);
                    a.weight[rows[kb]] = x;
                }
            }
            if (begins && !finishes && threadIdx.x == 0) a.open[w] = Open{begin, per, tiles, pair, j, 0};
        }
    }
}

// Joins what several workgroups have of a chunk: a workgroup for each that begins one and does not end it.
template <int BITS>
__global__ __launch_bounds__(kChunk) void weights_join_kernel(WeightsArgs a) {
    const int w = blockIdx.x;
    const Open o = a.open[w];
    if (o.pair < 0) return;
    float sum = a.slots[((size_t)w * 2 + 1) * kChunk + threadIdx.x];
    const long long end = o.start + o.tiles + kStart<BITS>;
    constexpr int kAhead = 8;  // loads on their way together
    for (int v = w + 1, to = 0; to < o.tiles && v < a.workgroups; v += kAhead) {
        float x[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const long long x0 = (v + e) * o.per, x1 = x0 + o.per;
            const int from = x0 >= end ? o.tiles : tiles_before<BITS>(x0, o.start, o.tiles);
            to = x1 >= end ? o.tiles : tiles_before<BITS>(x1, o.start, o.tiles);
            x[e] = from < to && v + e < a.workgroups ? a.slots[(size_t)(v + e) * 2 * kChunk + threadIdx.x] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) sum += x[e];
    }
    const int b = o.pair / a.gm.Hkv, hk = o.pair - b * a.gm.Hkv, key = o.chunk * kChunk + (int)threadIdx.x;
    const Seq s = seq_at(a.gm, a.c, a.seq_start, a.pos, b, a.max_new);
    if (key >= s.pos + s.n) return;
    const int page = page_of(a, b, key);
    if ((unsigned)page >= (unsigned)a.c.pages) return;
    const size_t row = pool_row(a.c, a.gm.Hkv, page, hk, key);
    if (a.weight_in && key < s.pos) sum = fmaf(a.decay, a.weight_in[row], sum);
    a.weight[row] = sum;
}

// Two to four on a CU.  Few rows, 64 tokens behind 8K of 32 / 8 heads (4 rows) by 512, 768 and 1024 workgroups: in e4m3 101, 93 and 96 us, in e2m1 68, 59 and 57; in bf16 with
// tiles of 16 rows 187, 175 and 175, of 32, by 512, 170.  20 rows, 30 sequences of 15K of 16 / 4 heads, by 512 and 768: in e4m3 50 and 48, in e2m1 30 and 29.  Many rows 267 with two, 251 with three.
constexpr int kManyWorkgroups = 768;
template <int BITS, int ROWS>
constexpr int kFewWorkgroups = BITS == 16 ? 512 : BITS == 4 && ROWS == 16 ? 1024 : 768;
bool few(const Geom& g, int max_new) { return (long long)(max_new < g.T ? max_new : g.T) * g.G <= kRows; }

// The workspace: sub-buffers at multiples of 256 bytes.
size_t lay_out(WeightsArgs& a, char* base) {
    const Geom& g = a.gm;
    if (few(g, a.max_new)) return 0;
    size_t at = 0;
    auto take = [&](auto*& p, size_t count) {
        p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += (count * sizeof(*p) + 255) / 256 * 256;
    };
    a.cap = g.T * g.G / kRows * kRows + g.B * kRows;
    a.chunks = (a.max_new < g.T ? a.max_new : g.T) / kChunk + 2;
    a.workgroups = kManyWorkgroups;
    const size_t pairs = (size_t)g.B * g.Hkv;
    take(a.listed, pairs);
    take(a.before, pairs * a.chunks);
    take(a.packed, (size_t)g.Hkv * a.cap * kD);
    take(a.numbers, (size_t)g.Hkv * a.cap / kRows);
    take(a.open, a.workgroups);
    take(a.slots, (size_t)a.workgroups * 2 * kChunk);
    return at;
}

}  // namespace

size_t weights_workspace(const Geom& g, int max_new) {
    WeightsArgs a{};
    a.gm = g, a.max_new = max_new;
    return lay_out(a, nullptr);
}

int cache_weights(const Geom& g, const Pages& c, const void* q, const int32_t* seq_start, const int32_t* pos, const float* lse, int max_new,
                  float decay, const float* weight_in, float* weight, void* workspace, hipStream_t st) {
    WeightsArgs a{g, c, (const __bf16*)q, seq_start, pos, lse, max_new, decay, weight_in, weight};
    lay_out(a, (char*)workspace);
    auto launch = [&](auto bits) {
        constexpr int BITS = decltype(bits)::value;
        if (few(g, max_new)) {
            KernelTimer kt("cache_weights", st);
            auto launch_few = [&](auto rows) {
                constexpr int ROWS = decltype(rows)::value;
                for (int b0 = 0; b0 < g.B; b0 += kMostSeqs)
                    hipLaunchKernelGGL((weights_few_kernel<BITS, ROWS>), dim3(kFewWorkgroups<BITS, ROWS>), dim3(64 * kWaves), 0, st, a, b0);
            };
            if (BITS < 16 && (long long)max_new * g.G <= 16) launch_few(std::integral_constant<int, BITS < 16 ? 16 : kRows>{});
            else launch_few(std::integral_constant<int, kRows>{});
            return;
        }
        {
            KernelTimer kt("weights_pack", st);
            hipLaunchKernelGGL(weights_pack_kernel, dim3(g.T / kPackTokens + g.B, g.Hkv), dim3(kPackThreads), 0, st, a);
        }
        for (int pair0 = 0; pair0 < g.B * g.Hkv; pair0 += kMostPairs) {
            {
                KernelTimer kt("cache_weights", st);
                hipLaunchKernelGGL(weights_many_kernel<BITS>, dim3(a.workgroups), dim3(64 * kWaves), 0, st, a, pair0);
            }
            KernelTimer kt("weights_join", st);
            hipLaunchKernelGGL(weights_join_kernel<BITS>, dim3(a.workgroups), dim3(kChunk), 0, st, a);
        }
    };
    if (c.bits == 16) launch(std::integral_constant<int, 16>{});
    else if (c.bits == 8) launch(std::integral_constant<int, 8>{});
    else launch(std::integral_constant<int, 4>{});
    return launch_status();
}

}  // namespace l2a
