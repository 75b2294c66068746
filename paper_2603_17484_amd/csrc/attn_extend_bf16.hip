// Attention of new tokens over a paged KV cache (bf16 on the matrix cores, D = 128): chunks of a prompt behind a cached prefix,
// drafts of a few tokens, single tokens, packed one sequence behind the other.
//
// A routed row's Global attention covers its window too, with the same scores.  So rows are not computed for each branch, but for
// each part of their keys: the window's (all rows) and those before it (routed rows that have some).  With (m, l, u) the
// maximum, sum and weighted sum of V of each part,
//     s = u_w / l_w,   a = (2^(m_w - m) u_w + 2^(m_p - m) u_p) / (2^(m_w - m) l_w + 2^(m_p - m) l_p),  m = max(m_w, m_p),
// and the window's keys are read and multiplied once for both branches.
//
//   extend_list_kernel     a workgroup per KV head of a sequence: its rows with keys before the window, ascending
//   extend_plan_kernel     one workgroup: the tiles (up to 32 NW rows of a KV head of a sequence, of one part) on a line, by their blocks
//                          of 64 keys, and which tile each workgroup of the next kernel begins in (extend_plan.hpp)
//   extend_kernel          every workgroup an equal stretch of that line: S^T = K Q^T, streaming softmax, O^T += V^T P^T.  Rows
//                          whose parts are complete are written out, sums of the others go to the workspace
//   extend_combine_kernel  joins these
// Calls in which no sequence has more than 128 rows per KV head make no lists, and with up to 512 KV heads of sequences every workgroup
// makes the plan for itself (extend_short_kernel, extend_combine_short_kernel): two launches instead of four, 25 us for a token behind 32K.
//
// Measured (us; one call among others on one card, "main" the kernel that attends): 64 tokens behind 8K in e4m3, 610 MB of cache, 126 (main 118: 5.3
// TB/s); 16 x 5 behind 32K 106; a token behind 32K 24 (18); 2048 behind 32K 338 (331), 4096 behind 124K 1697 (1642: 1.04 PFLOP/s, 1577 to 1734 from
// card to card; products of 8192 x 8192 matrices reach 1.28 with nothing between them); 128 behind 64K 98; 1000 beside 31 single ones at 16K 169 (142);
// 3 x 777 first tokens 61 (38).  Before the main kernel: lists 5 to 11, plan 7 to 14; behind it: sums joined, 6 to 27.
#include "paged.hpp"
#include "tiles.hpp"

namespace l2a {
namespace {

using plan::kKeys;
using plan::Pieces;
using plan::Place;
using plan::Range;
using plan::Seq;

constexpr int kPart = kD + 4;  // floats of a row's sums: maximum (log2 units), sum, 2 unused, O[128]

struct Tile {  // 64 bytes
    long long start;  // on the line
    int blocks, skip;  // there; blocks before these, which are segments
    int b, hk, kind;  // plan::kWindow or kPrefix
    int first, rows;  // of the sequence's rows, or of its list
    int lo, hi;       // keys
    int pos0, pos1;   // positions of the first and last row
    Seq s;
};
struct Pair {  // a KV head of a sequence
    int first_tile, listed;      // its first tile, windows first; rows with keys before the window
    int segments, first_segment; // of each of its tiles of many rows with keys before the window; the first of them
};
struct Short {  // a KV head of a sequence in a call without lists: all that the last kernel has to know
    Seq s;
    int pad;
    Place place[2];  // of its tiles on the line, by kind
};
struct Head {
    long long total;     // length of the line
    int per, tiles;      // its stretches; tiles on it
    int segments, pad;   // workgroups that have a segment
};
struct Segment {
    int tile, from, to;  // blocks, counted from the tile's first key on
};

struct ExtendArgs {
    Geom gm;             // gm.T = packed tokens; gm.W = -1: no Local branch
    Pages c;
    const __bf16* q;     // [T, Hq, D]
    const int32_t *seq_start, *pos;
    const uint8_t* mask;  // [mask_heads, T]; nullptr: every token routed
    int mask_heads, do_local, do_global, max_new;
    __bf16 *O, *S, *A;   // [T, Hq, D]
    float *lse_l, *lse_g;  // [Hq, T]
    // workspace
    Head* head;
    Tile* tiles;
    int most_tiles, workgroups, tile_rows, few;  // few: no sequence has more than 128 rows per KV head, and no lists are made
    int32_t* first_tile;  // [workgroups] of a stretch
    Segment* segment;     // [workgroups]
    Pair* pairs;          // [B * Hkv]
    Short* shorts;        // [B * Hkv] (few)
    int32_t* list;        // [Hkv][T G], a sequence's from its first row on: codes of the rows with keys before the window, ascending
    int32_t* rank;        // [Hkv][T G] place of a row in its list
    int32_t* token_seq;   // [T] (few)
    float* slots;         // [2 * workgroups][tile_rows][kPart]
    float* parts[2];      // [T * Hq][kPart]: rows of whole tiles, by kind
};

__device__ __forceinline__ Seq seq_of(const ExtendArgs& a, int b) { return seq_at(a.gm, a.c, a.seq_start, a.pos, b, a.max_new); }
__device__ __forceinline__ bool token_routed(const ExtendArgs& a, int token, int head) {
    if (!a.do_global) return false;
    if (!a.mask) return true;
    const int mh = a.mask_heads == 1 ? 0 : (a.mask_heads == a.gm.Hq ? head : head / a.gm.G);
    return a.mask[(size_t)mh * a.gm.T + token] != 0;
}
__device__ __forceinline__ Place place_of(const ExtendArgs& a, const Tile& t) { return Place{t.start, t.blocks, plan::block_cost(t.rows, a.c.fp8)}; }
// The decisions of a token for the heads of a KV head's group, a bit each.
__device__ __forceinline__ unsigned group_routed(const ExtendArgs& a, int token, int hk) {
    const int G = a.gm.G;
    const unsigned all = (1u << G) - 1u;
    if (!a.do_global) return 0u;
    if (!a.mask) return all;
    if (a.mask_heads != a.gm.Hq || G == 1) return token_routed(a, token, hk * G) ? all : 0u;
    const uint8_t* p = a.mask + (size_t)hk * G * a.gm.T + token;
    unsigned bits = 0;
#pragma unroll
    for (int g = 0; g < 16; ++g)  // the bytes' loads do not wait for one another
        bits |= (unsigned)(g < G && p[(size_t)min(g, G - 1) * a.gm.T] != 0) << g;
    return bits;
}
// Whether a row of a KV head is routed and has keys before its window.
__device__ __forceinline__ bool has_prefix(const ExtendArgs& a, const Seq& s, int hk) {
    unsigned any = 0;
#pragma unroll 4
    for (int t = plan::rows_without_prefix(s, 1, a.gm.W); t < s.n; ++t) any |= group_routed(a, s.start + t, hk);
    return any != 0;
}
__device__ __forceinline__ int window_tiles(const ExtendArgs& a, const Seq& s) {
    return a.do_local ? (s.n * a.gm.G + a.tile_rows - 1) / a.tile_rows : 0;
}
__device__ __forceinline__ int32_t* list_of(const ExtendArgs& a, int32_t* x, const Seq& s, int hk) {
    return x + (size_t)hk * a.gm.T * a.gm.G + (size_t)s.start * a.gm.G;
}

// The code (token in the sequence, head in the group) of row i of a tile's kind.
__device__ __forceinline__ int row_code(const ExtendArgs& a, const Tile& t, int i) {
    if (a.few || t.kind == plan::kWindow) return i;
    return plan::clamp(list_of(a, a.list, t.s, t.hk)[i], 0, t.s.n * a.gm.G - 1);
}
// A row's result: s (x), a (y), their log-sum-exps, four channels a lane
__device__ __forceinline__ void store_row(const ExtendArgs& a, int token, int head, int c4, const f32x4& x, const f32x4& y, float lse_l, float lse_g) {
    const size_t off = ((size_t)token * a.gm.Hq + head) * kD + c4;
    *reinterpret_cast<bf16x4*>(a.O + off) = __builtin_convertvector(x + y, bf16x4);
    if (a.S) *reinterpret_cast<bf16x4*>(a.S + off) = __builtin_convertvector(x, bf16x4);
    if (a.A) *reinterpret_cast<bf16x4*>(a.A + off) = __builtin_convertvector(y, bf16x4);
    if (c4 == 0) {
        const size_t so = (size_t)head * a.gm.T + token;
        if (a.lse_l) a.lse_l[so] = lse_l;
        if (a.lse_g) a.lse_g[so] = lse_g;
    }
}

// A thread per token, a round for every kListThreads of them: decisions counted, the counts summed over the workgroup, the rows written.
constexpr int kListThreads = 1024;
__global__ __launch_bounds__(kListThreads) void extend_list_kernel(ExtendArgs a) {
    __shared__ int sums[2][kListThreads / 64];
    const Geom& gm = a.gm;
    const int b = blockIdx.x / gm.Hkv, hk = blockIdx.x - b * gm.Hkv, G = gm.G;
    const Seq s = seq_of(a, b);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, skip = plan::rows_without_prefix(s, 1, gm.W);
    int32_t *list = list_of(a, a.list, s, hk), *rank = list_of(a, a.rank, s, hk);
    int total = 0;
    auto decisions = [&](int t) { return t < s.n ? group_routed(a, s.start + t, hk) : 0u; };
    unsigned bits = decisions(skip + (int)threadIdx.x);
    for (int t0 = skip, turn = 0; t0 < s.n; t0 += kListThreads, turn ^= 1) {
        const int t = t0 + (int)threadIdx.x, count = __popc(bits);
        const unsigned coming = decisions(t + kListThreads);
        int upto = count;  // of this wavefront's lanes up to this one
        for (int o = 1; o < 64; o <<= 1) {
            const int below = __shfl_up(upto, o);
            if (lane >= o) upto += below;
        }
        if (lane == 63) sums[turn][wave] = upto;
        __syncthreads();
        int at = total + upto - count;
        for (int w = 0; w < kListThreads / 64; ++w) {
            if (w < wave) at += sums[turn][w];
            total += sums[turn][w];
        }
        for (; bits; bits &= bits - 1) {
            const int code = t * G + __ffs((int)bits) - 1;
            rank[code] = at;
            list[at++] = code;
        }
        bits = coming;
    }
    if (threadIdx.x == 0) a.pairs[blockIdx.x].listed = total;
    if (a.do_local) return;
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};  // without windows, rows that are not routed have no tile
    for (int r = threadIdx.x >> 5; r < s.n * G; r += kListThreads / 32)
        if (!token_routed(a, s.start + r / G, hk * G + r % G)) store_row(a, s.start + r / G, hk * G + r % G, (threadIdx.x & 31) * 4, z, z, -INFINITY, -INFINITY);
}

// Sum over the threads before this one, and over all of them.
template <int THREADS, typename X>
__device__ __forceinline__ void scan(X x, X* sums, X& before, X& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    X upto = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const X below = __shfl_up(upto, o);
        if (lane >= o) upto += below;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    before = upto - x, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
}
// A tile of a kind that begins at row `first`.
__device__ __forceinline__ Tile make_tile(const ExtendArgs& a, const Seq& s, int b, int hk, int kind, int first, int of) {
    Tile t{};
    t.b = b, t.hk = hk, t.s = s, t.kind = kind, t.first = first, t.rows = min(a.tile_rows, of - first);
    t.pos0 = s.pos + row_code(a, t, first) / a.gm.G, t.pos1 = s.pos + row_code(a, t, first + t.rows - 1) / a.gm.G;
    const Range k = plan::tile_keys(kind, t.pos0, t.pos1, a.gm.W);
    t.lo = k.lo, t.hi = k.hi;
    t.blocks = plan::tile_blocks(k);
    return t;
}
// A thread per KV head of a sequence, then one per tile, then one per stretch's beginning.
// (1024 threads: 11.4 us for 10.1 at 2048 tokens behind 32K and 7.7 for 7.0 at 3 x 777, as fewer wavefronts meet faster; 12.8 for 14.6 with
// 900 tiles, a second round of them.  256: 12.3, 8.5 and 16.6.)
constexpr int kPlanThreads = 512;
__global__ __launch_bounds__(kPlanThreads) void extend_plan_kernel(ExtendArgs a) {
    __shared__ int sums[kPlanThreads / 64];
    __shared__ unsigned lengths[kPlanThreads / 64];  // (a round's tiles together are shorter than 2^32)
    __shared__ int ends[kPlanThreads];  // tiles up to and with a pair, of the pairs at hand
    const Geom& gm = a.gm;
    const int pairs = gm.B * gm.Hkv, G = gm.G;
    int tiles = 0;        // of the pairs before
    long long line = 0;   // where the next tile begins
    for (int p0 = 0; p0 < pairs; p0 += kPlanThreads) {
        const int mine = p0 + (int)threadIdx.x;
        int count = 0, listed = 0;
        if (mine < pairs) {
            const int b = mine / gm.Hkv, hk = mine - b * gm.Hkv;
            const Seq s = seq_of(a, b);
            if (a.few) {  // one tile of all the sequence's rows
                listed = has_prefix(a, s, hk) ? s.n * G : 0;
                a.shorts[mine].s = s;
                if (hk == 0)
                    for (int i = 0; i < s.n; ++i) a.token_seq[s.start + i] = b;
            } else {
                listed = min(a.pairs[mine].listed, s.n * G);
            }
            count = window_tiles(a, s) + (listed + a.tile_rows - 1) / a.tile_rows;
        }
        int before, here;
        scan<kPlanThreads>(count, sums, before, here);
        if (mine < pairs) a.pairs[mine] = Pair{tiles + before, listed, 0, 0};
        ends[threadIdx.x] = before + count;
        __syncthreads();
        const int of = min(pairs - p0, kPlanThreads);
        for (int i0 = 0; i0 < here && tiles + i0 < a.most_tiles; i0 += kPlanThreads) {  // (more: sequences that overlap)
            const int i = i0 + (int)threadIdx.x;
            Tile t{};
            const bool on = i < here && tiles + i < a.most_tiles;
            if (on) {
                int lo = 0, hi = of - 1;  // the first pair that ends behind tile i
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (ends[mid] > i) hi = mid;
                    else lo = mid + 1;
                }
                const int b = (p0 + lo) / gm.Hkv, hk = p0 + lo - b * gm.Hkv;
                const Seq s = seq_of(a, b);
                const int w = window_tiles(a, s), within = i - (lo ? ends[lo - 1] : 0);
                if (within < w) t = make_tile(a, s, b, hk, plan::kWindow, within * a.tile_rows, s.n * G);
                else t = make_tile(a, s, b, hk, plan::kPrefix, (within - w) * a.tile_rows, a.pairs[p0 + lo].listed);
            }
            unsigned at, sum;
            scan<kPlanThreads>(on ? (unsigned)place_of(a, t).length() : 0u, lengths, at, sum);
            if (on) {
                t.start = line + at;
                a.tiles[tiles + i] = t;
                if (a.few) a.shorts[t.b * gm.Hkv + t.hk].place[t.kind] = place_of(a, t);
            }
            line += sum;
        }
        tiles = min(tiles + here, a.most_tiles);
        __syncthreads();
    }
    const int dearest = plan::block_cost(a.tile_rows, a.c.fp8);
    int per = plan::stretch(line, a.workgroups, dearest), segments = 0;
    const int segment = plan::segment_blocks(per, dearest);
    if (!a.few && a.do_global && segment) {
        for (int p0 = 0; p0 < pairs; p0 += kPlanThreads) {  // how many each pair has
            const int mine = p0 + (int)threadIdx.x;
            int each = 0, of = 0;
            if (mine < pairs) {
                const Pair p = a.pairs[mine];
                const int first = p.first_tile + window_tiles(a, seq_of(a, mine / gm.Hkv));
                of = plan::many_tiles(p.listed, a.tile_rows);
                if (of && first + of <= tiles) each = plan::segments(a.tiles[first].blocks, segment);
            }
            int before, here;
            scan<kPlanThreads>(each * of, sums, before, here);
            if (mine < pairs) a.pairs[mine].segments = each, a.pairs[mine].first_segment = segments + before;
            segments += here;
        }
        __syncthreads();
        if (segments >= a.workgroups) {  // (lists that others wrote over, of sequences that overlap: a first tile that is not its pair's shortest)
            for (int i = threadIdx.x; i < pairs; i += kPlanThreads) a.pairs[i].segments = 0;
            segments = 0;
            __syncthreads();
        }
        line = 0;
        for (int i0 = 0; i0 < tiles; i0 += kPlanThreads) {  // which they are, and the line without them
            const int i = i0 + (int)threadIdx.x;
            Tile t{};
            if (i < tiles) {
                t = a.tiles[i];
                const Pair p = a.pairs[t.b * gm.Hkv + t.hk];
                const int of = plan::many_tiles(p.listed, a.tile_rows), j = t.first / a.tile_rows;
                if (t.kind == plan::kPrefix && j < of && p.segments) {
                    t.skip = p.segments * segment;
                    t.blocks = max(t.blocks - t.skip, 0);
                    for (int k = 0; k < p.segments; ++k) {
                        const int w = plan::segment_workgroup(p.first_segment, of, k, j);
                        if (w < a.workgroups) a.segment[w] = Segment{i, k * segment, (k + 1) * segment};
                    }
                }
                t.start = 0;
            }
            unsigned at, sum;
            scan<kPlanThreads>(i < tiles ? (unsigned)place_of(a, t).length() : 0u, lengths, at, sum);
            if (i < tiles) a.tiles[i].start = line + at, a.tiles[i].blocks = t.blocks, a.tiles[i].skip = t.skip;
            line += sum;
        }
        per = plan::stretch(line, max(a.workgroups - segments, 1), dearest);
    }
    if (threadIdx.x == 0) *a.head = Head{line, per, tiles, segments, 0};
    __syncthreads();
    // the tile each stretch begins in
    for (int i = threadIdx.x; i < tiles; i += kPlanThreads) {
        const Place p = place_of(a, a.tiles[i]);
        for (long long w = plan::workgroup_at(p.start + per - 1, per); w * per < p.end() && w < a.workgroups; ++w) a.first_tile[w] = i;
    }
}

// Blocks of keys in shared memory: 4 rows of 256 bytes, the keys of one load instruction, are 1024 bytes; the next 4 follow kFour
// further on.  Within them the 16-byte chunk c of row r lies at 256 (c / 4) + 64 r + 16 (c mod 4).  Both ways of reading, K's rows 16 bytes
// a lane and V's columns through the transposing read, touch every bank once, and an operand's place is one lane's number
// plus constants: they are the instructions' offsets.  (With the chunks of a row permuted by an exclusive or instead, a block's operands took 16
// registers and as many additions.)
constexpr int kFour = 1024 + 16;
constexpr int kBlockBytes = kKeys / 4 * kFour;
__device__ __forceinline__ constexpr int chunk_at(int row, int c) { return (row >> 2) * kFour + (row & 3) * 64 + (c >> 2) * 256 + (c & 3) * 16; }
// this lane's part of the places, and the operands: 16 channels 16 ks .. of rows 32 half .. ; 32 channels 32 d .. of rows 16 step ..
__device__ __forceinline__ unsigned k_lane(int lane) { return chunk_at(lane & 31, lane >> 5); }
__device__ __forceinline__ unsigned v_lane(int lane) {
    const int i = lane & 15;
    return (lane >> 5) * kFour + (i >> 2) * 64 + ((lane >> 4) & 1) * 32 + (i & 3) * 8;
}
__device__ __forceinline__ bf16x8 k_operand(lds_cptr at, int ks, int half) {
    return *(const __attribute__((address_space(3))) bf16x8*)(at + half * 8 * kFour + (ks >> 1) * 256 + (ks & 1) * 32);
}
__device__ __forceinline__ bf16x8 v_operand(lds_cptr at, int d, int step) {
    typedef s16x4 __attribute__((address_space(3)))* lds_ptr;
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + d * 256 + step * 4 * kFour));
    const s16x4 v2 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + d * 256 + (step * 4 + 2) * kFour));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v1, v2, 0, 1, 2, 3, 4, 5, 6, 7));
}
// The row and the 16 bytes of it that a lane loads, of the 4 (e4m3: 8) rows of an instruction.  e4m3: so that a lane's 16 elements become
// two chunks whose stores, eight lanes at a time, touch no bank twice.  (Counted: conflicts in 5 to 7 % of the cycles even so; none in bf16.)
template <bool FP8>
__device__ __forceinline__ int load_row(int lane) { return FP8 ? ((lane >> 1) & 3) + 4 * (lane >> 5) : (lane >> 2) & 3; }
template <bool FP8>
__device__ __forceinline__ int load_chunk(int lane) { return FP8 ? (lane & 1) + 2 * ((lane >> 3) & 3) : (lane >> 4) * 4 + (lane & 3); }
// e4m3: a lane's 16 elements of `row`, with the exponents of the row, become bf16
typedef __attribute__((address_space(3))) char* lds_ptr;
__device__ __forceinline__ void store_converted(const u32x4& x, uint32_t exponents, lds_ptr block, int row, int lane) {
    const int c = load_chunk<true>(lane);
    u32x4 y[2];
    dequantise16(x, exponent_value((exponents >> (8 * (c >> 1))) & 0xffu), y);
    __attribute__((address_space(3))) u32x4* const at = (__attribute__((address_space(3))) u32x4*)(block + chunk_at(row, 2 * c));
    at[0] = y[0], at[1] = y[1];
}

// Shared memory of a workgroup of NW wavefronts, in bytes from its beginning: rings of blocks of K and of V; e4m3: rings of what was loaded
// (K, V, their exponents: every wavefront's pieces its own, which it alone converts) and of the bf16 blocks made of it.  Blocks are
// loaded two walks of the loop ahead of their use.
template <bool FP8, int NW>
struct Lds {
    static constexpr int kK = FP8 ? 3 : 4, kV = FP8 ? 3 : 4, kRaw = 2;
    static constexpr unsigned k = 0, v = k + kK * kBlockBytes, raw_k = v + kV * kBlockBytes;
    static constexpr unsigned kRawBlock = kKeys * kD, kRawScales = kKeys / 8 * 256;
    static constexpr unsigned raw_v = raw_k + kRaw * kRawBlock, raw_ks = raw_v + kRaw * kRawBlock, raw_vs = raw_ks + kRaw * kRawScales;
    static constexpr unsigned used = FP8 ? raw_vs + kRaw * kRawScales : raw_k;
};
// A place in a ring of `of` blocks of `each` bytes that begins at `first`, moved on.
__device__ __forceinline__ unsigned next(unsigned at, unsigned first, unsigned each, int of) {
    at += each;
    return at == first + of * each ? first : at;
}

#define FENCE() __builtin_amdgcn_sched_barrier(0)
#define scalar __attribute__((address_space(4)))  // read through the scalar cache: the same for all lanes, written by earlier launches

__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }  // of all lanes
template <typename X>
__device__ __forceinline__ X uniform(const X* p) {
    struct Words {
        int w[sizeof(X) / 4];
    } x;
#pragma unroll
    for (unsigned i = 0; i < sizeof(X) / 4; ++i) x.w[i] = ((const scalar int*)(uintptr_t)p)[i];
    return __builtin_bit_cast(X, x);
}

// The blocks of a piece on their way to LDS.  Block i + 1 of K and block i of V go together (group i): a block's scores are computed
// before the block ahead of it is multiplied with V.  A wavefront loads its share of every block, 16 rows or 8, which lie in one page.
template <bool FP8, int NW>
struct Loader {
    typedef Lds<FP8, NW> L;
    static constexpr int kRowBytes = FP8 ? kD : kD * 2;
    static constexpr int kShare = kKeys / NW, kRows = FP8 ? 8 : 4, kEach = kShare / kRows;  // rows of a wavefront, of an instruction; instructions
    static constexpr int kHalf = kEach * (FP8 ? 2 : 1);  // instructions for K (e4m3: elements and exponents), and for V
    static constexpr unsigned kApart = FP8 ? 1024 : kFour;  // what the instructions' rows are apart in LDS
    const ExtendArgs& a;
    const scalar int32_t* table;
    int hk, lo, hi, jb0, blocks;  // keys lo .. hi may be read; blocks jb0 .. jb0 + blocks - 1
    int wave, lane;
    int issued;                   // last group issued
    unsigned k_to, v_to, ks_to, vs_to;  // where the next K and V go
    // the next group's K and V: the row of the pool where this wavefront's begin, and how many bytes behind that this lane's are
    size_t row_k, row_v;
    unsigned off_k[kHalf], off_v[kHalf];

    __device__ __forceinline__ unsigned k0() const { return (FP8 ? L::raw_k : L::k) + wave * kEach * kApart; }
    __device__ __forceinline__ unsigned v0() const { return (FP8 ? L::raw_v : L::v) + wave * kEach * kApart; }
    __device__ __forceinline__ void start() {
        issued = -2;
        k_to = k0(), v_to = v0();
        ks_to = L::raw_ks + wave * kEach * 256, vs_to = L::raw_vs + wave * kEach * 256;
        find(0);
    }
    // Keys out of lo .. hi (before the first row's window: their pages may have been given back; behind the last row: not written yet)
    // repeat the nearest key inside: always masked, and what lies in such rows must not meet a zero weight.
    __device__ __forceinline__ void find(int block) {
        const int key = (jb0 + block) * kKeys + wave * kShare, first = plan::clamp(key, lo & -kShare, hi & -kShare);
        row_k = pool_row(a.c, a.gm.Hkv, plan::clamp(table[first >> a.c.page_log2], 0, a.c.pages - 1), hk, first);
        int mine[kEach];  // rows behind the first
#pragma unroll
        for (int e = 0; e < kEach; ++e) mine[e] = e * kRows + load_row<FP8>(lane);
        if (key < lo || key + kShare - 1 > hi) {
#pragma unroll
            for (int e = 0; e < kEach; ++e) mine[e] = plan::clamp(key + mine[e], lo, hi) - first;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            off_k[e] = mine[e] * kRowBytes + load_chunk<FP8>(lane) * 16;
            if (FP8) off_k[kHalf - kEach + e] = mine[e] * kRowScales;
        }
    }
    // The next group, as far as there is one: its instructions one by one (K's, then V's), then what comes after it.
    __device__ __forceinline__ bool has_k() const { return issued + 2 < blocks; }
    __device__ __forceinline__ bool has_v() const { return issued + 1 >= 0 && issued + 1 < blocks; }
    __device__ __forceinline__ void issue_one(const char* pool, const unsigned char* scales, size_t row, const unsigned* off, unsigned to, unsigned scales_to, int e) const {
        if (!FP8 || e < kEach) dma16_so(pool + row * kRowBytes, off[e], to + e * kApart);
        else dma4_so(scales + row * kRowScales, off[e], scales_to + (e - kEach) * 256);
    }
    __device__ __forceinline__ void issue_k(int e) const {
        if (has_k()) issue_one(a.c.k, a.c.ks, row_k, off_k, k_to, ks_to, e);
    }
    __device__ __forceinline__ void issue_v(int e) const {
        if (has_v()) issue_one(a.c.v, a.c.vs, row_v, off_v, v_to, vs_to, e);
    }
    __device__ __forceinline__ void advance() {
        const int i = ++issued;
        if (i >= 0) {
            v_to = next(v_to, v0(), FP8 ? L::kRawBlock : kBlockBytes, FP8 ? L::kRaw : L::kV);
            if (FP8) vs_to = next(vs_to, L::raw_vs + wave * kEach * 256, L::kRawScales, L::kRaw);
        }
        k_to = next(k_to, k0(), FP8 ? L::kRawBlock : kBlockBytes, FP8 ? L::kRaw : L::kK);
        if (FP8) ks_to = next(ks_to, L::raw_ks + wave * kEach * 256, L::kRawScales, L::kRaw);
        row_v = row_k;
#pragma unroll
        for (int e = 0; e < kHalf; ++e) off_v[e] = off_k[e];
        find(min(i + 2, blocks - 1));
    }
    __device__ __forceinline__ void issue() {
#pragma unroll
        for (int e = 0; e < kHalf; ++e) issue_k(e);
#pragma unroll
        for (int e = 0; e < kHalf; ++e) issue_v(e);
        advance();
    }
    // Waits until at most the last group is on its way; those at the end have half their loads or none.
    __device__ __forceinline__ void wait() const {
        if (issued + 1 < blocks) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kHalf) : "memory");
        else if (issued < blocks) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kHalf) : "memory");
        else dma_wait();
    }
    // e4m3: this wavefront's pieces of a loaded block (the slot-th of the ring) become bf16.
    struct Raw {
        u32x4 x;
        uint32_t exponents;
    };
    __device__ __forceinline__ Raw raw_piece(unsigned raw, unsigned raw_scales, int slot, int e) const {
        return Raw{*(const __attribute__((address_space(3))) u32x4*)(uintptr_t)(raw + slot * L::kRawBlock + (wave * kEach + e) * 1024 + lane * 16),
                   *(const __attribute__((address_space(3))) uint32_t*)(uintptr_t)(raw_scales + slot * L::kRawScales + (wave * kEach + e) * 256 + lane * 4)};
    }
    __device__ __forceinline__ void store_piece(const Raw& r, unsigned block, int e) const {
        store_converted(r.x, r.exponents, (lds_ptr)(uintptr_t)block, wave * kShare + e * kRows + load_row<true>(lane), lane);
    }
    __device__ __forceinline__ void convert(unsigned raw, unsigned raw_scales, int slot, unsigned block) const {
#pragma unroll
        for (int e = 0; e < kEach; ++e) store_piece(raw_piece(raw, raw_scales, slot, e), block, e);
    }
};

// What a row has so far.  The maximum is one that some score had, not the largest: it moves when a score passes it by more than 2^kSlack
// (weights have the same 8 bits at any size), so that the two lanes of a row compare only then, and sums are rarely scaled.
constexpr float kSlack = 8.f;
constexpr float kNone = -3.0e38f;  // no key seen yet
struct RowSums {
    f32x16 o[4];
    float m = kNone, l = 0.f;
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
        m = kNone, l = 0.f;
    }
    __device__ __forceinline__ void scale(float by) {
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[d][e] *= by;
    }
    // mx: the largest score of this lane's keys, in log2 units.  Moves the maximum and the sum, returns what o is to be scaled by.
    __device__ __forceinline__ float move(float mx) {
        const float mnew = fmaxf(m, fmaxf(mx, __shfl_xor(mx, 32))), by = fast_exp2(m - mnew);
        m = mnew;
        l *= by;
        return by;
    }
    __device__ __forceinline__ void look(float mx) {
        if (__any(mx > m + kSlack)) scale(move(mx));
    }
    // An infinity or a NaN that came into a sum of values has stayed in it.  (Where the weights' sum, of both lanes of the row, is none either,
    // the row's own scores are to blame.)
    __device__ __forceinline__ bool finite() const {
        float z = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) z = fmaf(o[d][e], 0.f, z);
        return z == 0.f || l * 0.f != 0.f;
    }
};
__device__ __forceinline__ float largest(const f32x16& s) {
    float m[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) m[i] = fmaxf(fmaxf(s[3 * i], s[3 * i + 1]), s[3 * i + 2]);
    return fmaxf(fmaxf(fmaxf(m[0], m[1]), m[2]), fmaxf(fmaxf(m[3], m[4]), s[15]));
}

// Whether a lane of the workgroup says so; a barrier.  votes: NW words of LDS, not used again before another barrier.
template <int NW>
__device__ __forceinline__ bool vote(int* votes, bool yes) {
    if (__any(yes) && (threadIdx.x & 63) == 0) votes[threadIdx.x >> 6] = 1;
    else if ((threadIdx.x & 63) == 0) votes[threadIdx.x >> 6] = 0;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) any |= votes[i];
    return any != 0;
}
// Whether a row of a tile, given by its code, is routed.
__device__ __forceinline__ bool code_routed(const ExtendArgs& a, const Tile& t, int code) {
    return token_routed(a, t.s.start + code / a.gm.G, t.hk * a.gm.G + code % a.gm.G);
}
// Where the sums of row r of a piece go, and whether these are all it has: then its result does.
struct Out {
    int token, head;
    bool last, routed;  // last: O is written
    float* sums;
};
__device__ __forceinline__ Out out_of(const ExtendArgs& a, const Tile& t, const plan::Piece& piece, int w, int r, int code, bool routed) {
    const int tok = code / a.gm.G;
    Out o;
    o.token = t.s.start + tok, o.head = t.hk * a.gm.G + code - tok * a.gm.G;
    const bool whole = piece.first && piece.last;
    o.routed = routed;
    o.last = whole && t.kind == plan::kWindow && !(t.s.pos + tok > a.gm.W && o.routed);  // (routed: its window is all there is, a = s)
    o.sums = whole ? a.parts[t.kind] + ((size_t)o.token * a.gm.Hq + o.head) * kPart : a.slots + ((size_t)plan::slot(w, piece.first) * a.tile_rows + r) * kPart;
    return o;
}
// Four channels of a row's sums.
__device__ __forceinline__ void store_sums(const ExtendArgs& a, const Out& o, int c4, float m, float l, const f32x4& x) {
    if (o.last) {
        const float inv = 1.f / l, lse = (m + __builtin_amdgcn_logf(l)) * kLn2;
        const f32x4 y = x * inv, z = {0.f, 0.f, 0.f, 0.f};
        store_row(a, o.token, o.head, c4, y, o.routed ? y : z, lse, o.routed ? lse : -INFINITY);
    } else {
        if (c4 == 0) *reinterpret_cast<f32x2*>(o.sums) = f32x2{m, l};
        *reinterpret_cast<f32x4*>(o.sums + 4 + c4) = x;
    }
}
// A piece row by row and key by key: for those with keys that are not in every row's reach and with an infinity or a NaN in a sum.  It may
// come from such a key's values, as a weight of zero does not keep it out of the other rows' sums.
// (Looking for them among the values themselves, in the loops: 2.5 to 11 % of the main kernel's time.)
template <int NW>
__device__ __forceinline__ void rows_alone(const ExtendArgs& a, const Tile& t, const plan::Piece& piece, int w) {
    const Geom& gm = a.gm;
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, c4 = lane * 4;  // 32 lanes per row
    const int32_t* const table = a.c.table + (size_t)t.b * a.c.max_pages;
    const int b0 = (t.lo / kKeys + t.skip + piece.from) * kKeys, b1 = (t.lo / kKeys + t.skip + piece.to) * kKeys - 1;
    auto values = [&](const char* pool, const unsigned char* scales, size_t row) __attribute__((always_inline)) {
        if (!a.c.fp8) return __builtin_convertvector(*reinterpret_cast<const bf16x4*>(pool + row * (kD * 2) + c4 * 2), f32x4);
        const uint32_t x = *reinterpret_cast<const uint32_t*>(pool + row * kD + c4);
        const float e = exponent_value(scales[row * kRowScales + c4 / kScaleBlock]);
        const bf16x2 lo = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, e, false)), hi = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, e, true));
        return f32x4{(float)lo[0], (float)lo[1], (float)hi[0], (float)hi[1]};
    };
    for (int r = group; r < t.rows; r += 2 * NW) {
        const int code = row_code(a, t, t.first + r);
        const Out o = out_of(a, t, piece, w, r, code, code_routed(a, t, code));
        const Range keys = plan::row_keys(t.kind, t.s.pos + o.token - t.s.start, gm.W);
        const f32x4 q = __builtin_convertvector(*reinterpret_cast<const bf16x4*>(a.q + ((size_t)o.token * gm.Hq + o.head) * kD + c4), f32x4);
        float m = kNone, l = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int key = max(keys.lo, b0); key <= min(keys.hi, b1); ++key) {
            const size_t row = pool_row(a.c, gm.Hkv, plan::clamp(table[key >> a.c.page_log2], 0, a.c.pages - 1), t.hk, key);
            const f32x4 k = values(a.c.k, a.c.ks, row), v = values(a.c.v, a.c.vs, row);
            float s = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) s += __shfl_xor(s, d);
            s *= gm.scale_log2;
            const float mnew = fmaxf(m, s), by = fast_exp2(m - mnew), p = fast_exp2(s - mnew);
            l = fmaf(l, by, p), m = mnew;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = fmaf(x[e], by, p * v[e]);
        }
        store_sums(a, o, c4, m, l, x);
    }
}

// The functions that take a piece return false, in all lanes, where it is left to rows_alone.
//
// A tile of up to 32 rows, as decoding has them: bound by its loads.  Every wavefront takes 32 keys at a time, every eighth of the piece's,
// through shared memory of its own and with sums of its own, so that none waits for another before the end, where the eight sums are joined.
// (All wavefronts loading blocks of 64 keys for two of them to compute: 217 us for 64 sequences of 8K tokens in e4m3, 1.5 us a block.)
constexpr int kSub = 32;
template <int NW>
struct FewLds {
    static constexpr unsigned block = kSub / 4 * kFour, keys = NW * 2 * block, sums = NW * 32 * kPart * 4, votes = keys > sums ? keys : sums, used = votes + 64;
};
template <bool FP8, int NW>
__device__ __forceinline__ bool few_rows(const ExtendArgs& a, char* lds, const Tile& t, const plan::Piece& piece, int w) {
    const Geom& gm = a.gm;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, h = lane >> 5, G = gm.G, hk = t.hk;
    const float c2 = gm.scale_log2;
    const scalar int32_t* const table = (const scalar int32_t*)(a.c.table + (size_t)t.b * a.c.max_pages);
    // row r of the tile: its code, and from it the token
    auto code_of = [&](int r) __attribute__((always_inline)) { return row_code(a, t, t.first + min(r, t.rows - 1)); };
    const int jb0 = t.lo / kKeys + t.skip + piece.from, jb1 = t.lo / kKeys + t.skip + piece.to;
    const int sb1 = min(2 * jb1, t.hi / kSub + 1), sb0 = max(2 * jb0, t.lo / kSub) + wave;  // sub-blocks sb0, sb0 + 8, .. below sb1

    __syncthreads();  // LDS is free
    const unsigned k_to = wave * 2 * FewLds<NW>::block, v_to = k_to + FewLds<NW>::block;
    const lds_cptr k_at = (lds_cptr)(uintptr_t)(k_to + k_lane(lane)), v_at = (lds_cptr)(uintptr_t)(v_to + v_lane(lane));
    constexpr int kRows = FP8 ? 8 : 4, kEach = kSub / kRows;  // rows of an instruction, which lie in one page; instructions
    const int mine = load_row<FP8>(lane);
    u32x4 kx[FP8 ? kEach : 1], vx[FP8 ? kEach : 1];
    uint32_t kse[FP8 ? kEach : 1], vse[FP8 ? kEach : 1];
    size_t rows[kEach];   // where the instructions' rows begin in the pool, and how far behind that this lane's row is
    unsigned off[kEach];
    // keys out of the tile's repeat the nearest one in it (see Loader)
    auto find = [&](int sb) __attribute__((always_inline)) {
        const int k0 = sb * kSub;
        if (k0 >= t.lo && k0 + kSub - 1 <= t.hi) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const size_t row = pool_row(a.c, gm.Hkv, plan::clamp(table[(k0 + 16 * p) >> a.c.page_log2], 0, a.c.pages - 1), hk, k0 + 16 * p);
#pragma unroll
                for (int e = 0; e < kEach / 2; ++e) rows[p * (kEach / 2) + e] = row + e * kRows, off[p * (kEach / 2) + e] = mine;
            }
        } else {
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int first = plan::clamp(k0 + e * kRows, t.lo & -kRows, t.hi & -kRows);
                rows[e] = pool_row(a.c, gm.Hkv, plan::clamp(table[first >> a.c.page_log2], 0, a.c.pages - 1), hk, first);
                off[e] = plan::clamp(k0 + e * kRows + mine, t.lo, t.hi) - first;
            }
        }
    };
    auto load = [&](const char* pool, const unsigned char* scales, u32x4* x, uint32_t* se, unsigned to) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if constexpr (!FP8) {
                dma16_so(pool + rows[e] * (kD * 2), off[e] * (kD * 2) + load_chunk<FP8>(lane) * 16, to + e * kFour);
            } else {
                x[e] = *reinterpret_cast<const u32x4*>(pool + rows[e] * kD + off[e] * kD + load_chunk<FP8>(lane) * 16);
                se[e] = *reinterpret_cast<const uint32_t*>(scales + rows[e] * kRowScales + off[e] * kRowScales);
            }
        }
    };
    auto convert = [&](const u32x4* x, const uint32_t* se, unsigned block) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) store_converted(x[e], se[e], (lds_ptr)(uintptr_t)block, e * kRows + mine, lane);
    };
    if (sb0 < sb1) {
        find(sb0);
        load(a.c.k, a.c.ks, kx, kse, k_to);
        load(a.c.v, a.c.vs, vx, vse, v_to);
    }
    const int code = code_of(n), local_tok = code / G;
    const Range keys = plan::row_keys(t.kind, t.s.pos + local_tok, gm.W);
    bf16x8 qreg[8];
    const __bf16* qp = a.q + ((size_t)(t.s.start + local_tok) * gm.Hq + hk * G + code - local_tok * G) * kD + 8 * h;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) qreg[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) asm volatile("" : "+v"(qreg[ks]));  // waited for here, and so not in the loop, behind its loads
    const int lo_max = t.kind == plan::kWindow ? max(t.pos1 - gm.W, 0) : 0, hi_min = t.kind == plan::kWindow ? t.pos0 : t.pos0 - gm.W - 1;
    auto masked = [&](int sb) __attribute__((always_inline)) { return sb * kSub < lo_max || sb * kSub + kSub - 1 > hi_min; };
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const bf16x2 one2 = {(__bf16)1.0f, (__bf16)1.0f};
    RowSums row;
    row.clear();
    for (int sb = sb0; sb < sb1; sb += NW) {
        const bool more = sb + NW < sb1;
        if (more) find(sb + NW);
        if constexpr (FP8) convert(kx, kse, k_to);
        else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kEach) : "memory");  // K; V, loaded after it, may be on its way still
        bf16x8 op[8];
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) op[ks] = k_operand(k_at, ks, 0);
        if constexpr (FP8) {
            if (more) load(a.c.k, a.c.ks, kx, kse, k_to);
        }
        FENCE();
        f32x16 sc;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) sc = mfma32(op[ks], qreg[ks], ks == 0 ? zero16 : sc);
        if constexpr (!FP8) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the reads of K have returned
            if (more) load(a.c.k, a.c.ks, kx, kse, k_to);
            if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kEach) : "memory");
            else dma_wait();
        } else {
            convert(vx, vse, v_to);
            if (more) load(a.c.v, a.c.vs, vx, vse, v_to);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) op[i] = v_operand(v_at, i & 3, i >> 2);
        FENCE();
        const int k0 = sb * kSub;
        if (masked(sb)) {
            const int first = keys.lo - k0 - 4 * h, last = keys.hi - k0 - 4 * h;
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] = c_row(e, 0) >= first && c_row(e, 0) <= last ? sc[e] : -INFINITY;
        }
        row.look(largest(sc) * c2);
        u32x4 p[2];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            f32x2 f = {fast_exp2(fmaf(sc[e], c2, -row.m)), fast_exp2(fmaf(sc[e + 1], c2, -row.m))};
            const bf16x2 pb = __builtin_convertvector(f, bf16x2);
            row.l = __builtin_amdgcn_fdot2_f32_bf16(pb, one2, row.l, false);
            p[e >> 3][(e & 7) >> 1] = __builtin_bit_cast(uint32_t, pb);
        }
        if constexpr (!FP8) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the reads of V have returned
            if (more) load(a.c.v, a.c.vs, vx, vse, v_to);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) row.o[i & 3] = mfma32(op[i], __builtin_bit_cast(bf16x8, p[i >> 2]), row.o[i & 3]);
    }

    // ---- the eight wavefronts' sums, joined: 16 threads per row, eight channels each
    row.l += __shfl_xor(row.l, 32);
    float* const sums = reinterpret_cast<float*>(lds);  // [wave][row][kPart]
    const bool some_masked = masked(sb0 - wave) || masked(sb1 - 1);
    if (vote<NW>(reinterpret_cast<int*>(lds + FewLds<NW>::votes), some_masked && !row.finite())) return false;
    // (every wavefront is done with its part of LDS)
    {
        float* const at = sums + (wave * 32 + n) * kPart;
        if (h == 0) *reinterpret_cast<f32x2*>(at) = f32x2{row.m, row.l};
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4*>(at + 4 + d * 32 + c_row(e, h)) = f32x4{row.o[d][e], row.o[d][e + 1], row.o[d][e + 2], row.o[d][e + 3]};
    }
    __syncthreads();
    const int c8 = (threadIdx.x & 15) * 8;
    for (int r = threadIdx.x >> 4; r < t.rows; r += NW * 4) {
        float m = kNone, l = 0.f;
        f32x2 ml[NW];
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            ml[v] = *reinterpret_cast<const f32x2*>(sums + (v * 32 + r) * kPart);
            m = fmaxf(m, ml[v][0]);
        }
        f32x4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const float by = fast_exp2(ml[v][0] - m);
            const f32x4* const at = reinterpret_cast<const f32x4*>(sums + (v * 32 + r) * kPart + 4 + c8);
            l = fmaf(ml[v][1], by, l);
            x += at[0] * by, y += at[1] * by;
        }
        const int out_code = code_of(r);
        const Out o = out_of(a, t, piece, w, r, out_code, code_routed(a, t, out_code));
        store_sums(a, o, c8, m, l, x);
        store_sums(a, o, c8 + 4, m, l, y);
    }
    return true;
}

// Workgroups are dealt round-robin to the 8 XCDs: each XCD takes neighbouring segments and stretches.
__device__ __forceinline__ int workgroup(const ExtendArgs& a) { return (int)(blockIdx.x & 7) * (a.workgroups >> 3) + (int)(blockIdx.x >> 3); }
// A workgroup's pieces, in order: f(tile, piece, workgroup).
template <typename F>
__device__ __forceinline__ void for_pieces(const ExtendArgs& a, F&& f) {
    const int w = workgroup(a);
    const Head line = uniform(a.head);
    const bool segment = w < line.segments;  // all it does; the others share the line
    const int stretch = w - line.segments;
    if (!segment && (long long)stretch * line.per >= line.total) return;
    const Segment mine = segment ? uniform(a.segment + w) : Segment{uniform(a.first_tile + stretch), 0, 0};
    const long long x1 = (long long)(stretch + 1) * line.per;
    for (int T = mine.tile; T < line.tiles; ++T) {
        const Tile t = uniform(a.tiles + T);
        plan::Piece piece{mine.from - t.skip, mine.to - t.skip, 0, 0};
        if (!segment) {
            if (t.start >= x1) break;
            piece = plan::piece(place_of(a, t), line.per, stretch);
            if (piece.from == piece.to) continue;
        } else if (T != mine.tile) {
            break;
        }
        f(t, piece, w);
    }
}
// Shared memory is written and read by address: all of it there is begins at 0.
__device__ __forceinline__ void by_address(char* lds) { asm volatile("" ::"s"(__builtin_amdgcn_readfirstlane(lds_offset(lds))) : "memory"); }

// A tile by 8 wavefronts of 32 rows, two on a SIMD.  (4 wavefronts of 64 rows, each with a SIMD and its 512 registers to itself and every operand
// serving two matrix instructions, took as long at 4096 tokens behind 126976: 1732 us and 1730 on one card, at clocks of
// 2.1 GHz and 1.9: the one that needs fewer cycles gets fewer of them.)
// HALVES, up to 128 rows: wavefronts 4 .. 7 take the second half of the keys of every block for the rows of wavefronts 0 .. 3.
constexpr int kWaves = 8, kHalvesRows = 32 * kWaves / 2;
static_assert(kHalvesRows == plan::kManyRows && kSub == plan::kFewRows, "costs and kernels agree on what are few rows, and many");
template <bool FP8>
struct TileLds {
    static constexpr unsigned many = Lds<FP8, kWaves>::used + 64, used = many > FewLds<kWaves>::used ? many : FewLds<kWaves>::used;  // (64: votes)
    // behind these, half a block of V that is zero, for extend_kernel: what the first of a tile's products has beside weights of zero
    static constexpr unsigned zeros = used, kZeros = kKeys / 8 * kFour;
};
template <bool FP8, bool HALVES>
__device__ __forceinline__ bool some_rows(const ExtendArgs& a, char* lds, const Tile& t, const plan::Piece& piece, int w) {
    typedef Lds<FP8, kWaves> L;
    const Geom& gm = a.gm;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, h = lane >> 5, G = gm.G;
    const float c2 = gm.scale_log2;
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const bf16x2 one2 = {(__bf16)1.0f, (__bf16)1.0f};

    const int hk = t.hk, jb0 = t.lo / kKeys + t.skip + piece.from, blocks = piece.to - piece.from;
    const Seq s = t.s;
    __syncthreads();  // LDS is free
    Loader<FP8, kWaves> load{a, (const scalar int32_t*)(a.c.table + (size_t)t.b * a.c.max_pages), hk, t.lo, t.hi, jb0, blocks, wave, lane};
    load.start();
    load.issue();
    load.issue();

    // ---- this lane's row (rows past the end repeat the last one: computed, never written)
    const int r = (HALVES ? wave & (kWaves / 2 - 1) : wave) * 32 + n;
    const bool valid = r < t.rows, wave_on = r - n < t.rows;
    const int code = row_code(a, t, t.first + min(r, t.rows - 1)), tok = code / G, token = s.start + tok, head = hk * G + code - tok * G, pos = s.pos + tok;
    const Range keys = plan::row_keys(t.kind, pos, gm.W);
    bf16x8 qreg[8];
    const __bf16* qp = a.q + ((size_t)token * gm.Hq + head) * kD + 8 * h;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) qreg[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
    int routed = token_routed(a, token, head);
    asm volatile("" : "+v"(routed));
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) asm volatile("" : "+v"(qreg[ks]));  // waited for here, and so not in the loop, behind its loads
    // blocks that every row of the tile sees whole: from `whole0` to `whole1` - 1
    const int lo_max = t.kind == plan::kWindow ? max(t.pos1 - gm.W, 0) : 0, hi_min = t.kind == plan::kWindow ? t.pos0 : t.pos0 - gm.W - 1;
    const int whole0 = (lo_max + kKeys - 1) / kKeys, whole1 = (hi_min + 1) / kKeys;
    auto masked = [&](int jb) __attribute__((always_inline)) { return jb < whole0 || jb >= whole1; };
    // scores of 32 keys from k0 on, those out of the row's reach taken out
    auto mask = [&](f32x16& sc, int k0) __attribute__((always_inline)) {
        const int first = keys.lo - k0 - 4 * h, last = keys.hi - k0 - 4 * h;
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[e] = c_row(e, 0) >= first && c_row(e, 0) <= last ? sc[e] : -INFINITY;
    };

    RowSums row;
    row.clear();
    unsigned kb = L::k, vb = L::v;  // block j
    auto next_k = [&]() __attribute__((always_inline)) { return next(kb, L::k, kBlockBytes, L::kK); };
    auto next_v = [&]() __attribute__((always_inline)) { return next(vb, L::v, kBlockBytes, L::kV); };
    if constexpr (FP8) {
        load.wait();
        load.convert(L::raw_k, L::raw_ks, 0, L::k);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load.issue();
        load.wait();
        if (blocks > 1) load.convert(L::raw_k, L::raw_ks, 1, L::k + kBlockBytes);
        load.convert(L::raw_v, L::raw_vs, 0, L::v);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load.issue();
    } else {
        load.issue();
        load.wait();
    }
    __syncthreads();
    // begins a block's work: more on its way, and e4m3 of the next group made bf16
    auto begin = [&](int j) __attribute__((always_inline)) {
        if constexpr (FP8) {
            if (j + 1 < blocks) {
                load.wait();
                if (j + 2 < blocks) load.convert(L::raw_k, L::raw_ks, j & 1, next(next_k(), L::k, kBlockBytes, L::kK));
                load.convert(L::raw_v, L::raw_vs, (j + 1) & 1, next_v());
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
        }
        load.issue();
    };
    auto end = [&](int j) __attribute__((always_inline)) {
        if constexpr (!FP8) load.wait();
        __syncthreads();
        kb = next_k(), vb = next_v();
    };
    const unsigned k_mine = k_lane(lane), v_mine = v_lane(lane);
    auto k_block = [&](unsigned at) __attribute__((always_inline)) { return (lds_cptr)(uintptr_t)(at + k_mine); };
    auto v_block = [&](unsigned at) __attribute__((always_inline)) { return (lds_cptr)(uintptr_t)(at + v_mine); };
    // Weights of a pair of scores, rounded to bf16; the sum is that of the weights as the matrix cores see them, so that what
    // they are divided by is exact for them.
    auto weight = [&](const f32x16& sc, int e) __attribute__((always_inline)) { return fast_exp2(fmaf(sc[e], c2, -row.m)); };
    auto pair = [&](float x, float y) __attribute__((always_inline)) {
        f32x2 f = {x, y};
        const bf16x2 pb = __builtin_convertvector(f, bf16x2);
        row.l = __builtin_amdgcn_fdot2_f32_bf16(pb, one2, row.l, false);
        return __builtin_bit_cast(uint32_t, pb);
    };
    if constexpr (HALVES) {
        // One half of 32 keys per wavefront and block, all operands read ahead; short of rows, the loads set the pace.
        const int half = wave / (kWaves / 2);
        for (int j = 0; j < blocks; ++j) {
            begin(j);
            if (wave_on) {
                const lds_cptr ka = k_block(kb) + half * 8 * kFour, va = v_block(vb) + half * 8 * kFour;
                bf16x8 kop[8], vop[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) kop[i] = k_operand(ka, i, 0);
#pragma unroll
                for (int i = 0; i < 8; ++i) vop[i] = v_operand(va, i & 3, i >> 2);
                FENCE();
                f32x16 sc;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) sc = mfma32(kop[ks], qreg[ks], ks == 0 ? zero16 : sc);
                if (masked(jb0 + j)) mask(sc, (jb0 + j) * kKeys + half * 32);
                row.look(largest(sc) * c2);
                u32x4 p[2];
#pragma unroll
                for (int e = 0; e < 16; e += 2) p[e >> 3][(e & 7) >> 1] = pair(weight(sc, e), weight(sc, e + 1));
#pragma unroll
                for (int i = 0; i < 8; ++i) row.o[i & 3] = mfma32(vop[i], __builtin_bit_cast(bf16x8, p[i >> 2]), row.o[i & 3]);
            }
            end(j);
        }
    } else {
        // All keys for 32 rows a wavefront, in steps of 32.  While the vector units find the weights of a step's keys, the matrix
        // cores compute the scores of the next step's and the product of the step before with V, neither of which waits for these
        // weights: 16 matrix instructions, a slot each; operands are read kAhead slots before their use.  (With the product of the
        // same step in the second half of the slots the weights had to be found in the first ones: 1755 us at 4096 tokens behind 126976.)
        constexpr int kAhead = 2;
        f32x16 sa, sb;
        u32x4 pa[2], pb[2];
        float mx;
        auto step = [&](auto half_tag, const f32x16& cur, f32x16& nxt, const u32x4 (&before)[2], u32x4 (&p)[2], lds_cptr ka, lds_cptr va, int k0_next, bool masked_next) __attribute__((always_inline)) {
            constexpr int H = decltype(half_tag)::value;  // nxt: the block's second half, or the next block's first
            float by = 1.f;
            const bool grew = __any(mx > row.m + kSlack);
            if (grew) by = row.move(mx);
            bf16x8 op[16 + kAhead];
            auto read = [&](auto oc) __attribute__((always_inline)) {
                constexpr int o = decltype(oc)::value;
                if constexpr (o < 8) op[o] = k_operand(ka, o, 1 - H);
                else if constexpr (o < 16) op[o] = v_operand(va, o & 3, 2 * (1 - H) + ((o - 8) >> 2));
            };
            static_for<0, kAhead>([&](auto oc) { read(oc); });
            FENCE();
            static_for<0, 16>([&](auto sc_) __attribute__((always_inline)) {
                constexpr int slot = decltype(sc_)::value;
                if constexpr (slot < 8) nxt = mfma32(op[slot], qreg[slot], slot == 0 ? zero16 : nxt);
                else row.o[slot & 3] = mfma32(op[slot], __builtin_bit_cast(bf16x8, before[(slot - 8) >> 2]), row.o[slot & 3]);
                read(std::integral_constant<int, slot + kAhead>{});
                if constexpr (slot % 2 == 0) p[slot >> 3][(slot >> 1) & 3] = pair(weight(cur, slot), weight(cur, slot + 1));
                if constexpr (slot == 13) {
                    if (masked_next) mask(nxt, k0_next);
                    mx = largest(nxt) * c2;
                }
                FENCE();
            });
            if (grew) row.scale(by);
        };
        typedef std::integral_constant<int, 0> H0;
        typedef std::integral_constant<int, 1> H1;
        {
            const lds_cptr ka = k_block(kb);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) sa = mfma32(k_operand(ka, ks, 0), qreg[ks], ks == 0 ? zero16 : sa);
        }
        if (masked(jb0)) mask(sa, jb0 * kKeys);
        mx = largest(sa) * c2;
        // before the first step: weights of zero, and values of zero beside them (an infinity among the piece's own would be a NaN in all rows)
        lds_cptr va = v_block(TileLds<FP8>::zeros - kKeys / 8 * kFour);  // its second half is what that step reads
        pb[0] = pb[1] = u32x4{0u, 0u, 0u, 0u};
        for (int j = 0; j < blocks; ++j) {
            const int jb = jb0 + j;
            begin(j);
            step(H0{}, sa, sb, pb, pa, k_block(kb), va, jb * kKeys + 32, masked(jb));
            va = v_block(vb);
            step(H1{}, sb, sa, pa, pb, k_block(next_k()), va, (jb + 1) * kKeys, masked(jb + 1));
            end(j);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) row.o[i & 3] = mfma32(v_operand(va, i & 3, 2 + (i >> 2)), __builtin_bit_cast(bf16x8, pb[i >> 2]), row.o[i & 3]);
    }

    row.l += __shfl_xor(row.l, 32);
    if ((masked(jb0) || masked(jb0 + blocks - 1)) && vote<kWaves>(reinterpret_cast<int*>(lds + L::used), !row.finite())) return false;

    // ---- out
    if constexpr (HALVES) {  // the second half's sums join the first's, through LDS (16-byte pieces of a lane side by side)
        f32x4* const there = reinterpret_cast<f32x4*>(lds) + (wave & (kWaves / 2 - 1)) * (17 * 64) + lane;
        if (wave_on && wave >= kWaves / 2) {
            there[0] = f32x4{row.m, row.l, 0.f, 0.f};
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 4) there[(1 + d * 4 + e / 4) * 64] = f32x4{row.o[d][e], row.o[d][e + 1], row.o[d][e + 2], row.o[d][e + 3]};
        }
        __syncthreads();
        if (wave_on && wave < kWaves / 2) {
            const f32x4 ml = there[0];
            const float mnew = fmaxf(row.m, ml[0]), by = fast_exp2(ml[0] - mnew), own = fast_exp2(row.m - mnew);
            row.scale(own);
            row.m = mnew;
            row.l = fmaf(ml[1], by, row.l * own);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 x = there[(1 + d * 4 + e / 4) * 64];
#pragma unroll
                    for (int i = 0; i < 4; ++i) row.o[d][e + i] = fmaf(x[i], by, row.o[d][e + i]);
                }
        }
    }
    if (!valid || (HALVES && wave >= kWaves / 2)) return true;
    const Out o = out_of(a, t, piece, w, r, code, routed);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) store_sums(a, o, d * 32 + c_row(e, h), row.m, row.l, f32x4{row.o[d][e], row.o[d][e + 1], row.o[d][e + 2], row.o[d][e + 3]});
    return true;
}

template <bool FP8>
__global__ __launch_bounds__(64 * kWaves, 2) void extend_kernel(ExtendArgs a) {
    typedef TileLds<FP8> L;
    __shared__ __attribute__((aligned(1024))) char lds[L::zeros + L::kZeros];
    by_address(lds);
    for (unsigned at = L::zeros + threadIdx.x * 16; at < L::zeros + L::kZeros; at += 64 * kWaves * 16)  // (every tile begins with a barrier)
        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)at = u32x4{0u, 0u, 0u, 0u};
    for_pieces(a, [&](const Tile& t, const plan::Piece& piece, int w) __attribute__((always_inline)) {
        bool done;
        if (t.rows <= kSub) done = few_rows<FP8, kWaves>(a, lds, t, piece, w);
        else if (t.rows <= kHalvesRows) done = some_rows<FP8, true>(a, lds, t, piece, w);
        else done = some_rows<FP8, false>(a, lds, t, piece, w);
        if (!__any(done)) rows_alone<kWaves>(a, t, piece, w);
    });
}

// Calls whose sequences all have up to 128 rows per KV head, a tile for each part of its keys; FEW: up to 32.  SELF: every workgroup makes the plan
// for itself, a thread per KV head of a sequence (at most as many as threads), and the first one leaves it for the last kernel: a
// launch less.
constexpr int kShortPairs = 64 * kWaves;
struct ShortPlan {
    int start[2 * kShortPairs], of[2 * kShortPairs];  // of a tile: its place in the line; twice its pair, plus its kind
    Seq seq[kShortPairs];
    int sums[kWaves], first;
};
template <bool FP8, bool FEW, bool SELF>
__global__ __launch_bounds__(64 * kWaves, 2) void extend_short_kernel(ExtendArgs a) {
    constexpr unsigned kLds = FEW ? FewLds<kWaves>::used : TileLds<FP8>::used;
    __shared__ __attribute__((aligned(1024))) char lds[kLds + (SELF ? sizeof(ShortPlan) : 0)];
    by_address(lds);
    auto rows = [&](const Tile& t, const plan::Piece& piece, int w) __attribute__((always_inline)) {
        bool done;
        if (FEW || t.rows <= kSub) done = few_rows<FP8, kWaves>(a, lds, t, piece, w);
        else done = some_rows<FP8, true>(a, lds, t, piece, w);
        if (!__any(done)) rows_alone<kWaves>(a, t, piece, w);
    };
    if constexpr (!SELF) {
        for_pieces(a, rows);
    } else {
        ShortPlan& plan_ = *reinterpret_cast<ShortPlan*>(lds + kLds);
        const Geom& gm = a.gm;
        const int w = workgroup(a), mine = threadIdx.x, pairs = gm.B * gm.Hkv;
        Tile t[2];
        bool on[2] = {false, false};
        Seq s{};
        const int b = mine / gm.Hkv, hk = mine - b * gm.Hkv;
        if (mine < pairs) {
            s = seq_of(a, b);
            on[plan::kWindow] = a.do_local && s.n;
            on[plan::kPrefix] = has_prefix(a, s, hk);
            plan_.seq[mine] = s;
        }
        int length[2] = {0, 0};
#pragma unroll
        for (int kind = 0; kind < 2; ++kind)
            if (on[kind]) {
                t[kind] = make_tile(a, s, b, hk, kind, 0, s.n * gm.G);
                length[kind] = place_of(a, t[kind]).length();
            }
        int T, tiles, at, total;
        scan<64 * kWaves>(on[0] + on[1], plan_.sums, T, tiles);
        scan<64 * kWaves>(length[0] + length[1], plan_.sums, at, total);
        total = same(total), tiles = same(tiles);
        const int per = same(plan::stretch(total, a.workgroups, plan::block_cost(FEW ? kSub : kHalvesRows, FP8))), x0 = w * per;
#pragma unroll
        for (int kind = 0; kind < 2; ++kind)
            if (on[kind]) {
                plan_.start[T] = at, plan_.of[T] = 2 * mine + kind;
                if (at <= x0 && x0 < at + length[kind]) plan_.first = T;
                if (w == 0) {
                    t[kind].start = at;
                    a.shorts[mine].place[kind] = place_of(a, t[kind]);
                }
                ++T, at += length[kind];
            }
        if (w == 0 && mine < pairs) {
            a.shorts[mine].s = s;
            if (hk == 0)
                for (int i = 0; i < s.n; ++i) a.token_seq[s.start + i] = b;
            if (mine == 0) *a.head = Head{total, per, tiles, 0, 0};
        }
        __syncthreads();
        if (x0 >= total) return;
        for (int i = same(plan_.first); i < tiles; ++i) {
            const int start = same(plan_.start[i]), of = same(plan_.of[i]);
            if (start >= x0 + per) break;
            const int p = of >> 1, tb = same(p / gm.Hkv);
            const Seq ts{same(plan_.seq[p].start), same(plan_.seq[p].n), same(plan_.seq[p].pos)};
            Tile tile = make_tile(a, ts, tb, p - tb * gm.Hkv, of & 1, 0, ts.n * gm.G);
            tile.start = start, tile.pos0 = same(tile.pos0), tile.pos1 = same(tile.pos1), tile.lo = same(tile.lo), tile.hi = same(tile.hi), tile.blocks = same(tile.blocks);
            const plan::Piece piece = plan::piece(place_of(a, tile), per, w);
            if (piece.from != piece.to) rows(tile, piece, w);
        }
    }
}

// Thirty-two lanes per row, four channels each.
struct Sums {
    float m = kNone, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void join(float m2, float l2, const f32x4& o2) {
        const float mn = fmaxf(m, m2), s0 = fast_exp2(m - mn), s1 = fast_exp2(m2 - mn);
        l = fmaf(l, s0, l2 * s1);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(o[e], s0, o2[e] * s1);
        m = mn;
    }
    __device__ __forceinline__ f32x4 value() const { return o / l; }
    __device__ __forceinline__ float lse() const { return (m + __builtin_amdgcn_logf(l)) * kLn2; }
};
// Where the i-th of the sums that row r of a tile has in pieces are; row_part: if it is the line's and the tile is whole there.
__device__ __forceinline__ const float* sums_at(const ExtendArgs& a, const Pieces& p, int i, int r, const float* row_part) {
    const float* const part = a.slots + ((size_t)p.slot_of(i) * a.tile_rows + r) * kPart;
    return p.in_parts(i) ? row_part : part;
}
// Every `step`-th of n sums from the `from`-th on, at(i), joined: f(i, maximum, sum, four channels).  AHEAD loads are on their way together
// (past the end the first is read again, for nobody).
template <int AHEAD, typename At, typename F>
__device__ __forceinline__ void each_part(int n, int from, int step, int c4, At&& at, F&& f) {
    for (int i0 = from; i0 < n; i0 += AHEAD * step) {
        f32x2 ml[AHEAD];
        f32x4 x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const float* const part = at(i0 + j * step < n ? i0 + j * step : i0);
            ml[j] = *reinterpret_cast<const f32x2*>(part);
            x[j] = *reinterpret_cast<const f32x4*>(part + 4 + c4);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (i0 + j * step < n) f(i0 + j * step, ml[j][0], ml[j][1], x[j]);
    }
}
__device__ __forceinline__ const float* row_part(const ExtendArgs& a, int kind, int token, int head) {
    return a.parts[kind] + ((size_t)token * a.gm.Hq + head) * kPart;
}
// Rows of tiles of many, 16 of a tile per workgroup: a thread per row finds out whether something is left to do (rows of whole tiles that have no
// keys before their window were written by the kernel before) and where its sums lie, then 32 lanes take a row each of those.
// (32 rows a workgroup, and so four for each group of lanes one behind the other: 18.6 us for 14.0 at 300 tokens behind 3000, 19.7 for 16.7 at 1000
// beside 31 single ones, 15.5 for 12.5 at 500 beside 39; but 10.6 for 12.5 at 3 x 777, where most rows have nothing left to do.)
constexpr int kCombineRows = 16;
__global__ __launch_bounds__(kThreads) void extend_combine_kernel(ExtendArgs a) {
    struct Row {
        int token, head, r, routed, prefix_row;  // r: in the tile; prefix_row: in its tile of keys before the window, -1: it has none
        Pieces prefix;
    };
    __shared__ Row rows[kCombineRows];
    __shared__ int count;
    const Geom& gm = a.gm;
    const Head head_ = uniform(a.head);
    const Tile t = uniform(a.tiles + blockIdx.x);  // (beside the head: there is room for as many tiles as workgroups)
    if ((int)blockIdx.x >= head_.tiles) return;
    const int c4 = (threadIdx.x & 31) * 4, G = gm.G, r0 = blockIdx.y * kCombineRows;
    if (r0 >= t.rows || (a.do_local && t.kind != plan::kWindow)) return;
    const Pieces own = plan::pieces_of(place_of(a, t), head_.per, head_.segments);
    if (threadIdx.x < kCombineRows) {
        const Pair pair = uniform(a.pairs + t.b * gm.Hkv + t.hk);
        const int first_prefix = pair.first_tile + window_tiles(a, t.s), many = plan::many_tiles(pair.listed, a.tile_rows), r = r0 + (int)threadIdx.x;
        Row row{};
        bool todo = false;
        if (r < t.rows) {
            const int code = row_code(a, t, t.first + r), tok = code / G;
            row.r = r, row.head = t.hk * G + code - tok * G, row.token = t.s.start + tok, row.prefix_row = -1;
            row.routed = token_routed(a, row.token, row.head);
            const bool prefix = row.routed && t.s.pos + tok > gm.W;
            todo = !(a.do_local && own.whole() && !prefix);
            if (prefix) {
                const int i = plan::clamp(list_of(a, a.rank, t.s, t.hk)[code], 0, max(pair.listed - 1, 0)), j = i / a.tile_rows;
                row.prefix_row = i - j * a.tile_rows;
                row.prefix = plan::pieces_of(place_of(a, a.tiles[min(first_prefix + j, head_.tiles - 1)]), head_.per, head_.segments);
                row.prefix.segments = j < many ? pair.segments : 0, row.prefix.first_segment = plan::segment_workgroup(pair.first_segment, many, 0, j), row.prefix.of = many;
            }
        }
        const unsigned long long set = __ballot(todo);
        if (todo) rows[__popcll(set & ((1ull << threadIdx.x) - 1ull))] = row;
        if (threadIdx.x == 0) count = __popcll(set);
    }
    __syncthreads();
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
    for (int i = threadIdx.x >> 5; i < count; i += kThreads / 32) {
        const Row row = rows[i];
        Sums sums, prefix;
        f32x4 x = z;
        float lse_l = -INFINITY;
        const int mine = a.do_local ? own.count() : 0, n = mine + (row.prefix_row >= 0 ? row.prefix.count() : 0);
        each_part<4>(n, 0, 1, c4,
                     [&](int i) {
                         return i < mine ? sums_at(a, own, i, row.r, row_part(a, plan::kWindow, row.token, row.head))
                                         : sums_at(a, row.prefix, i - mine, row.prefix_row, row_part(a, plan::kPrefix, row.token, row.head));
                     },
                     [&](int i, float m, float l, const f32x4& o) {
                         if (i < mine) sums.join(m, l, o);
                         else prefix.join(m, l, o);
                     });
        if (a.do_local) x = sums.value(), lse_l = sums.lse();
        sums.join(prefix.m, prefix.l, prefix.o);
        store_row(a, row.token, row.head, c4, x, row.routed ? sums.value() : z, lse_l, row.routed ? sums.lse() : -INFINITY);
    }
}
// Rows of short calls: a workgroup per row (from row0 on), whose pieces, many where the cache is long, are shared by kSlices groups of lanes.
constexpr int kSlices = 8;
constexpr int kShortRows = 1 << 23;  // of a launch, whose threads have to be fewer than 2^32
__global__ __launch_bounds__(32 * kSlices) void extend_combine_short_kernel(ExtendArgs a, int row0) {
    __shared__ __attribute__((aligned(16))) float part[2][kSlices][kPart];
    const Geom& gm = a.gm;
    const int c4 = (threadIdx.x & 31) * 4, slice = threadIdx.x >> 5, G = gm.G;
    const int row = row0 + (int)blockIdx.x, token = row / gm.Hq, head = row - token * gm.Hq, hk = head / G;
    const int b = *(const scalar int*)(uintptr_t)(a.token_seq + token);  // of a token that is in no sequence: whatever was there
    const Head head_ = uniform(a.head);
    const bool routed = token_routed(a, token, head);
    if (b < 0 || b >= gm.B) return;
    const Short call = uniform(a.shorts + b * gm.Hkv + hk);
    const int at = token - call.s.start;
    if (at < 0 || at >= call.s.n) return;
    const bool prefix = routed && call.s.pos + at > gm.W;
    const int r = at * G + head - hk * G;
    Sums sums[2];  // of the window's keys, of those before it
    for (int kind = 0; kind < 2; ++kind) {
        if (!(kind == plan::kWindow ? a.do_local : prefix)) continue;
        const Pieces p = plan::pieces_of(call.place[kind], head_.per, head_.segments);
        if (kind == plan::kWindow && p.whole() && !prefix) return;  // written already
        each_part<8>(p.count(), slice, kSlices, c4, [&](int i) { return sums_at(a, p, i, r, row_part(a, kind, token, head)); },
                     [&](int, float m, float l, const f32x4& o) { sums[kind].join(m, l, o); });
    }
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        float* const out = part[kind][slice];
        if (c4 == 0) out[0] = sums[kind].m, out[1] = sums[kind].l;
        *reinterpret_cast<f32x4*>(out + 4 + c4) = sums[kind].o;
    }
    __syncthreads();
    if (slice) return;
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
    f32x4 x = z;
    float lse_l = -INFINITY;
    Sums all;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
#pragma unroll
        for (int i = 0; i < kSlices; ++i) {
            const float* const in = part[kind][i];
            all.join(in[0], in[1], *reinterpret_cast<const f32x4*>(in + 4 + c4));
        }
        if (kind == plan::kWindow && a.do_local) x = all.value(), lse_l = all.lse();
    }
    store_row(a, token, head, c4, x, routed ? all.value() : z, lse_l, routed ? all.lse() : -INFINITY);
}

constexpr int kWorkgroups = 256;  // one per CU

// The workspace: sub-buffers at multiples of 256 bytes.
size_t lay_out(ExtendArgs& a, char* base) {
    const Geom& g = a.gm;
    size_t at = 0;
    auto take = [&](auto*& p, size_t count) {
        p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(base + at);
        at += (count * sizeof(*p) + 255) / 256 * 256;
    };
    const size_t rows = (size_t)g.T * g.G, pairs = (size_t)g.B * g.Hkv;
    a.workgroups = kWorkgroups;
    const long long most = (long long)a.max_new * g.G;  // rows of a KV head of a sequence
    a.few = most <= kHalvesRows;
    a.tile_rows = most <= kSub ? kSub : a.few ? kHalvesRows : 32 * kWaves;
    a.most_tiles = (int)(2 * g.Hkv * (rows / a.tile_rows + g.B));
    take(a.head, 1);
    take(a.tiles, a.most_tiles);
    take(a.first_tile, a.workgroups);
    take(a.segment, a.workgroups);
    take(a.pairs, pairs);
    take(a.shorts, a.few ? pairs : 0);
    take(a.list, a.few ? 0 : rows * g.Hkv);
    take(a.rank, a.few ? 0 : rows * g.Hkv);
    take(a.token_seq, a.few ? g.T : 0);
    take(a.slots, (size_t)2 * a.workgroups * a.tile_rows * kPart);
    take(a.parts[0], rows * g.Hkv * kPart);
    take(a.parts[1], rows * g.Hkv * kPart);
    return at;
}

}  // namespace

size_t extend_workspace(const Geom& g, int max_new) {
    ExtendArgs a{};
    a.gm = g;
    a.max_new = max_new;
    return lay_out(a, nullptr);
}

int mfma_extend(const Geom& g, const Pages& c, const void* q, const int32_t* seq_start, const int32_t* pos, const uint8_t* mask,
                int mask_heads, int max_new, int do_local, int do_global, void* O, float* lse_l, float* lse_g, void* S, void* A,
                void* workspace, hipStream_t st) {
    ExtendArgs a{};
    a.gm = g;
    if (!do_local) a.gm.W = -1;
    a.c = c;
    a.q = (const __bf16*)q;
    a.seq_start = seq_start, a.pos = pos;
    a.mask = mask, a.mask_heads = mask_heads;
    a.do_local = do_local, a.do_global = do_global, a.max_new = max_new;
    a.O = (__bf16*)O, a.S = (__bf16*)S, a.A = (__bf16*)A;
    a.lse_l = lse_l, a.lse_g = lse_g;
    lay_out(a, (char*)workspace);
    if (!a.few) {
        KernelTimer kt("extend_list", st);
        hipLaunchKernelGGL(extend_list_kernel, dim3(g.B * g.Hkv), dim3(kListThreads), 0, st, a);
    }
    const bool self = a.few && g.B * g.Hkv <= kShortPairs;
    if (!self) {
        KernelTimer kt("extend_plan", st);
        hipLaunchKernelGGL(extend_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
    }
    {
        KernelTimer kt("extend", st);
        auto launch = [&](auto fp8) {
            constexpr bool FP8 = decltype(fp8)::value;
            const dim3 grid(a.workgroups), threads(64 * kWaves);
            if (!a.few) hipLaunchKernelGGL(extend_kernel<FP8>, grid, threads, 0, st, a);
            else if (a.tile_rows == kSub && self) hipLaunchKernelGGL((extend_short_kernel<FP8, true, true>), grid, threads, 0, st, a);
            else if (a.tile_rows == kSub) hipLaunchKernelGGL((extend_short_kernel<FP8, true, false>), grid, threads, 0, st, a);
            else if (self) hipLaunchKernelGGL((extend_short_kernel<FP8, false, true>), grid, threads, 0, st, a);
            else hipLaunchKernelGGL((extend_short_kernel<FP8, false, false>), grid, threads, 0, st, a);
        };
        if (c.fp8) launch(std::true_type{});
        else launch(std::false_type{});
    }
    {
        KernelTimer kt("extend_combine", st);
        if (a.few) {
            const int rows = g.T * g.Hq;
            for (int row0 = 0; row0 < rows; row0 += kShortRows)
                hipLaunchKernelGGL(extend_combine_short_kernel, dim3(rows - row0 < kShortRows ? rows - row0 : kShortRows), dim3(32 * kSlices), 0, st, a, row0);
        } else hipLaunchKernelGGL(extend_combine_kernel, dim3(a.most_tiles, a.tile_rows / kCombineRows), dim3(kThreads), 0, st, a);
    }
    return launch_status();
}

}  // namespace l2a
