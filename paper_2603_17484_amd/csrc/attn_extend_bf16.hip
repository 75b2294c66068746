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
#include "paged.hpp"
#include "tiles.hpp"

namespace l2a {
namespace {

using plan::kKeys;
using plan::Place;
using plan::Range;
using plan::Seq;

constexpr int kPart = kD + 4;  // floats of a row's sums: maximum (log2 units), sum, 2 unused, O[128]

struct Tile {
    long long start;  // on the line
    int blocks;
    int pair, kind;   // b * Hkv + KV head; plan::kWindow or kPrefix
    int first, rows;  // of the sequence's rows, or of its list
    int lo, hi;       // keys
    int pad;
};
struct Head {
    long long total;
    int per, tiles;
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
    int most_tiles, workgroups, tile_rows;
    int32_t* first_tile;  // [workgroups]
    int32_t* pair_tile;   // [B * Hkv] index of the pair's first tile
    int32_t* listed;      // [B * Hkv] rows with keys before the window
    int32_t* list;        // [Hkv][T G], a sequence's from its first row on: row codes
    int32_t* rank;        // [Hkv][T G] place of a row in its list
    int32_t* token_seq;   // [T]
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
__device__ __forceinline__ int window_tiles(const ExtendArgs& a, const Seq& s) {
    return a.do_local ? (s.n * a.gm.G + a.tile_rows - 1) / a.tile_rows : 0;
}
__device__ __forceinline__ int32_t* list_of(const ExtendArgs& a, int32_t* x, const Seq& s, int hk) {
    return x + (size_t)hk * a.gm.T * a.gm.G + (size_t)s.start * a.gm.G;
}

// Every thread takes consecutive tokens: their decisions counted, the counts summed over the workgroup, the rows written.
constexpr int kListThreads = 1024;
__global__ __launch_bounds__(kListThreads) void extend_list_kernel(ExtendArgs a) {
    __shared__ int sums[kListThreads / 64];
    const Geom& gm = a.gm;
    const int b = blockIdx.x / gm.Hkv, hk = blockIdx.x - b * gm.Hkv, G = gm.G;
    const Seq s = seq_of(a, b);
    if (hk == 0)
        for (int i = threadIdx.x; i < s.n; i += kListThreads) a.token_seq[s.start + i] = b;
    const int skip = plan::rows_without_prefix(s, G, gm.W) / G, n = s.n - skip;
    const int each = (n + kListThreads - 1) / kListThreads;
    const int t0 = min(skip + (int)threadIdx.x * each, s.n), t1 = min(t0 + each, s.n);
    int count = 0;
    for (int t = t0; t < t1; ++t)
        for (int g = 0; g < G; ++g) count += token_routed(a, s.start + t, hk * G + g);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int upto = count;  // of this wavefront's lanes up to this one
    for (int o = 1; o < 64; o <<= 1) {
        const int below = __shfl_up(upto, o);
        if (lane >= o) upto += below;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int at = upto - count, total = 0;
    for (int w = 0; w < kListThreads / 64; ++w) {
        if (w < wave) at += sums[w];
        total += sums[w];
    }
    if (threadIdx.x == 0) a.listed[blockIdx.x] = total;
    int32_t *list = list_of(a, a.list, s, hk), *rank = list_of(a, a.rank, s, hk);
    for (int t = t0; t < t1; ++t)
        for (int g = 0; g < G; ++g)
            if (token_routed(a, s.start + t, hk * G + g)) {
                rank[t * G + g] = at;
                list[at++] = t * G + g;
            }
}

// Sum over the threads before this one, and over all of them.
constexpr int kPlanThreads = 1024;
__device__ __forceinline__ void scan(long long x, long long* sums, long long& before, long long& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    long long upto = x;
    for (int o = 1; o < 64; o <<= 1) {
        const long long below = __shfl_up(upto, o);
        if (lane >= o) upto += below;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    before = upto - x, total = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
}
__global__ __launch_bounds__(kPlanThreads) void extend_plan_kernel(ExtendArgs a) {
    __shared__ long long sums[kPlanThreads / 64];
    __shared__ int ends[kPlanThreads];  // tiles up to and with a pair, of the pairs at hand
    const Geom& gm = a.gm;
    const int pairs = gm.B * gm.Hkv, G = gm.G;
    int tiles = 0;       // of the pairs before
    long long line = 0;  // where the next tile begins
    for (int p0 = 0; p0 < pairs; p0 += kPlanThreads) {
        const int mine = p0 + (int)threadIdx.x;
        int count = 0;
        if (mine < pairs) {
            const Seq s = seq_of(a, mine / gm.Hkv);
            count = window_tiles(a, s) + (a.listed[mine] + a.tile_rows - 1) / a.tile_rows;
        }
        long long before, here;
        scan(count, sums, before, here);
        if (mine < pairs) a.pair_tile[mine] = tiles + (int)before;
        ends[threadIdx.x] = (int)before + count;
        __syncthreads();
        const int of = min(pairs - p0, kPlanThreads);
        for (int i0 = 0; i0 < (int)here; i0 += kPlanThreads) {
            const int i = i0 + (int)threadIdx.x;
            Tile t{};
            const bool on = i < (int)here && tiles + i < a.most_tiles;
            if (on) {
                int lo = 0, hi = of - 1;  // the first pair that ends behind tile i
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (ends[mid] > i) hi = mid;
                    else lo = mid + 1;
                }
                const int pair = p0 + lo, b = pair / gm.Hkv, hk = pair - b * gm.Hkv;
                const Seq s = seq_of(a, b);
                const int windows = window_tiles(a, s), within = i - (lo ? ends[lo - 1] : 0), rows = s.n * G;
                t.pair = pair;
                t.kind = within < windows ? plan::kWindow : plan::kPrefix;
                t.first = (t.kind == plan::kWindow ? within : within - windows) * a.tile_rows;
                t.rows = min(a.tile_rows, (t.kind == plan::kWindow ? rows : min(a.listed[pair], rows)) - t.first);
                int c0 = t.first, c1 = t.first + t.rows - 1;
                if (t.kind == plan::kPrefix) {
                    const int32_t* list = list_of(a, a.list, s, hk);
                    c0 = plan::clamp(list[c0], 0, rows - 1), c1 = plan::clamp(list[c1], 0, rows - 1);
                }
                const Range k = plan::tile_keys(t.kind, s.pos + c0 / G, s.pos + c1 / G, gm.W);
                t.lo = k.lo, t.hi = k.hi;
                t.blocks = plan::tile_blocks(k);
            }
            long long at, sum;
            scan(on ? t.blocks + plan::kStart : 0, sums, at, sum);
            if (on) {
                t.start = line + at;
                a.tiles[tiles + i] = t;
            }
            line += sum;
        }
        tiles += (int)here;
        __syncthreads();
    }
    tiles = min(tiles, a.most_tiles);
    const int per = max(plan::stretch(line, a.workgroups), 1);
    if (threadIdx.x == 0) *a.head = Head{line, per, tiles};
    __syncthreads();
    // the tile each stretch begins in
    for (int i = threadIdx.x; i < tiles; i += kPlanThreads) {
        const Place p{a.tiles[i].start, a.tiles[i].blocks};
        for (long long w = (p.start + per - 1) / per; w * per < p.start + p.length() && w < a.workgroups; ++w) a.first_tile[w] = i;
    }
}

__device__ __forceinline__ void dma16_at(const void* lane_src, unsigned lds_base) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_base), "v"(lane_src) : "memory");
}

struct ExtendLds {
    __bf16 k[2][kKeys * 128];
    __bf16 v[2][kKeys * 128];
};

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

template <bool FP8, int NW>
__global__ __launch_bounds__(64 * NW, 2) void extend_kernel(ExtendArgs a) {
    __shared__ __attribute__((aligned(1024))) ExtendLds lds;
    const Geom& gm = a.gm;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, h = lane >> 5, G = gm.G;
    // workgroups are dealt round-robin to the 8 XCDs: each XCD takes neighbouring stretches
    const int w = (int)(blockIdx.x & 7) * (a.workgroups >> 3) + (int)(blockIdx.x >> 3);
    const Head line = *a.head;
    if ((long long)w * line.per >= line.total) return;
    const long long x1 = (long long)(w + 1) * line.per;

    for (int T = a.first_tile[w]; T < line.tiles; ++T) {
        const Tile t = a.tiles[T];
        if (t.start >= x1) break;
        const plan::Piece piece = plan::piece(Place{t.start, t.blocks}, line.per, w);
        if (piece.from == piece.to) continue;
        const int b = t.pair / gm.Hkv, hk = t.pair - b * gm.Hkv;
        const Seq s = seq_of(a, b);
        const int32_t* table = a.c.table + (size_t)b * a.c.max_pages;

        // ---- this lane's row (rows past the end repeat the last one: computed, never written)
        const int r = wave * 32 + n;
        const bool valid = r < t.rows, wave_on = wave * 32 < t.rows;
        int code = t.first + min(r, t.rows - 1);
        if (t.kind == plan::kPrefix) code = plan::clamp(list_of(a, a.list, s, hk)[code], 0, s.n * G - 1);
        const int local_tok = code / G, g = code - local_tok * G, head = hk * G + g, token = s.start + local_tok, pos = s.pos + local_tok;
        const Range keys = plan::row_keys(t.kind, pos, gm.W);
        const int first_lo = __builtin_amdgcn_readlane(keys.lo, 0), last_lo = __builtin_amdgcn_readlane(keys.lo, 31);
        const int first_hi = __builtin_amdgcn_readlane(keys.hi, 0), last_hi = __builtin_amdgcn_readlane(keys.hi, 31);
        bf16x8 qreg[8];
        const __bf16* qp = a.q + ((size_t)token * gm.Hq + head) * kD + 8 * h;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qreg[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);

        // ---- loads.  Keys out of the tile's range (before its first row's window: their pages may have been given back; behind its
        // last row: not written yet) repeat the nearest one in it: always masked, and what lies in such rows must not meet a zero weight
        const int jb0 = t.lo / kKeys + piece.from, jb1 = t.lo / kKeys + piece.to;  // blocks jb0 .. jb1 - 1
        auto row_at = [&](int key) __attribute__((always_inline)) {
            key = plan::clamp(key, t.lo, t.hi);
            const int page = plan::clamp(table[key >> a.c.page_log2], 0, a.c.pages - 1);
            return pool_row(a.c, gm.Hkv, page, hk, key);
        };
        constexpr int NL = 16 / NW;  // bf16: instructions of a wavefront per K or V block, 4 rows each
        constexpr int NR = 8 / NW;   // e4m3: the same, 8 rows each
        u32x4 kx[NR], vx[NR];
        uint32_t kse[NR], vse[NR];
        auto load = [&](int jb, int buf) __attribute__((always_inline)) {
            if constexpr (!FP8) {
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const int row = (i * NW + wave) * 4 + (lane >> 4);
                    const size_t off = row_at(jb * kKeys + row) * (kD * 2) + (((lane & 15) ^ rm_tr_swizzle(row)) * 16);
                    dma16_at(a.c.k + off, __builtin_amdgcn_readfirstlane(lds_offset(&lds.k[buf][0])) + (i * NW + wave) * 1024);
                    dma16_at(a.c.v + off, __builtin_amdgcn_readfirstlane(lds_offset(&lds.v[buf][0])) + (i * NW + wave) * 1024);
                }
            } else {
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    const size_t at = row_at(jb * kKeys + (i * NW + wave) * 8 + (lane >> 3));
                    kx[i] = *reinterpret_cast<const u32x4*>(a.c.k + at * kD + (lane & 7) * 16);
                    vx[i] = *reinterpret_cast<const u32x4*>(a.c.v + at * kD + (lane & 7) * 16);
                    kse[i] = *reinterpret_cast<const uint32_t*>(a.c.ks + at * kRowScales);
                    vse[i] = *reinterpret_cast<const uint32_t*>(a.c.vs + at * kRowScales);
                }
            }
        };
        auto commit = [&](int buf) __attribute__((always_inline)) {  // e4m3: what was loaded becomes bf16 in LDS
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < NR; ++i) {
                    const int row = (i * NW + wave) * 8 + (lane >> 3), c = 2 * (lane & 7), sh = 8 * ((lane & 7) >> 1);
                    auto put = [&](const u32x4& x, uint32_t e, __bf16* tile) __attribute__((always_inline)) {
                        u32x4 y[2];
                        dequantise16(x, exponent_value((e >> sh) & 0xffu), y);
                        *reinterpret_cast<u32x4*>(tile + row * 128 + ((c ^ rm_tr_swizzle(row)) * 8)) = y[0];
                        *reinterpret_cast<u32x4*>(tile + row * 128 + (((c + 1) ^ rm_tr_swizzle(row)) * 8)) = y[1];
                    };
                    put(kx[i], kse[i], &lds.k[buf][0]);
                    put(vx[i], vse[i], &lds.v[buf][0]);
                }
            }
        };

        f32x16 oacc[4];
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) oacc[d][e] = 0.f;
        const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

        __syncthreads();  // the buffers are free
        load(jb0, 0);
        if constexpr (FP8) {
            commit(0);
            if (jb0 + 1 < jb1) load(jb0 + 1, 0);
        }
        for (int jb = jb0; jb < jb1; ++jb) {
            const int cur = (jb - jb0) & 1;
            if constexpr (!FP8) dma_wait();
            __syncthreads();  // this block is there, and every wavefront is done with the other buffer
            if constexpr (FP8) {
                if (jb + 1 < jb1) commit(cur ^ 1);
                if (jb + 2 < jb1) load(jb + 2, 0);
            } else {
                if (jb + 1 < jb1) load(jb + 1, cur ^ 1);
            }
            const int k0 = jb * kKeys;
            if (!wave_on || k0 > last_hi || k0 + kKeys - 1 < first_lo) continue;
            const bool masked = k0 + kKeys - 1 > first_hi || k0 < last_lo;
            const __bf16 *kt = &lds.k[cur][0], *vt = &lds.v[cur][0];
            f32x16 sc[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) sc[kb] = mfma32(rm_tr_row_operand(kt, kb * 32 + n, ks, h), qreg[ks], ks == 0 ? zero16 : sc[kb]);
            if (masked) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int key = k0 + kb * 32 + c_row(e, h);
                        sc[kb][e] = key >= keys.lo && key <= keys.hi ? sc[kb][e] : -INFINITY;
                    }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[kb][e]);
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float mnew = fmaxf(m, mx * gm.scale_log2);
            if (__any(mnew > m)) {
                const float alpha = mnew > m ? fast_exp2(m - mnew) : 1.f;
                l *= alpha;
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) oacc[d][e] *= alpha;
                m = mnew;
            }
            const float negm = m == -INFINITY ? 0.f : -m;  // no key seen yet
            const bf16x2 one2 = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                u32x4 p[2];
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    f32x2 f = {fast_exp2(fmaf(sc[kb][e], gm.scale_log2, negm)), fast_exp2(fmaf(sc[kb][e + 1], gm.scale_log2, negm))};
                    const bf16x2 pb = __builtin_convertvector(f, bf16x2);
                    // the sum of the weights as the matrix cores see them, rounded to bf16: what they are divided by is exact for them
                    l = __builtin_amdgcn_fdot2_f32_bf16(pb, one2, l, false);
                    p[e >> 3][(e & 7) >> 1] = __builtin_bit_cast(uint32_t, pb);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        oacc[d] = mfma32(rm_tr_col_operand(vt, d, 2 * kb + i, lane), __builtin_bit_cast(bf16x8, p[i]), oacc[d]);
            }
        }

        // ---- out
        if (!valid) continue;
        const float lt = l + __shfl_xor(l, 32);
        const bool whole = piece.first && piece.last;
        if (whole && t.kind == plan::kWindow && !(pos > gm.W && token_routed(a, token, head))) {
            const bool routed = token_routed(a, token, head);  // its window is all there is: a = s
            const float inv = 1.f / lt, lse = (m + __builtin_amdgcn_logf(lt)) * kLn2;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const f32x4 x = {oacc[d][e] * inv, oacc[d][e + 1] * inv, oacc[d][e + 2] * inv, oacc[d][e + 3] * inv};
                    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
                    store_row(a, token, head, d * 32 + c_row(e, h), x, routed ? x : z, lse, routed ? lse : -INFINITY);
                }
            continue;
        }
        float* out = whole ? a.parts[t.kind] + ((size_t)token * gm.Hq + head) * kPart
                           : a.slots + ((size_t)plan::slot(w, piece.first) * a.tile_rows + r) * kPart;
        if (h == 0) *reinterpret_cast<f32x2*>(out) = f32x2{m, lt};
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4*>(out + 4 + d * 32 + c_row(e, h)) = f32x4{oacc[d][e], oacc[d][e + 1], oacc[d][e + 2], oacc[d][e + 3]};
    }
}

// Thirty-two lanes per row, four channels each.
struct Sums {
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void join(float m2, float l2, const f32x4& o2) {
        const float mn = fmaxf(m, m2), ref = mn == -INFINITY ? 0.f : mn;
        const float s0 = fast_exp2(m - ref), s1 = fast_exp2(m2 - ref);
        l = fmaf(l, s0, l2 * s1);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(o[e], s0, o2[e] * s1);
        m = mn;
    }
    __device__ __forceinline__ void join(const float* part, int c4) {
        const f32x2 ml = *reinterpret_cast<const f32x2*>(part);
        join(ml[0], ml[1], *reinterpret_cast<const f32x4*>(part + 4 + c4));
    }
    __device__ __forceinline__ f32x4 value() const { return o / l; }
    __device__ __forceinline__ float lse() const { return (m + __builtin_amdgcn_logf(l)) * kLn2; }
};
__global__ __launch_bounds__(kThreads) void extend_combine_kernel(ExtendArgs a) {
    const Geom& gm = a.gm;
    const int c4 = (threadIdx.x & 31) * 4, G = gm.G;
    const long long row = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (row >= (long long)gm.T * gm.Hq) return;
    const int token = (int)(row / gm.Hq), head = (int)(row - (long long)token * gm.Hq), hk = head / G, g = head - hk * G;
    const int b = a.token_seq[token];  // of a token that is in no sequence: whatever was there
    if (b < 0 || b >= gm.B) return;
    const Seq s = seq_of(a, b);
    const int at = token - s.start;
    if (at < 0 || at >= s.n) return;
    const int pair = b * gm.Hkv + hk, code = at * G + g, per = a.head->per, tiles = a.head->tiles;
    const bool routed = token_routed(a, token, head), prefix = routed && s.pos + at > gm.W;
    Sums sums;
    // the pieces of tile T; false: the tile is whole
    auto pieces = [&](int T, int r) {
        if (T >= tiles) return true;
        const Place p{a.tiles[T].start, a.tiles[T].blocks};
        const int f = plan::first_of(p, per), l = plan::last_of(p, per);
        if (f >= l) return false;
        for (int w = f; w <= l; ++w) sums.join(a.slots + ((size_t)plan::slot(w, w == f) * a.tile_rows + r) * kPart, c4);
        return true;
    };
    const f32x4 z = {0.f, 0.f, 0.f, 0.f};
    f32x4 x = z;
    float lse_l = -INFINITY;
    if (a.do_local) {
        if (!pieces(a.pair_tile[pair] + code / a.tile_rows, code % a.tile_rows)) {
            if (!prefix) return;  // written already
            sums.join(a.parts[plan::kWindow] + (size_t)row * kPart, c4);
        }
        x = sums.value(), lse_l = sums.lse();
    }
    if (prefix) {
        const int i = plan::clamp(list_of(a, a.rank, s, hk)[code], 0, s.n * G - 1);
        if (!pieces(a.pair_tile[pair] + window_tiles(a, s) + i / a.tile_rows, i % a.tile_rows))
            sums.join(a.parts[plan::kPrefix] + (size_t)row * kPart, c4);
    }
    store_row(a, token, head, c4, x, routed ? sums.value() : z, lse_l, routed ? sums.lse() : -INFINITY);
}

constexpr int kTileWaves = 8;
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
    a.tile_rows = 32 * kTileWaves;
    a.most_tiles = (int)(2 * g.Hkv * (rows / a.tile_rows + g.B));
    take(a.head, 1);
    take(a.tiles, a.most_tiles);
    take(a.first_tile, a.workgroups);
    take(a.pair_tile, pairs);
    take(a.listed, pairs);
    take(a.list, rows * g.Hkv);
    take(a.rank, rows * g.Hkv);
    take(a.token_seq, g.T);
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
    {
        KernelTimer kt("extend_list", st);
        hipLaunchKernelGGL(extend_list_kernel, dim3(g.B * g.Hkv), dim3(kListThreads), 0, st, a);
    }
    {
        KernelTimer kt("extend_plan", st);
        hipLaunchKernelGGL(extend_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
    }
    {
        KernelTimer kt("extend", st);
        if (c.fp8) hipLaunchKernelGGL((extend_kernel<true, kTileWaves>), dim3(a.workgroups), dim3(64 * kTileWaves), 0, st, a);
        else hipLaunchKernelGGL((extend_kernel<false, kTileWaves>), dim3(a.workgroups), dim3(64 * kTileWaves), 0, st, a);
    }
    {
        KernelTimer kt("extend_combine", st);
        const long long rows = (long long)g.T * g.Hq;
        hipLaunchKernelGGL(extend_combine_kernel, dim3((unsigned)((rows + kThreads / 32 - 1) / (kThreads / 32))), dim3(kThreads), 0, st, a);
    }
    return launch_status();
}

}  // namespace l2a
