// Rows of a paged KV cache written and read back (the cache's layout: paged.hpp).
//
//   write   row of token i of sequence b, at position pos[b] + i - seq_start[b]: copied (bf16), or quantised: with
//           amax = max |x| over the block's 32 channels, e the least integer with amax <= 448 2^e (448: e4m3's largest), y = x 2^-e rounded to
//           nearest, ties to even.  No element passes 448 and the largest passes 224, so that it keeps its 4 bits; the scale itself rounds nothing.
//   read    x = y 2^e, exact in bf16.
//
// Memory-bound: every byte of the new rows and of their cache rows is moved once.  65536 tokens of 8 KV heads read out of an e4m3 cache (407 MB)
// 95 us, 4.3 TB/s (a copy of 4 GiB: 4.75); 8192 written into one (51 MB) 11 us; 7500 of 4 read in bf16 (34 MB) 9.5; 64 written 3.4.
#include "paged.hpp"

namespace l2a {
namespace {

struct RowsArgs {
    Geom gm;  // gm.T = packed tokens
    Pages c;
    char *k, *v;  // [T, Hkv, 128] bf16
    const int32_t *seq_start, *pos;
};

// The sequence that holds packed token i, or -1: the last one that begins at or before i.
__device__ __forceinline__ int seq_of(const RowsArgs& a, int i) {
    int lo = 0, hi = a.gm.B;  // seq_start[lo] <= i < seq_start[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.seq_start[mid] <= i) lo = mid;
        else hi = mid;
    }
    const int s = a.seq_start[lo];
    return i >= s && i < a.seq_start[lo + 1] ? lo : -1;
}

constexpr long long kManyRows = 16384;  // of a call, from which on a group takes several

// The exponent of a block (not biased) whose largest magnitude is amax.
__device__ __forceinline__ int block_exponent(float amax) {
    const unsigned bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 2^8
    return min(max(e, kMinExponent), kMaxExponent);
}

// A row is 16 lanes of 8 channels (bf16) or 8 of 16 (e4m3); a group of them takes ROWS tokens of a KV head, whose loads are on their
// way together, and groups side by side the KV heads: packed rows are read or written as they lie, and ROWS rows of a page are one run.
// blockIdx.y: K or V.  65536 tokens of 8 KV heads out of an e4m3 cache (407 MB) with ROWS = 1 and 8 channels a lane: 139 us.
template <bool FP8, bool READ, int ROWS>
__global__ __launch_bounds__(kThreads) void cache_rows_kernel(RowsArgs a) {
    constexpr int kLanes = FP8 ? 8 : 16;
    const Geom& gm = a.gm;
    const long long unit = (long long)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
    const int c = threadIdx.x % kLanes, block = (int)(unit / gm.Hkv), hk = (int)(unit - (long long)block * gm.Hkv);
    char* const packed = (blockIdx.y ? a.v : a.k) + c * (FP8 ? 32 : 16);
    char* const pool = (blockIdx.y ? a.c.v : a.c.k) + c * 16;
    unsigned char* const scales = (blockIdx.y ? a.c.vs : a.c.ks) + (c >> 1);
    size_t at[ROWS], row[ROWS];  // rows of the pool, and packed
    bool on[ROWS];
    int b = -1;
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int tok = block * ROWS + j;
        on[j] = false, at[j] = 0, row[j] = 0;
        if (tok >= gm.T) continue;
        if (b < 0 || tok >= a.seq_start[b + 1]) b = seq_of(a, tok);
        if (b < 0) continue;
        // places outside the table, and page numbers outside the pool, are never followed
        const long long t = (long long)a.pos[b] + tok - a.seq_start[b];
        if (t < 0 || t >= a.c.capacity()) continue;
        const int page = a.c.table[(size_t)b * a.c.max_pages + (int)(t >> a.c.page_log2)];
        on[j] = page >= 0 && page < a.c.pages;
        at[j] = on[j] ? pool_row(a.c, gm.Hkv, page, hk, (int)t) : 0;
        row[j] = (size_t)tok * gm.Hkv + hk;
    }
    if constexpr (!FP8) {
        u32x4 x[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) x[j] = *reinterpret_cast<const u32x4*>(READ ? pool + at[j] * (kD * 2) : packed + row[j] * (kD * 2));
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) *reinterpret_cast<u32x4*>(READ ? packed + row[j] * (kD * 2) : pool + at[j] * (kD * 2)) = x[j];
    } else if constexpr (READ) {
        u32x4 y[ROWS];
        unsigned e[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) y[j] = *reinterpret_cast<const u32x4*>(pool + at[j] * kD), e[j] = scales[at[j] * kRowScales];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) {
                u32x4 x[2];
                dequantise16(y[j], exponent_value(e[j]), x);
                u32x4* const out = reinterpret_cast<u32x4*>(packed + row[j] * (kD * 2));
                out[0] = x[0], out[1] = x[1];
            }
    } else {
        bf16x8 x[ROWS][2];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) {
                const bf16x8* const in = reinterpret_cast<const bf16x8*>(packed + row[j] * (kD * 2));
                x[j][0] = in[0], x[j][1] = in[1];
            }
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            float f[16], amax = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = on[j] ? (float)x[j][i >> 3][i & 7] : 0.f, amax = fmaxf(amax, fabsf(f[i]));
            amax = fmaxf(amax, __shfl_xor(amax, 1));  // the block's other half
            if (!on[j]) continue;
            const int e = block_exponent(amax);
            const float inv = exponent_value(127 - e), most = 448.f * exponent_value(127 + kMaxExponent);
            if (e == kMaxExponent) {  // bf16 reaches 2^128 (1 - 2^-8), beyond what an element stands for at most, 1.75 2^127
#pragma unroll
                for (int i = 0; i < 16; ++i) f[i] = fabsf(f[i]) < INFINITY ? fminf(fmaxf(f[i], -most), most) : __builtin_nanf("");
            }
            u32x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i] * inv, f[4 * i + 1] * inv, 0, false);
                y[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2] * inv, f[4 * i + 3] * inv, w, true);
            }
            *reinterpret_cast<u32x4*>(pool + at[j] * kD) = y;
            if ((c & 1) == 0) scales[at[j] * kRowScales] = (unsigned char)(e + 127);
        }
    }
}

template <bool FP8, bool READ>
void launch_rows(const RowsArgs& a, hipStream_t st) {
    // short calls: a token each, for more workgroups; long ones: more loads on their way
    constexpr int kMany = 4;
    constexpr long long kGroups = kThreads / (FP8 ? 8 : 16);
    const bool many = (long long)a.gm.T * a.gm.Hkv >= kManyRows;
    const long long units = (many ? ((long long)a.gm.T + kMany - 1) / kMany : a.gm.T) * a.gm.Hkv;
    const dim3 grid((unsigned)((units + kGroups - 1) / kGroups), 2);
    if (many) hipLaunchKernelGGL((cache_rows_kernel<FP8, READ, kMany>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((cache_rows_kernel<FP8, READ, 1>), grid, dim3(kThreads), 0, st, a);
}

}  // namespace

int cache_rows(const Geom& g, const Pages& c, bool read, void* k, void* v, const int32_t* seq_start, const int32_t* pos, hipStream_t st) {
    const RowsArgs a{g, c, (char*)k, (char*)v, seq_start, pos};
    KernelTimer kt(read ? "cache_read" : "cache_write", st);
    if (c.fp8 && read) launch_rows<true, true>(a, st);
    else if (c.fp8) launch_rows<true, false>(a, st);
    else if (read) launch_rows<false, true>(a, st);
    else launch_rows<false, false>(a, st);
    return launch_status();
}

}  // namespace l2a
