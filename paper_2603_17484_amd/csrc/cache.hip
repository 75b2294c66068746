// Rows of a paged KV cache written and read back (the cache's layout: paged.hpp).
//
//   write   row of token i of sequence b, at position pos[b] + i - seq_start[b]: copied (bf16), or quantised: with
//           amax = max |x| over the block's 32 channels, e the least integer with amax <= 448 2^e (448: e4m3's largest), y = x 2^-e rounded to
//           nearest, ties to even.  No element passes 448 and the largest passes 224, so that it keeps its 4 bits; the scale itself rounds nothing.
//   read    x = y 2^e, exact in bf16.
//
// Memory-bound: every byte of the new rows and of their cache rows is moved once.
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

// The exponent of a block (not biased) whose largest magnitude is amax.
__device__ __forceinline__ int block_exponent(float amax) {
    const unsigned bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);  // 448 = 1.75 2^8
    return min(max(e, kMinExponent), kMaxExponent);
}

// Sixteen lanes per row, eight channels each; blockIdx.y: K or V.
template <bool FP8, bool READ>
__global__ __launch_bounds__(kThreads) void cache_rows_kernel(RowsArgs a) {
    const Geom& gm = a.gm;
    const long long row = (long long)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    if (row >= (long long)gm.T * gm.Hkv) return;
    const int tok = (int)(row / gm.Hkv), hk = (int)(row - (long long)tok * gm.Hkv), c = threadIdx.x & 15;
    const int b = seq_of(a, tok);
    if (b < 0) return;
    // places outside the table, and page numbers outside the pool, are never followed
    const long long t = (long long)a.pos[b] + (tok - a.seq_start[b]);
    if (t < 0 || t >= a.c.capacity()) return;
    const int page = a.c.table[(size_t)b * a.c.max_pages + (int)(t >> a.c.page_log2)];
    if (page < 0 || page >= a.c.pages) return;
    const size_t at = pool_row(a.c, gm.Hkv, page, hk, (int)t);
    char* const packed = (blockIdx.y ? a.v : a.k) + (size_t)row * (kD * 2) + c * 16;
    char* const pool = blockIdx.y ? a.c.v : a.c.k;
    if constexpr (!FP8) {
        u32x4* const cell = reinterpret_cast<u32x4*>(pool + at * (kD * 2) + c * 16);
        if (READ) *reinterpret_cast<u32x4*>(packed) = *cell;
        else *cell = *reinterpret_cast<const u32x4*>(packed);
    } else {
        unsigned char* const scale = (blockIdx.y ? a.c.vs : a.c.ks) + at * kRowScales + (c >> 2);
        u32x2* const cell = reinterpret_cast<u32x2*>(pool + at * kD + c * 8);
        if constexpr (READ) {
            const u32x2 y = *cell;
            const float s = exponent_value(*scale);
            u32x4 x;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y[i], s, false));
                x[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y[i], s, true));
            }
            *reinterpret_cast<u32x4*>(packed) = x;
        } else {
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(packed);
            f32x8 f = __builtin_convertvector(x, f32x8);
            float amax = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(f[i]));
            amax = fmaxf(amax, __shfl_xor(amax, 1));
            amax = fmaxf(amax, __shfl_xor(amax, 2));
            const int e = block_exponent(amax);
            const float inv = exponent_value(127 - e), most = 448.f * exponent_value(127 + kMaxExponent);
            if (e == kMaxExponent) {  // bf16 reaches 2^128 (1 - 2^-8), beyond what an element stands for at most, 1.75 2^127
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = fabsf(f[i]) < INFINITY ? fminf(fmaxf(f[i], -most), most) : __builtin_nanf("");
            }
            u32x2 y;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i] * inv, f[4 * i + 1] * inv, 0, false);
                y[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2] * inv, f[4 * i + 3] * inv, w, true);
            }
            *cell = y;
            if ((c & 3) == 0) *scale = (unsigned char)(e + 127);
        }
    }
}

}  // namespace

int cache_rows(const Geom& g, const Pages& c, bool read, void* k, void* v, const int32_t* seq_start, const int32_t* pos, hipStream_t st) {
    const RowsArgs a{g, c, (char*)k, (char*)v, seq_start, pos};
    const long long groups = ((long long)g.T * g.Hkv + kThreads / 16 - 1) / (kThreads / 16);
    if (groups > 0x7fffffffLL) return L2A_ERR_SHAPE;
    const dim3 grid((unsigned)groups, 2);
    KernelTimer kt(read ? "cache_read" : "cache_write", st);
    if (c.fp8 && read) hipLaunchKernelGGL((cache_rows_kernel<true, true>), grid, dim3(kThreads), 0, st, a);
    else if (c.fp8) hipLaunchKernelGGL((cache_rows_kernel<true, false>), grid, dim3(kThreads), 0, st, a);
    else if (read) hipLaunchKernelGGL((cache_rows_kernel<false, true>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((cache_rows_kernel<false, false>), grid, dim3(kThreads), 0, st, a);
    return launch_status();
}

}  // namespace l2a
