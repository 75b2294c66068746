// A KV cache in pages as the kernels see it: [pages, Hkv, page tokens, 128] elements of K and of V, and a table of page numbers per
// sequence.  The rows of a KV head in a page lie one behind the other: what a workgroup reads of a page is one run of memory.
//
// Cache elements of 8 bits are e4m3 in blocks of 32 channels, each with a power of two of its own as a biased exponent: the element
// stands for e4m3 * 2^(exponent - 127).  Four significant bits times a power of two are a bf16 number, so that reading such a cache
// rounds nothing, the conversion instruction takes the scale along, and the matrix cores see bf16 either way.  (One float
// per row would cost the same four bytes, and a multiplication of every score and every weight.)
#pragma once
#include "extend_plan.hpp"
#include "mfma.hpp"

namespace l2a {

struct Pages {
    char *k, *v;
    unsigned char *ks, *vs;  // e4m3: 4 exponents per row; otherwise null
    const int32_t* table;    // [B, max_pages]
    int pages, page_log2, max_pages, fp8;
    __host__ __device__ int capacity() const { return max_pages << page_log2; }
};

constexpr int kScaleBlock = 32;                  // channels that share an exponent
constexpr int kRowScales = kD / kScaleBlock;     // exponents of a row
constexpr int kMinExponent = -118, kMaxExponent = 119;  // 2^-9 (the smallest element) and 448 times these are bf16 numbers

// The row of a token in the pool (rows of all pages counted through), page number p.
__device__ __forceinline__ size_t pool_row(const Pages& c, int hkv, int p, int hk, int t) {
    return (((size_t)p * hkv + hk) << c.page_log2) + (t & ((1 << c.page_log2) - 1));
}
__device__ __forceinline__ plan::Seq seq_at(const Geom& gm, const Pages& c, const int32_t* seq_start, const int32_t* pos, int b, int max_new) {
    return plan::make_seq(seq_start[b], seq_start[b + 1], pos[b], gm.T, max_new, c.capacity());
}
// 2^(e - 127) for the exponents that the cache holds
__device__ __forceinline__ float exponent_value(unsigned e) { return __uint_as_float(e << 23); }

// Sixteen e4m3 elements -> sixteen bf16 values, all times `scale`.
__device__ __forceinline__ void dequantise16(const u32x4& x, float scale, u32x4 (&y)[2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i >> 1][(i & 1) * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, false));
        y[i >> 1][(i & 1) * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, true));
    }
}

}  // namespace l2a
