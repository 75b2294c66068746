// A KV cache in pages as the kernels see it: [pages, Hkv, page tokens, 128] elements of K and of V, and a table of page numbers per
// sequence.  The rows of a KV head in a page lie one behind the other: what a workgroup reads of a page is one run of memory.
//
// Cache elements of 8 bits are e4m3 in blocks of 32 channels, each with a power of two of its own as a biased exponent: the element
// stands for e4m3 * 2^(exponent - 127).  Four significant bits times a power of two are a bf16 number, so that reading such a cache
// rounds nothing, the conversion instruction takes the scale along, and the matrix cores see bf16 either way.  (One float
// per row would cost the same four bytes, and a multiplication of every score and every weight.)
// Elements of 4 bits are e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6) in the same blocks, the lower channel of a byte in its lower bits; they too are bf16
// numbers with their scale.  The elements hold neither infinities nor NaN: the exponent byte 255 makes a block NaN, which the conversion
// instruction does by itself.
#pragma once
#include "extend_plan.hpp"
#include "mfma.hpp"

namespace l2a {

struct Pages {
    char *k, *v;
    unsigned char *ks, *vs;  // e4m3, e2m1: 4 exponents per row; otherwise null
    const int32_t* table;    // [B, max_pages]
    int pages, page_log2, max_pages, bits;  // bits: of an element, 16 (bf16), 8 (e4m3) or 4 (e2m1)
    __host__ __device__ int capacity() const { return max_pages << page_log2; }
};

constexpr int kScaleBlock = 32;                  // channels that share an exponent
constexpr int kRowScales = kD / kScaleBlock;     // exponents of a row
// of a block: the smallest element (e4m3 2^-9, e2m1 2^-1) and the largest (448, 6) times 2 to these are bf16 numbers
template <int BITS>
constexpr int kMinExponent = BITS == 8 ? -118 : -125;
template <int BITS>
constexpr int kMaxExponent = BITS == 8 ? 119 : 125;

// The row of a token in the pool (rows of all pages counted through), page number p.
__device__ __forceinline__ size_t pool_row(const Pages& c, int hkv, int p, int hk, int t) {
    return (((size_t)p * hkv + hk) << c.page_log2) + (t & ((1 << c.page_log2) - 1));
}
__device__ __forceinline__ plan::Seq seq_at(const Geom& gm, const Pages& c, const int32_t* seq_start, const int32_t* pos, int b, int max_new) {
    return plan::make_seq(seq_start[b], seq_start[b + 1], pos[b], gm.T, max_new, c.capacity());
}
// 2^(e - 127) for the exponents that the cache holds
__device__ __forceinline__ float exponent_value(unsigned e) { return __uint_as_float(e << 23); }

// Eight e2m1 elements -> bf16 values, times `scale`.
__device__ __forceinline__ void dequantise8(uint32_t x, float scale, u32x4& y) {
    y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0));
    y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1));
    y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2));
    y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3));
}
// Sixteen bytes of elements -> bf16 values, all times `scale`: 16 of e4m3 in two vectors, 32 of e2m1 in four.
template <int BITS>
__device__ __forceinline__ void dequantise(const u32x4& x, float scale, u32x4 (&y)[16 / BITS]) {
    if constexpr (BITS == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i >> 1][(i & 1) * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, false));
            y[i >> 1][(i & 1) * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, true));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) dequantise8(x[i], scale, y[i]);
    }
}

// Keys that go straight from memory into an operand of the matrix instructions, a lane a key's row (or, with h, half of it).  Slot (ks, h) of the
// products over the channels stands for eight channels from here on, so that what a lane loads at once, 16 bytes of a row, is whole slots of its half.
template <int BITS>
__device__ __forceinline__ int slot_channel(int ks, int h) {
    constexpr int kVec = 128 / BITS, kSlots = kVec / 8;
    return (ks / kSlots) * 2 * kVec + h * kVec + (ks % kSlots) * 8;
}
// A lane's bytes of its key, and the operand they become.
template <int BITS>
struct RawKeys {
    static constexpr int kSlots = 16 / BITS, kLoads = 8 / kSlots;  // slots of a load
    u32x4 x[kLoads];
    uint32_t exponents;
    __device__ __forceinline__ void load(const Pages& c, size_t row, int h) {
        const char* const p = c.k + row * (kD * BITS / 8) + h * 16;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) x[i] = *reinterpret_cast<const u32x4*>(p + i * 32);
        if constexpr (BITS < 16) exponents = *reinterpret_cast<const uint32_t*>(c.ks + row * kRowScales);
    }
    __device__ __forceinline__ void get(int h, bf16x8 (&k)[8]) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if constexpr (BITS == 16) {
                k[i] = __builtin_bit_cast(bf16x8, x[i]);
            } else {
                u32x4 y[kSlots];
                dequantise<BITS>(x[i], exponent_value((exponents >> (BITS == 8 ? 8 * i : 8 * (2 * i + h))) & 0xffu), y);
#pragma unroll
                for (int j = 0; j < kSlots; ++j) k[i * kSlots + j] = __builtin_bit_cast(bf16x8, y[j]);
            }
        }
    }
};

}  // namespace l2a
