// Rows of a paged KV cache written and read back (the cache's layout: paged.hpp).
//
//   write   row of token i of sequence b, at position pos[b] + i - seq_start[b]: copied (bf16), or quantised: with
//           amax = max |x| over the block's 32 channels, e the least integer with amax <= 448 2^e (448: e4m3's largest), y = x 2^-e rounded to
//           nearest, ties to even.  No element passes 448 and the largest passes 224, so that it keeps its 4 bits; the scale itself rounds nothing.
//           In 4 bits (e2m1) alike, with 6 for 448; a block with an infinity or a NaN, which its elements cannot hold, is NaN (exponent byte 255).
//   read    x = y 2^e, exact in bf16.
//
// Memory-bound: every byte of the new rows and of their cache rows is moved once.  65536 tokens of 8 KV heads read out of an e4m3 cache (407 MB)
// 95 us, 4.3 TB/s (a copy of 4 GiB: 4.75), out of one in 4 bits (340 MB) 75; 8192 written into an e4m3 cache (51 MB) 11 us; 7500 of 4 read in bf16 (34 MB) 9.5; 64 written 3.4.
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
template <int BITS>
__device__ __forceinline__ int block_exponent(float amax) {
    const unsigned bits = __float_as_uint(amax);
    // the largest element: 448 = 1.75 2^8, 6 = 1.5 2^2
    const int e = (int)(bits >> 23) - 127 - (BITS == 8 ? 8 : 2) + ((bits & 0x7fffffu) > (BITS == 8 ? 0x600000u : 0x400000u) ? 1 : 0);
    return min(max(e, kMinExponent<BITS>), kMaxExponent<BITS>);
}

// A row is 16 lanes of 8 channels (bf16), 8 of 16 (e4m3), or 8 of twice 8, one in each half of the row (e2m1: what the lanes store of packed rows at once
// are whole lines of memory, 75 us for 89 at 65536 tokens); a group of them takes ROWS tokens of a KV head, whose loads are on their
// way together, and groups side by side the KV heads: packed rows are read or written as they lie, and ROWS rows of a page are one run.
// blockIdx.y: K or V.  65536 tokens of 8 KV heads out of an e4m3 cache (407 MB) with ROWS = 1 and 8 channels a lane: 139 us.
template <int BITS, bool READ, int ROWS>
__global__ __launch_bounds__(kThreads) void cache_rows_kernel(RowsArgs a) {
    constexpr int kLanes = BITS < 16 ? 8 : 16, kRowBytes = kD * BITS / 8;
    const Geom& gm = a.gm;
    const long long unit = (long long)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
    const int c = threadIdx.x % kLanes, block = (int)(unit / gm.Hkv), hk = (int)(unit - (long long)block * gm.Hkv);
    char* const packed = (blockIdx.y ? a.v : a.k) + c * (BITS == 8 ? 32 : 16);
    char* const pool = (blockIdx.y ? a.c.v : a.c.k) + c * (BITS == 4 ? 4 : 16);
    unsigned char* const scales = (blockIdx.y ? a.c.vs : a.c.ks) + (BITS == 4 ? c >> 2 : c >> 1);
    size_t at[ROWS], row[ROWS];  // rows of the pool, and packed
    bool on[ROWS];
    long long place[ROWS];       // of the rows in their sequences
    int page[ROWS];
    // Most groups lie in one sequence, which is looked for once; the table's entries are then on their way together.  (One row's lookups behind the
    // other's: 65536 tokens of 8 KV heads out of a cache in 4 bits 96 us for 89.)
    int b = block * ROWS < gm.T ? seq_of(a, block * ROWS) : -1;
    int start = 0, end = 0;
    long long first = 0;
    auto enter = [&]() __attribute__((always_inline)) {
        if (b >= 0) start = a.seq_start[b], end = a.seq_start[b + 1], first = a.pos[b];
    };
    enter();
    size_t entry[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int tok = block * ROWS + j;
        if (tok < gm.T && (b < 0 || tok >= end)) b = seq_of(a, tok), enter();
        // places outside the table, and page numbers outside the pool, are never followed
        place[j] = first + tok - start;
        on[j] = tok < gm.T && b >= 0 && place[j] >= 0 && place[j] < a.c.capacity();
        entry[j] = on[j] ? (size_t)b * a.c.max_pages + (int)(place[j] >> a.c.page_log2) : 0;
        row[j] = (size_t)tok * gm.Hkv + hk;
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) page[j] = a.c.table[entry[j]];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        on[j] = on[j] && page[j] >= 0 && page[j] < a.c.pages;
        at[j] = on[j] ? pool_row(a.c, gm.Hkv, page[j], hk, (int)place[j]) : 0;
    }
    if constexpr (BITS == 16) {
        u32x4 x[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) x[j] = *reinterpret_cast<const u32x4*>(READ ? pool + at[j] * (kD * 2) : packed + row[j] * (kD * 2));
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) *reinterpret_cast<u32x4*>(READ ? packed + row[j] * (kD * 2) : pool + at[j] * (kD * 2)) = x[j];
    } else if constexpr (READ && BITS == 4) {
        uint32_t y[ROWS][2];
        unsigned e[ROWS][2];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) {
#pragma unroll
                for (int i = 0; i < 2; ++i) y[j][i] = *reinterpret_cast<const uint32_t*>(pool + at[j] * kRowBytes + i * (kRowBytes / 2)), e[j][i] = scales[at[j] * kRowScales + 2 * i];
            }
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) {
#pragma unroll
                for (int i = 0; i < 2; ++i) dequantise8(y[j][i], exponent_value(e[j][i]), *reinterpret_cast<u32x4*>(packed + row[j] * (kD * 2) + i * kD));
            }
    } else if constexpr (BITS == 4) {
        bf16x8 x[ROWS][2];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (on[j]) {
#pragma unroll
                for (int i = 0; i < 2; ++i) x[j][i] = *reinterpret_cast<const bf16x8*>(packed + row[j] * (kD * 2) + i * kD);
            }
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float f[8], amax = 0.f;
                int none = 0;  // something that is no finite number
#pragma unroll
                for (int k = 0; k < 8; ++k) f[k] = on[j] ? (float)x[j][i][k] : 0.f, amax = fmaxf(amax, fabsf(f[k])), none |= !(fabsf(f[k]) < INFINITY);
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o)), none |= __shfl_xor(none, o);  // the block's other lanes
                if (!on[j]) continue;
                const int e = block_exponent<4>(amax);
                const float inv = exponent_value(127 - e);  // (multiplied first: 2^-e itself rounds nothing, of subnormal numbers either)
                // (magnitudes beyond 6 2^kMaxExponent become that)
                uint32_t y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, f[0] * inv, f[1] * inv, 1.f, 0);
                y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(y, f[2] * inv, f[3] * inv, 1.f, 1);
                y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(y, f[4] * inv, f[5] * inv, 1.f, 2);
                y = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(y, f[6] * inv, f[7] * inv, 1.f, 3);
                *reinterpret_cast<uint32_t*>(pool + at[j] * kRowBytes + i * (kRowBytes / 2)) = y;
                if ((c & 3) == 0) scales[at[j] * kRowScales + 2 * i] = (unsigned char)(none ? 255 : e + 127);
            }
        }
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
                dequantise<8>(y[j], exponent_value(e[j]), x);
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
            const int e = block_exponent<8>(amax);
            const float inv = exponent_value(127 - e), most = 448.f * exponent_value(127 + kMaxExponent<8>);
            if (e == kMaxExponent<8>) {  // bf16 reaches 2^128 (1 - 2^-8), beyond what an element stands for at most, 1.75 2^127
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

template <int BITS, bool READ>
void launch_rows(const RowsArgs& a, hipStream_t st) {
    // short calls: a token each, for more workgroups; long ones: more loads on their way
    constexpr int kMany = 4;
    constexpr long long kGroups = kThreads / (BITS < 16 ? 8 : 16);
    const bool many = (long long)a.gm.T * a.gm.Hkv >= kManyRows;
    const long long units = (many ? ((long long)a.gm.T + kMany - 1) / kMany : a.gm.T) * a.gm.Hkv;
    const dim3 grid((unsigned)((units + kGroups - 1) / kGroups), 2);
    if (many) hipLaunchKernelGGL((cache_rows_kernel<BITS, READ, kMany>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((cache_rows_kernel<BITS, READ, 1>), grid, dim3(kThreads), 0, st, a);
}

}  // namespace

int cache_rows(const Geom& g, const Pages& c, bool read, void* k, void* v, const int32_t* seq_start, const int32_t* pos, hipStream_t st) {
    const RowsArgs a{g, c, (char*)k, (char*)v, seq_start, pos};
    KernelTimer kt(read ? "cache_read" : "cache_write", st);
    auto launch = [&](auto bits) {
        if (read) launch_rows<decltype(bits)::value, true>(a, st);
        else launch_rows<decltype(bits)::value, false>(a, st);
    };
    if (c.bits == 16) launch(std::integral_constant<int, 16>{});
    else if (c.bits == 8) launch(std::integral_constant<int, 8>{});
    else launch(std::integral_constant<int, 4>{});
    return launch_status();
}

}  // namespace l2a
