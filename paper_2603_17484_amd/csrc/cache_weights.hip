// The attention weights that cached rows receive from the new tokens of a call:
//   w_j <- decay w_j + sum over the group's heads and the tokens t >= j with a finite log-sum-exp of exp(scale <q_t, k_j> - lse_t),
// rows of the new tokens themselves beginning at zero.  With the log-sum-exps that the attention left, weights need neither V nor a maximum, and
// every key's sum is its own: no key's infinity or NaN enters another's.
//
// A wavefront holds 32 keys in registers as an operand of the matrix instructions (B: a lane owns a key) and walks the rows in
// tiles of 32 (A): S = Q K^T leaves a lane with 16 rows' scores of its key, whose exponentials it adds up.  Nothing is shared between
// wavefronts, so that there are neither atomics nor partial sums, and the order of every sum is fixed.
#include "paged.hpp"

namespace l2a {
namespace {

using plan::Seq;

constexpr int kSub = 32;  // keys of a wavefront

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
};

// Slot (ks, h) of the products over the channels: which eight channels it stands for, so that what a lane loads at once, 16 bytes of a row,
// is whole slots of its own half h.
template <int BITS>
__device__ __forceinline__ int slot_channel(int ks, int h) {
    constexpr int kVec = 128 / BITS, kSlots = kVec / 8;
    return (ks / kSlots) * 2 * kVec + h * kVec + (ks % kSlots) * 8;
}
// The operand of key row `row` of the pool.
template <int BITS>
__device__ __forceinline__ void load_keys(const Pages& c, size_t row, int h, bf16x8 (&k)[8]) {
    constexpr int kVec = 128 / BITS, kSlots = kVec / 8;
    const char* const p = c.k + row * (kD * BITS / 8) + h * 16;
    u32x4 x[8 / kSlots];
#pragma unroll
    for (int i = 0; i < 8 / kSlots; ++i) x[i] = *reinterpret_cast<const u32x4*>(p + i * 32);
    if constexpr (BITS == 16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) k[i] = __builtin_bit_cast(bf16x8, x[i]);
    } else {
        const uint32_t e = *reinterpret_cast<const uint32_t*>(c.ks + row * kRowScales);
#pragma unroll
        for (int i = 0; i < 8 / kSlots; ++i) {
            u32x4 y[kSlots];
            dequantise<BITS>(x[i], exponent_value((e >> (BITS == 8 ? 8 * i : 8 * (2 * i + h))) & 0xffu), y);
#pragma unroll
            for (int j = 0; j < kSlots; ++j) k[i * kSlots + j] = __builtin_bit_cast(bf16x8, y[j]);
        }
    }
}

constexpr int kMostSeqs = 1024;  // of a launch: their lengths are summed in shared memory
constexpr int kWaves = 4;

// Units: 32 keys of a KV head of a sequence.  Those of a KV head lie one behind the other, a wavefront takes every so-manieth.
template <int BITS>
__global__ __launch_bounds__(64 * kWaves) void weights_kernel(WeightsArgs a, int b0) {
    __shared__ int ends[kMostSeqs], sums[kWaves];
    const Geom& gm = a.gm;
    const int seqs = min(gm.B - b0, kMostSeqs), lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, G = gm.G;
    // key blocks of all sequences up to and with each
    int total = 0;
    for (int s0 = 0; s0 < seqs; s0 += 64 * kWaves) {
        const int i = s0 + (int)threadIdx.x;
        int blocks = 0;
        if (i < seqs) {
            const Seq s = seq_at(gm, a.c, a.seq_start, a.pos, b0 + i, a.max_new);
            blocks = s.n ? (s.pos + s.n + kSub - 1) / kSub : 0;
        }
        int upto = blocks;
        for (int o = 1; o < 64; o <<= 1) {
            const int below = __shfl_up(upto, o);
            if (lane >= o) upto += below;
        }
        __syncthreads();
        if (lane == 63) sums[threadIdx.x >> 6] = upto;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) {
            if (w < (int)(threadIdx.x >> 6)) upto += sums[w];
        }
        if (i < seqs) ends[i] = total + upto;
        for (int w = 0; w < kWaves; ++w) total += sums[w];
    }
    __syncthreads();
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const long long units = (long long)total * gm.Hkv;
    for (long long u = (long long)blockIdx.x * kWaves + (threadIdx.x >> 6); u < units; u += (long long)gridDim.x * kWaves) {
        const int hk = (int)(u / total), at = (int)(u - (long long)hk * total);
        int lo = 0, hi = seqs - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (ends[mid] > at) hi = mid;
            else lo = mid + 1;
        }
        const int b = b0 + lo, block = at - (lo ? ends[lo - 1] : 0);
        const Seq s = seq_at(gm, a.c, a.seq_start, a.pos, b, a.max_new);
        const int last = s.pos + s.n - 1, key = block * kSub + n, mine = min(key, last);  // (keys behind the last row repeat it, for nobody)
        const int page = a.c.table[(size_t)b * a.c.max_pages + (mine >> a.c.page_log2)];
        const size_t row = pool_row(a.c, gm.Hkv, plan::clamp(page, 0, a.c.pages - 1), hk, mine);
        bf16x8 k[8];
        load_keys<BITS>(a.c, row, h, k);
        float sum = 0.f;
        const int rows = s.n * G, first = max(block * kSub - s.pos, 0) * G;  // rows before see none of these keys
        for (int r0 = first; r0 < rows; r0 += 32) {
            const int r = min(r0 + n, rows - 1), tok = r / G;
            const __bf16* const q = a.q + ((size_t)(s.start + tok) * gm.Hq + hk * G + r - tok * G) * kD;
            f32x16 sc = zero16;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) sc = mfma32(*reinterpret_cast<const bf16x8*>(q + slot_channel<BITS>(ks, h)), k[ks], sc);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int re = r0 + c_row(e, h), te = min(re, rows - 1) / G;
                const float lse = a.lse[(size_t)(hk * G + min(re, rows - 1) - te * G) * gm.T + s.start + te];
                const bool sees = re < rows && s.pos + te >= key && fabsf(lse) < INFINITY;
                sum += sees ? fast_exp2(fmaf(sc[e], gm.scale_log2, -lse * kLog2e)) : 0.f;
            }
        }
        sum += __shfl_xor(sum, 32);
        if (h == 0 && key <= last && (unsigned)page < (unsigned)a.c.pages) {
            if (a.weight_in && key < s.pos) sum = fmaf(a.decay, a.weight_in[row], sum);
            a.weight[row] = sum;
        }
    }
}

}  // namespace

size_t weights_workspace(const Geom&, int) { return 0; }

int cache_weights(const Geom& g, const Pages& c, const void* q, const int32_t* seq_start, const int32_t* pos, const float* lse, int max_new,
                  float decay, const float* weight_in, float* weight, void*, hipStream_t st) {
    const WeightsArgs a{g, c, (const __bf16*)q, seq_start, pos, lse, max_new, decay, weight_in, weight};
    KernelTimer kt("cache_weights", st);
    for (int b0 = 0; b0 < g.B; b0 += kMostSeqs) {
        if (c.bits == 16) hipLaunchKernelGGL(weights_kernel<16>, dim3(1024), dim3(64 * kWaves), 0, st, a, b0);
        else if (c.bits == 8) hipLaunchKernelGGL(weights_kernel<8>, dim3(1024), dim3(64 * kWaves), 0, st, a, b0);
        else hipLaunchKernelGGL(weights_kernel<4>, dim3(1024), dim3(64 * kWaves), 0, st, a, b0);
    }
    return launch_status();
}

}  // namespace l2a
