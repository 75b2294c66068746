// Rotary positions with several axes: channel pair i of every row of q and k is turned by the angle pos[axis of i][token] freq[i],
//   (x, y) -> (x cos - y sin, y cos + x sin),
// and back by L2A_ROTARY_INVERSE, which is also the gradient: the turn is orthogonal, its transpose the turn by the opposite angle.
// Pair i is channels i and n + i (n pairs in all), or 2 i and 2 i + 1 with L2A_ROTARY_ADJACENT; channels from 2 n on are copied.
//
// The angle is found in 64 bits, in turns: positions have up to 31 bits, and 24-bit frequencies times them would leave no fraction in 32.
// Two products and a constant are off by 2.5 2^-53 of up to 2^28.4 |freq| turns: below 2^-23 of a turn, at any position, for frequencies up to 1, and in
// proportion beyond.  Cosine and sine are then 32-bit functions of the fraction.
//
// Memory-bound: every row is read once and written once.  A workgroup finds the cosines and sines of its tokens once, for all heads, while
// its first rows are on their way.  16384 tokens of 28 + 4 heads in bf16 (269 MB) 47 us, 5.7 TB/s (a copy of 4 GiB: 4.8; a part stays in the last-level
// cache); 4094 of 32 + 8 in fp32 (168 MB) 35; 64 of 28 + 4 3.2, of which the launch is most.
#include "common.hpp"

namespace l2a {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kAhead = 4;        // rows of a thread on their way together
constexpr int kMostPairs = 64;   // D <= 128
constexpr int kMostTokens = 8;   // of a workgroup
constexpr int kMostGroups = 1 << 23;  // of a launch, whose threads have to be fewer than 2^32

struct RopeArgs {
    const char *q, *k;
    char *q_out, *k_out;
    long long q_stride, k_stride, q_out_stride, k_out_stride;  // bytes from token to token
    const int32_t* pos;  // [axes][tokens]
    const float* freq;
    long long tokens, from;  // from: the launch's first
    int Hq, heads;       // heads: of q (0 without it) and k together
    int pairs, ends[4];  // pairs of the axes up to and with each
    int per;             // tokens of a workgroup
    float sign;
};

template <typename V, int D>
constexpr int row_units = D * (int)sizeof(V{}[0]) / 32;  // threads of a row, two vectors of 16 bytes each

template <typename V, bool ADJACENT>
__device__ __forceinline__ void turn(V& x, V& y, const f32x2* cs) {
    constexpr int N = 16 / sizeof(x[0]);
    if constexpr (ADJACENT) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float a = (float)x[2 * i], b = (float)x[2 * i + 1], c = (float)y[2 * i], d = (float)y[2 * i + 1];
            const f32x2 s = cs[i], t = cs[N / 2 + i];
            x[2 * i] = a * s[0] - b * s[1], x[2 * i + 1] = b * s[0] + a * s[1];
            y[2 * i] = c * t[0] - d * t[1], y[2 * i + 1] = d * t[0] + c * t[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float a = (float)x[i], b = (float)y[i];
            const f32x2 s = cs[i];
            x[i] = a * s[0] - b * s[1], y[i] = b * s[0] + a * s[1];
        }
    }
}

// A thread takes the same two vectors of 16 bytes of row after row: the two halves of its pairs, or neighbours where pairs are adjacent.
template <typename V, int D, bool ADJACENT>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
    constexpr int E = sizeof(V{}[0]), kVec = 16 / E, kUnits = row_units<V, D>;  // bytes of a channel; channels of a vector; threads of a row
    __shared__ f32x2 cs[kMostTokens * kMostPairs];
    const long long token0 = a.from + (long long)blockIdx.x * a.per;
    const int tokens = (int)(a.tokens - token0 < a.per ? a.tokens - token0 : a.per), rows = tokens * a.heads;
    const int unit = threadIdx.x % kUnits, first = threadIdx.x / kUnits, half = a.pairs / kVec;  // half: vectors of the pairs' first channels
    const bool turned = unit < half;
    const int vx = !turned ? 2 * unit : ADJACENT ? 2 * unit : unit, vy = !turned ? 2 * unit + 1 : ADJACENT ? 2 * unit + 1 : unit + half;
    struct Row {
        const char* in;
        char* out;
        int token;
    };
    auto row_at = [&](int r) {
        const int token = r / a.heads, head = r - token * a.heads;
        const bool is_q = head < a.Hq;
        const long long t = token0 + token, at = (long long)(is_q ? head : head - a.Hq) * (D * E);
        return Row{(is_q ? a.q + t * a.q_stride : a.k + t * a.k_stride) + at, (is_q ? a.q_out + t * a.q_out_stride : a.k_out + t * a.k_out_stride) + at, token};
    };
    constexpr int kStep = kThreads / kUnits;
    for (int r0 = first; r0 < rows || r0 == first; r0 += kAhead * kStep) {
        V x[kAhead], y[kAhead];
        Row row[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (r0 + j * kStep < rows) {
                row[j] = row_at(r0 + j * kStep);
                x[j] = reinterpret_cast<const V*>(row[j].in)[vx], y[j] = reinterpret_cast<const V*>(row[j].in)[vy];
            }
        if (r0 == first) {
            for (int i = threadIdx.x; i < tokens * a.pairs; i += kThreads) {
                const int t = i / a.pairs, p = i - t * a.pairs;
                int axis = 0;
#pragma unroll
                for (int e = 0; e < 3; ++e) axis += p >= a.ends[e];
                const double turns = (double)a.pos[axis * a.tokens + token0 + t] * (double)a.freq[p] * 0.15915494309189533577;  // 1 / (2 pi)
                float s, c;
                sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
                cs[i] = f32x2{c, s * a.sign};
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (r0 + j * kStep < rows) {
                if (turned) turn<V, ADJACENT>(x[j], y[j], cs + row[j].token * a.pairs + unit * kVec);
                reinterpret_cast<V*>(row[j].out)[vx] = x[j], reinterpret_cast<V*>(row[j].out)[vy] = y[j];
            }
    }
}

}  // namespace

int rope(const l2a_params& p, const l2a_rotary& r, const void* q, const void* k, const int32_t* pos, void* q_out, void* k_out, hipStream_t st) {
    RopeArgs a{};
    const int each = p.dtype == L2A_BF16 ? 2 : 4;
    a.q = (const char*)q, a.k = (const char*)k, a.q_out = (char*)q_out, a.k_out = (char*)k_out;
    a.q_stride = (long long)(r.q_stride ? r.q_stride : p.Hq * p.D) * each, a.k_stride = (long long)(r.k_stride ? r.k_stride : p.Hkv * p.D) * each;
    a.q_out_stride = (long long)(r.q_out_stride ? r.q_out_stride : p.Hq * p.D) * each;
    a.k_out_stride = (long long)(r.k_out_stride ? r.k_out_stride : p.Hkv * p.D) * each;
    a.pos = pos, a.freq = r.freq;
    a.tokens = (long long)p.B * p.T;
    a.Hq = q ? p.Hq : 0, a.heads = a.Hq + (k ? p.Hkv : 0);
    for (int i = 0; i < 4; ++i) a.ends[i] = a.pairs += i < r.axes ? r.pairs[i] : 0;
    a.sign = r.flags & L2A_ROTARY_INVERSE ? -1.f : 1.f;
    KernelTimer kt("rope", st);
    auto launch = [&](auto vec, auto dim) {
        typedef decltype(vec) V;
        constexpr int D = decltype(dim)::value, kUnits = row_units<V, D>;
        // Tokens of a workgroup: so many that a thread has about one row.  16384 tokens in bf16, us with 1, 2, 4 and 8 tokens: 28 + 4 heads 47, 49, 53, 59; 12 + 1
        // heads 31, 23, 25, 29; 4 heads 18, 11, 9, 9.
        a.per = kThreads / (a.heads * kUnits);
        a.per = a.per < 1 ? 1 : a.per > kMostTokens ? kMostTokens : a.per;
        for (a.from = 0; a.from < a.tokens; a.from += (long long)kMostGroups * a.per) {
            const long long groups = (a.tokens - a.from + a.per - 1) / a.per;
            const dim3 grid((unsigned)(groups < kMostGroups ? groups : kMostGroups));
            if (r.flags & L2A_ROTARY_ADJACENT) hipLaunchKernelGGL((rope_kernel<V, D, true>), grid, dim3(kThreads), 0, st, a);
            else hipLaunchKernelGGL((rope_kernel<V, D, false>), grid, dim3(kThreads), 0, st, a);
        }
    };
    auto launch_dim = [&](auto vec) {
        if (p.D == 128) launch(vec, std::integral_constant<int, 128>{});
        else launch(vec, std::integral_constant<int, 64>{});
    };
    if (p.dtype == L2A_BF16) launch_dim(bf16x8{});
    else launch_dim(f32x4{});
    return launch_status();
}

}  // namespace l2a
