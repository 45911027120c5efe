// Norms of query and key heads with their rotation by position, one pass.
//
// For a head x of Dh dims: y = x rsqrt(mean(x^2) + eps) w, then each pair (a, b) of y
// turns by t = pos * inv_freq.  Dh / 16 lanes hold a head, 16 dims each as two
// 16-byte words (of bf16): dims 8 j .. and rot / 2 + 8 j .. where pairs lie half a
// rotation apart, 16 j .. where they are neighbours or not rotated, so that a pair is
// always in one lane and the sum of squares is the only exchange.
//
// A workgroup takes all or some heads of one to four tokens.  Its threads first take
// one sine and cosine each to LDS, which all heads then share: t in turns is reduced
// in fp64 (pos * inv_freq is right to 2^-53 of itself; fp32 would be off by 0.06
// radians at a million), the rest in fp32.
//
// Bound by memory for prompts, by latency for single tokens.
#include <algorithm>

#include "device_common.hpp"
#include "kernels.hpp"

namespace cmc {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// Eight elements as loaded, and stored: fp32 as two words, bf16 as one.
template <typename T>
__device__ __forceinline__ void load8(const T *p, float (&x)[8]) {
    constexpr int M = Vec16<T>::N;
#pragma unroll
    for (int i = 0; i < 8 / M; ++i) {
        float f[M];
        Vec16<T>::widen(reinterpret_cast<const uint4 *>(p)[i], f);
#pragma unroll
        for (int e = 0; e < M; ++e) x[M * i + e] = f[e];
    }
}
__device__ __forceinline__ void store8(void *base, size_t at, bool bf16, const float (&x)[8]) {
    if (bf16) {
        st16_nt(static_cast<uint16_t *>(base) + at, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                               pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
    } else {
        float *p = static_cast<float *>(base) + at;
#pragma unroll
        for (int i = 0; i < 8; i += 4)
            st16_nt(p + i, make_uint4(__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]),
                                      __float_as_uint(x[i + 3])));
    }
}

constexpr int kThreads = 256;

// tokens: a workgroup's; heads: how many of a token's Hq + Hkv (+ Hkv) heads it takes.
template <typename T, int DH>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(RopeParams p, int tokens, int heads, bool q_bf16, bool kv_bf16) {
    constexpr int L = DH / 16;            // lanes to a head
    constexpr int R = kThreads / L;       // heads at a time
    constexpr int kMostTokens = 4;
    __shared__ __attribute__((aligned(16))) float s_cos[kMostTokens][DH / 2], s_sin[kMostTokens][DH / 2];
    const int total = p.B * p.T;
    const int token0 = blockIdx.x * tokens;
    const int mine = min(tokens, total - token0);
    const int half = p.rot >> 1;
    for (int i = threadIdx.x; i < mine * half; i += kThreads) {
        const int t = i / half, f = i - t * half;
        const double turns = (double)p.pos[token0 + t] * ((double)p.inv_freq[f] * 0.15915494309189533577);
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        s_cos[t][f] = c;
        s_sin[t][f] = s;
    }
    __syncthreads();
    const int j = threadIdx.x % L;
    const bool turned = j < p.rot / 16;
    const int da = turned && !p.interleaved ? 8 * j : 16 * j;
    const int db = turned && !p.interleaved ? half + 8 * j : 16 * j + 8;
    const int all = p.Hq + (p.k ? p.Hkv : 0) + (p.v ? p.Hkv : 0);
    const int head0 = blockIdx.y * heads, span = min(heads, all - head0);
    for (int i = threadIdx.x / L; i < mine * span; i += R) {  // whole groups of L lanes
        const int t = i / span;
        const size_t token = token0 + t;
        int h = head0 + (i - t * span);
        const T *src;
        const float *weight = nullptr;
        void *dst;
        size_t to;
        bool bf16 = kv_bf16, value = false;
        if (h < p.Hq) {
            src = static_cast<const T *>(p.q) + token * p.q_stride;
            weight = p.q_weight;
            dst = p.out_q;
            bf16 = q_bf16;
            to = (token * p.Hq + h) * DH;
        } else {
            h -= p.Hq;
            value = h >= p.Hkv;
            h -= value ? p.Hkv : 0;
            src = value ? static_cast<const T *>(p.v) + token * p.v_stride : static_cast<const T *>(p.k) + token * p.k_stride;
            weight = value ? nullptr : p.k_weight;
            dst = value ? p.out_v : p.out_k;
            const int b = (int)token / p.T;
            to = (((size_t)b * p.Hkv + h) * p.T + (token - (size_t)b * p.T)) * DH;
        }
        src += (size_t)h * DH;
        float a[8], b[8];
        load8(src + da, a);
        load8(src + db, b);
        if (weight) {
            float wa[8], wb[8];
            load8(weight + da, wa);
            load8(weight + db, wb);
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(a[e], a[e], fmaf(b[e], b[e], ss));
            ss = lane_reduce<OpSum, 1, L>(ss);
            // Squares out of fp32's range, or with eps below their size near its end, in fp64.
            if (__builtin_expect(ss > 0x1p-80f && ss < 0x1p120f, 1)) {
                const float r = rsqrtf(fmaf(ss, 1.f / DH, p.eps));
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    a[e] = a[e] * r * wa[e];
                    b[e] = b[e] * r * wb[e];
                }
            } else {
                double sd = 0.0;
#pragma unroll
                for (int e = 0; e < 8; ++e) sd += (double)a[e] * a[e] + (double)b[e] * b[e];
#pragma unroll
                for (int m = 1; m < L; m <<= 1) sd += __shfl_xor(sd, m);
                const double r = 1.0 / sqrt(sd / DH + (double)p.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    a[e] = (float)(a[e] * r * wa[e]);
                    b[e] = (float)(b[e] * r * wb[e]);
                }
            }
        }
        if (turned && !value) {
            float c[8], s[8];
            load8(&s_cos[t][8 * j], c);
            load8(&s_sin[t][8 * j], s);
            if (p.interleaved) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float a0 = a[e], a1 = a[e + 1], b0 = b[e], b1 = b[e + 1];
                    const float ca = c[e / 2], sa = s[e / 2], cb = c[4 + e / 2], sb = s[4 + e / 2];
                    a[e] = fmaf(a0, ca, -(a1 * sa));
                    a[e + 1] = fmaf(a1, ca, a0 * sa);
                    b[e] = fmaf(b0, cb, -(b1 * sb));
                    b[e + 1] = fmaf(b1, cb, b0 * sb);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = a[e], y = b[e];
                    a[e] = fmaf(x, c[e], -(y * s[e]));
                    b[e] = fmaf(y, c[e], x * s[e]);
                }
            }
        }
        store8(dst, to + da, bf16, a);
        store8(dst, to + db, bf16, b);
    }
}

template <typename T>
hipError_t launch_type(const RopeParams &p, bool q_bf16, bool kv_bf16, hipStream_t stream) {
    const int total = p.B * p.T;
    const int all = p.Hq + (p.k ? p.Hkv : 0) + (p.v ? p.Hkv : 0);
    const int tokens = total >= 2048 ? 4 : 1;
    const int at_once = kThreads / (p.Dh / 16);
    const int heads = total >= 2048 ? all : std::min(all, at_once);
    const dim3 grid((total + tokens - 1) / tokens, (all + heads - 1) / heads);
#define CMC_LAUNCH(DH_) norm_rope_kernel<T, DH_><<<grid, kThreads, 0, stream>>>(p, tokens, heads, q_bf16, kv_bf16)
    switch (p.Dh) {
        case 64: CMC_LAUNCH(64); break;
        case 128: CMC_LAUNCH(128); break;
        case 256: CMC_LAUNCH(256); break;
        default: return hipErrorInvalidValue;
    }
#undef CMC_LAUNCH
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rope(const RopeParams &p, bool in_bf16, bool q_bf16, bool kv_bf16, hipStream_t stream) {
    return in_bf16 ? launch_type<uint16_t>(p, q_bf16, kv_bf16, stream) : launch_type<float>(p, q_bf16, kv_bf16, stream);
}

}  // namespace cmc
