// Norms of query and key heads with their rotation by position, one pass.
//
// For a head x of Dh dims: y = x rsqrt(mean(x^2) + eps) w, then each pair (a, b) of y
// turns by t = pos * inv_freq.  Dh / 16 lanes hold a head, 16 dims each as two runs of
// eight: dims 8 j .. and rot / 2 + 8 j .. where pairs lie half a rotation apart, 8 j ..
// and Dh / 2 + 8 j .. where they are neighbours, so that a pair is always in one lane
// and the sum of squares is the only exchange.
//
// A workgroup takes one token, every head of it up to 512 threads.  The heads are
// requested first; while they come, the first waves take one sine and cosine each to LDS,
// which all heads then share: t in turns is reduced in fp64 (pos * inv_freq is right to
// 2^-51 of itself, three roundings; fp32 would be off by 0.06 radians at a million), the
// rest in fp32.
//
// Bound by memory for prompts: 8192 tokens of 32 + 16 heads of 128, bf16 to fp32 queries
// and bf16 keys and values, 268 MB in 49.7 us, 5.4 TB/s (four tokens to a workgroup in
// turns of 32 heads, sines first: 62.3).  By latency for single tokens: 2.7 us for one,
// 3.3 for 64 of 80 heads in neighbouring pairs.
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
// FAR: bf16 past the caches, which the output would not fit.
template <bool FAR>
__device__ __forceinline__ void store8(void *head, int d, bool bf16, const float (&x)[8]) {
    if (bf16) {
        const uint4 w = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        uint16_t *const at = static_cast<uint16_t *>(head) + d;
        if constexpr (FAR) st16_nt(at, w);
        else *reinterpret_cast<uint4 *>(at) = w;
    } else {
        float4 *const at = reinterpret_cast<float4 *>(static_cast<float *>(head) + d);
        at[0] = make_float4(x[0], x[1], x[2], x[3]);
        at[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// Eight elements of global memory, requested by themselves.
template <typename T>
struct Raw {
    uint4 r[8 / Vec16<T>::N];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < 8 / Vec16<T>::N; ++i) r[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
};

constexpr int kMostThreads = 512;

// One token, or `heads` of its Hq + Hkv (+ Hkv) heads: a head for every DH / 16 lanes.
template <typename T, int DH, bool FAR>
__global__ __launch_bounds__(kMostThreads) void norm_rope_kernel(RopeParams p, int heads, bool q_bf16, bool kv_bf16) {
    constexpr int L = DH / 16;  // lanes to a head
    __shared__ __attribute__((aligned(16))) float s_cos[DH / 2], s_sin[DH / 2];
    const size_t token = (size_t)blockIdx.z * gridDim.x + blockIdx.x;
    if (token >= (size_t)p.B * p.T) return;  // uniform
    const int half = p.rot >> 1;
    const int j = threadIdx.x % L;
    const bool apart = !p.interleaved && j < p.rot / 16;
    const int da = p.interleaved || apart ? 8 * j : 16 * j;
    const int db = p.interleaved ? DH / 2 + 8 * j : apart ? half + 8 * j : 16 * j + 8;
    const int all = p.Hq + (p.k ? p.Hkv : 0) + (p.v ? p.Hkv : 0);
    const int head = blockIdx.y * heads + threadIdx.x / L;
    const bool live = threadIdx.x / L < heads && head < all;
    const T *src;
    const float *weight;
    void *dst;
    size_t to;
    bool bf16 = kv_bf16, value = false;
    int h = live ? head : 0;
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
    Raw<T> ra, rb;
    ra.load(src + da);
    rb.load(src + db);
    for (int i = threadIdx.x; i < half; i += blockDim.x) {
        const double turns = (double)p.pos[token] * ((double)p.inv_freq[i] * 0.15915494309189533577);
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        s_cos[i] = c;
        s_sin[i] = s;
    }
    __syncthreads();
    if (live) {
        float a[8], b[8];
        load8(reinterpret_cast<const T *>(ra.r), a);
        load8(reinterpret_cast<const T *>(rb.r), b);
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
        if (!value && p.interleaved) {
            const auto turn = [&](float (&x)[8], int d) {
                const float4 c = *reinterpret_cast<const float4 *>(&s_cos[d / 2]), s = *reinterpret_cast<const float4 *>(&s_sin[d / 2]);
                const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = x[2 * e], z = x[2 * e + 1];
                    x[2 * e] = fmaf(y, cs[e], -(z * sn[e]));
                    x[2 * e + 1] = fmaf(z, cs[e], y * sn[e]);
                }
            };
            if (da < p.rot) turn(a, da);  // rot is a multiple of 16
            if (db < p.rot) turn(b, db);
        } else if (!value && apart) {
            float c[8], s[8];
            load8(&s_cos[8 * j], c);
            load8(&s_sin[8 * j], s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = a[e], y = b[e];
                a[e] = fmaf(x, c[e], -(y * s[e]));
                b[e] = fmaf(y, c[e], x * s[e]);
            }
        }
        void *const out = static_cast<char *>(dst) + to * (bf16 ? 2 : 4);
        store8<FAR>(out, da, bf16, a);
        store8<FAR>(out, db, bf16, b);
    }
}

template <typename T>
hipError_t launch_type(const RopeParams &p, bool q_bf16, bool kv_bf16, hipStream_t stream) {
    const int lanes = p.Dh / 16;
    const int all = p.Hq + (p.k ? p.Hkv : 0) + (p.v ? p.Hkv : 0);
    const int groups = (all * lanes + kMostThreads - 1) / kMostThreads;
    const int heads = (all + groups - 1) / groups;
    const int threads = (heads * lanes + 63) / 64 * 64;
    // A grid holds less than 2^32 threads a dimension.
    const int total = p.B * p.T, row = std::min(total, 1 << 22);
    const dim3 grid(row, groups, (total + row - 1LL) / row);
    // Non-temporal stores: 2048 tokens of 32 + 16 heads to bf16 10.9 us (13.0 without),
    // but with fp32 queries, whose lanes write every other 16 bytes at a time, 36 (17.9).
    const bool far = kv_bf16 && (q_bf16 || !p.q) && (long long)p.B * p.T * all * p.Dh >= 1 << 23;
#define CMC_LAUNCH(DH_)                                                                                 \
    far ? norm_rope_kernel<T, DH_, true><<<grid, threads, 0, stream>>>(p, heads, q_bf16, kv_bf16)       \
        : norm_rope_kernel<T, DH_, false><<<grid, threads, 0, stream>>>(p, heads, q_bf16, kv_bf16)
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
