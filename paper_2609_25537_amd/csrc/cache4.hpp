// The 4-bit cache format (device side), shared by the kernels that write, read
// and attend over it.
//
// A (sequence, kv head)'s rows are held as e2m1 codes, two dims to a byte (the
// even one in the low half), with one e8m0 scale for every 32 dims of a row: scale
// byte s stands for 2^(s - 127), 255 for NaN, and an element's value is code *
// scale.  With a the largest finite magnitude of the 32 elements, s is the least
// byte >= 1 for which a <= 6 * 2^(s - 127), and code = x / scale rounded to nearest
// even (half a step: at most 1/4 of the scale below 2 scales, 1/2 below 4, 1
// above).  Infinities take the largest code; a NaN makes its 32 dims NaN, with
// codes 0, since e2m1 has no code for it.
//
// A row has scales of its own because 4 bits span a factor of 12 only: one scale
// over several rows, as the 8-bit cache has it, would cost the smaller rows most of
// their codes.  With them no append touches another row.
#pragma once

#include "device_common.hpp"

namespace cmc {

constexpr int kGroup4 = 32;  // dims of a scale

// The eight codes of a word as bf16 pairs (dims 2i and 2i + 1) times 2^(e - 127), e
// the bits 23 to 30 of `scale`; its other bits do not count, and e = 255 gives NaN.
// bf16 holds every value of the cache that fp32 holds.
template <int I>
__device__ __forceinline__ uint32_t bf16_pair4(uint32_t w, uint32_t scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(scale), I));
}
__device__ __forceinline__ uint4 bf16_word4(uint32_t w, uint32_t scale) {
    return make_uint4(bf16_pair4<0>(w, scale), bf16_pair4<1>(w, scale), bf16_pair4<2>(w, scale), bf16_pair4<3>(w, scale));
}

// Scale byte for the largest magnitude whose fp32 bits are `a` (finite): 6 is
// 1.5 * 2^2.
__device__ __forceinline__ uint32_t scale_byte4(uint32_t a) {
    const int s = (int)(a >> 23) - 2 + ((a & 0x7fffffu) > 0x400000u ? 1 : 0);
    return s < 1 ? 1u : (uint32_t)s;
}

// The largest over a quad of lanes.
__device__ __forceinline__ uint32_t quad_umax(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));  // ^1
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));  // ^2
}

// Eight consecutive elements of a row as loaded: 16 bytes of bf16, 32 of fp32.
template <typename T>
struct Raw8 {
    static constexpr int M = Vec16<T>::N, N = 8 / M;
    uint4 r[N];
    // STREAM: past the caches.
    template <bool STREAM>
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const u32x4 *const at = reinterpret_cast<const u32x4 *>(p) + i;
            const u32x4 x = STREAM ? __builtin_nontemporal_load(at) : *at;
            r[i] = make_uint4(x[0], x[1], x[2], x[3]);
        }
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f[M];
            Vec16<T>::widen(r[i], f);
#pragma unroll
            for (int j = 0; j < M; ++j) x[M * i + j] = f[j];
        }
    }
};

// A word of codes and the scale byte of its 32 dims from eight elements, by four
// neighbouring lanes (a quad) that hold 32 in order.
__device__ __forceinline__ uint32_t quantise4(const float (&x)[8], uint32_t &byte) {
    constexpr uint32_t inf = 0x7f800000u;
    uint32_t a = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(x[e]) & 0x7fffffffu);
    a = quad_umax(a);
    bool nan = false;
    if (__builtin_expect(__any(a >= inf), 0)) {
        nan = a > inf;
        uint32_t f = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t u = __float_as_uint(x[e]) & 0x7fffffffu;
            f = max(f, u < inf ? u : 0u);
        }
        f = quad_umax(f);
        a = a < inf ? a : f;
    }
    const uint32_t s = scale_byte4(a);
    const float scale = __uint_as_float(s << 23);
    uint32_t w = 0;  // the conversion rounds to nearest even and takes what is past 6 scales to 6
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    byte = nan ? 255u : s;
    return nan ? 0u : w;
}

// Where a word of eight dims lies: arrays of one (sequence, kv head), shift =
// log2(Dh / 8).
struct Row4 {
    uint8_t *codes, *scales;
    __device__ __forceinline__ void store(size_t row, int word, int shift, uint32_t w, uint32_t byte) const {
        reinterpret_cast<uint32_t *>(codes)[(row << shift) + word] = w;
        if ((word & 3) == 0) scales[(row << (shift - 2)) + (word >> 2)] = (uint8_t)byte;
    }
    // To be called by whole quads of lanes.
    template <typename T>
    __device__ __forceinline__ void put(size_t row, int word, int shift, const Raw8<T> &raw, bool live) const {
        float x[8];
        raw.widen(x);
        uint32_t byte;
        const uint32_t w = quantise4(x, byte);
        if (live) store(row, word, shift, w, byte);
    }
};

}  // namespace cmc
