// The 8-bit cache format (device side), shared by the kernels that write,
// read and attend over it.
//
// A (sequence, kv head)'s rows are held as 8-bit codes, with one fp32 scale
// for each block of `block` consecutive rows; an element's value is code *
// scale.  With a the largest finite magnitude of the block's live rows and M
// the codes' largest magnitude, scale = 2^e with e the least integer >= -126
// for which a <= M 2^e, and code = x / scale rounded to nearest even.
//
// The scale is a power of two so that dividing by it is exact: the code's
// rounding is the only one (e4m3: half a step of 2^-3 of the value's binade,
// so at most 2^-4 of the value above 2^-6 scale; int8: scale / 2).  And when a
// block's scale changes because a row was appended, the old rows' codes move
// by whole binades: a falling scale is exact for both codes, a growing one
// costs e4m3 bits only where a code becomes subnormal, and int8 half of the new
// step per binade, one step in all at the largest scale a row has lived
// through.  A scale fitted to a itself would round every old row anew
// each time the maximum moved.
#pragma once

#include <float.h>

#include "device_common.hpp"

namespace cmc {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));

// A constant loaded where it is used, on a rare path: the decode's loop fills the
// scalar registers, and with one more constant kept in them its pointers were spilled
// (batch-1 step 9.05 -> 9.2 us, 64 sequences 36.7 -> 37.1).
__device__ __forceinline__ float made_here(float c) {
    asm("" : "+v"(c));
    return c;
}

// e4m3 (OCP: no infinities, 0x7f and 0xff are NaN).
struct CodeE4M3 {
    static constexpr float kMost = 448.f;
    static constexpr int kTopExp = 8;               // 448 = 1.75 * 2^8
    static constexpr uint32_t kTopFrac = 0x600000;  // .75
    static constexpr bool kHasNaN = true;
    // The largest magnitude of sixteen codes, as a float; NaN codes do not
    // count.  Magnitudes order as their codes do, two to a 32-bit operation.
    __device__ __forceinline__ static float top16(const uint4 &c) {
        u16x2 t = {0, 0};
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, w[i] & 0x007f007fu));
            t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, (w[i] >> 8) & 0x007f007fu));
        }
        uint32_t m = t[0] > t[1] ? t[0] : t[1];
        if (m == 0x7f) {  // a NaN among them
            m = 0;
            for (int i = 0; i < 4; ++i)
                for (int b = 0; b < 32; b += 8) {
                    const uint32_t x = (w[i] >> b) & 0x7f;
                    m = x != 0x7f && x > m ? x : m;
                }
        }
        return __builtin_amdgcn_cvt_pk_f32_fp8((int)m, false)[0];
    }
    // Four values (within [-kMost, kMost] or NaN) to a word of codes.
    __device__ __forceinline__ static uint32_t pack4(float a, float b, float c, float d) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
    __device__ __forceinline__ static void widen4(uint32_t w, float (&f)[4]) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
    }
    // Four codes as fp16, which holds every code exactly, times a power of two.
    __device__ __forceinline__ static void half4(uint32_t w, uint32_t &lo, uint32_t &hi, float by = 1.f) {
        lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, by, false));
        hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, by, true));
    }
    // The factor of 2^-13 that weights times 2^13 leave to a block's codes or to its
    // scale.  The scale takes it where it stays a normal number.  Codes hold it exactly
    // too, but as subnormals, of whose products the matrix units keep a bit less.
    struct Down13 {
        float by;
        __device__ __forceinline__ explicit Down13(float &scale) {
            uint32_t e = __builtin_amdgcn_ubfe(__float_as_uint(scale), 23, 8);
            asm("" : "+v"(e));  // compared as it is, with a constant that needs no register
            const bool small = e < 127 - 113;
            by = ldexpf(1.f, small ? -13 : 0);
            scale = ldexpf(scale, small ? 0 : -13);
        }
        __device__ __forceinline__ void half4(uint32_t w, uint32_t &lo, uint32_t &hi) const { CodeE4M3::half4(w, lo, hi, by); }
    };
};

struct CodeI8 {
    static constexpr float kMost = 127.f;
    static constexpr int kTopExp = 6;               // 127 = 1.984375 * 2^6
    static constexpr uint32_t kTopFrac = 0x7e0000;  // .984375
    static constexpr bool kHasNaN = false;
    __device__ __forceinline__ static float top16(const uint4 &c) {
        typedef short s16x2 __attribute__((ext_vector_type(2)));
        s16x2 hi = {0, 0}, lo = {0, 0};
        const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const s16x2 odd = __builtin_bit_cast(s16x2, w[i]) >> 8, even = __builtin_bit_cast(s16x2, w[i] << 8) >> 8;
            hi = __builtin_elementwise_max(hi, __builtin_elementwise_max(odd, even));
            lo = __builtin_elementwise_min(lo, __builtin_elementwise_min(odd, even));
        }
        const int h = hi[0] > hi[1] ? hi[0] : hi[1], l = lo[0] < lo[1] ? lo[0] : lo[1];
        return (float)(h > -l ? h : -l);
    }
    // Adding 1.5 * 2^23 rounds to an integer (nearest even), whose two's
    // complement the low bits then hold.
    __device__ __forceinline__ static uint32_t pack4(float a, float b, float c, float d) {
        constexpr float kMagic = 12582912.f;
        const uint32_t ab = __builtin_amdgcn_perm(__float_as_uint(b + kMagic), __float_as_uint(a + kMagic), 0x0c0c0400);
        const uint32_t cd = __builtin_amdgcn_perm(__float_as_uint(d + kMagic), __float_as_uint(c + kMagic), 0x0c0c0400);
        return __builtin_amdgcn_perm(cd, ab, 0x05040100);
    }
    __device__ __forceinline__ static void widen4(uint32_t w, float (&f)[4]) {
        f[0] = (float)(int8_t)w;
        f[1] = (float)(int8_t)(w >> 8);
        f[2] = (float)(int8_t)(w >> 16);
        f[3] = (float)((int32_t)w >> 24);
    }
    // fp16 with the bits 0x6400 | u is 1024 + u for u < 1024, and u = code +
    // 128 is the code with its sign bit flipped: subtracting 1152 is exact.  With
    // an exponent DOWN lower all of it is times 2^-DOWN.
    template <int DOWN = 0>
    __device__ __forceinline__ static void half4(uint32_t w, uint32_t &lo, uint32_t &hi) {
        constexpr uint32_t top = (0x64u - (DOWN << 2)) * 0x01010101u;
        constexpr float mid = 1152.f / (1 << DOWN);
        const uint32_t u = w ^ 0x80808080u;
        const halfx2 k = {(_Float16)mid, (_Float16)mid};
        lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(halfx2, __builtin_amdgcn_perm(top, u, 0x04010400)) - k);
        hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(halfx2, __builtin_amdgcn_perm(top, u, 0x04030402)) - k);
    }
    // As CodeE4M3's: whole numbers times 2^-13 are normal, so the codes take it always.
    struct Down13 {
        __device__ __forceinline__ explicit Down13(float &) {}
        __device__ __forceinline__ void half4(uint32_t w, uint32_t &lo, uint32_t &hi) const { CodeI8::half4<13>(w, lo, hi); }
    };
};

// e of the scale 2^e for the largest magnitude whose fp32 bits are `a` (finite).
template <class F>
__device__ __forceinline__ int scale_exp(uint32_t a) {
    const int e = (int)(a >> 23) - 127 - F::kTopExp + ((a & 0x7fffffu) > F::kTopFrac ? 1 : 0);
    return e < -126 ? -126 : e;
}
__device__ __forceinline__ float exp_scale(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// 2^-e: e is at most 122, so this is normal too.
__device__ __forceinline__ float exp_inverse(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }

constexpr uint32_t kInfBits = 0x7f800000u;

// The magnitude bits of x, 0 if it is not finite.
__device__ __forceinline__ uint32_t finite_mag(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < kInfBits ? u : 0u;
}

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));   // ^1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));   // ^2
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));  // ^7
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));  // ^15
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)a[0], (uint32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)b[0], (uint32_t)b[1]);
}

// Code of x / scale with inv = 1 / scale, for any x: infinities take the
// largest code, NaN the NaN code (int8, which has none: 0).
template <class F>
__device__ __forceinline__ float to_code_range(float x, float inv) {
    const float y = __builtin_amdgcn_fmed3f(x * inv, -F::kMost, F::kMost);
    return x == x ? y : (F::kHasNaN ? x : 0.f);
}

// Sixteen consecutive elements of a row as loaded: 32 bytes of bf16, 64 of fp32.
template <typename T>
struct Raw16 {
    static constexpr int M = Vec16<T>::N, N = 16 / M;
    uint4 r[N];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = reinterpret_cast<const uint4 *>(p)[i];
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void widen(float (&x)[16]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float f[M];
            Vec16<T>::widen(r[i], f);
#pragma unroll
            for (int j = 0; j < M; ++j) x[M * i + j] = f[j];
        }
    }
    // The largest magnitude's fp32 bits, infinities and NaN counting.
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                m = max(max(m, max(r[i].x & 0x7fffffffu, r[i].y & 0x7fffffffu)),
                        max(r[i].z & 0x7fffffffu, r[i].w & 0x7fffffffu));
        } else {
            u16x2 t = {0, 0};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t w[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, w[e] & 0x7fff7fffu));
            }
            m = (uint32_t)(t[0] > t[1] ? t[0] : t[1]) << 16;
        }
        return m;
    }
    // The same of the finite elements alone.
    __device__ __forceinline__ uint32_t finite_top() const {
        float x[16];
        widen(x);
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) m = max(m, finite_mag(x[e]));
        return m;
    }
};

template <class F>
__device__ __forceinline__ void widen16(const uint4 &c, float (&x)[16]) {
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float f[4];
        F::widen4(w[q], f);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * q + e] = f[e];
    }
}

// The largest magnitude of a block's old codes as a part of its new maximum.  A
// top of 0 (no live old row, or only zeros) counts for nothing, whatever the old
// scale holds.  Codes may stand for more than fp32's largest number (elements within
// half a step of 2^128, and infinities next to those): they count as that number,
// whose scale is the one that they have.
__device__ __forceinline__ uint32_t old_mag(float codes_top, float old_scale) {
    return codes_top > 0.f ? __float_as_uint(fminf(fabsf(codes_top * old_scale), FLT_MAX)) : 0u;
}

// Codes of sixteen elements.  plain: all of them are finite, so that none
// passes the largest code.
template <class F>
__device__ __forceinline__ uint4 pack16(const float (&x)[16], float inv, bool plain) {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = plain ? x[4 * q + e] * inv : to_code_range<F>(x[4 * q + e], inv);
        w[q] = F::pack4(y[0], y[1], y[2], y[3]);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Codes under a new scale of sixteen codes under an old one, by the scales' ratio:
// the values themselves may lie past fp32's largest number.  Only where all codes are
// 0 may the ratio.
template <class F>
__device__ __forceinline__ uint4 repack16(const uint4 &c, float old_scale, float inv) {
    const float most = made_here(FLT_MAX), ratio = __builtin_amdgcn_fmed3f(old_scale * inv, -most, most);
    float x[16];
    widen16<F>(c, x);
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] *= ratio;
    return pack16<F>(x, 1.f, false);
}

// The ring blocks that an append of T_new rows at slot0 writes: consecutive
// from first, round the ring's nb blocks.
struct TouchedBlocks {
    int first, count, nb;
    __device__ __forceinline__ void set(int slot0, int T_new, int W, int log2_block) {
        nb = (int)(((unsigned)W + (1u << log2_block) - 1u) >> log2_block);
        first = slot0 >> log2_block;
        const int room = W - slot0;  // slots up to the ring's end
        if (T_new <= room) count = ((slot0 + T_new - 1) >> log2_block) - first + 1;
        else count = min(nb, nb - first + ((T_new - room - 1) >> log2_block) + 1);
    }
    __device__ __forceinline__ int block(int i) const { return first + i < nb ? first + i : first + i - nb; }
    __device__ __forceinline__ bool has(int j) const {
        const int d = j - first;
        return (d < 0 ? d + nb : d) < count;
    }
};

// A workgroup of NT threads brings a ring block of K and V of one (sequence, kv
// head) up to date with the rows appended at slot0, of which all make at most
// NT words of 16 codes: the scales from the new rows and the live old ones, then
// the codes.  A thread keeps one word of the new rows, requested together with
// the old codes.  Where no scale moves, only the new rows are written.
// row_shift: log2 of a row's words; filled: slots that are live after the append.
// A barrier is needed before anyone reads the block or another block is begun.
template <typename T, class F, int NT>
__device__ __forceinline__ void append_block(const T *const (&rows)[2], uint8_t *const (&codes)[2], float *const (&scales)[2],
                                             int j, int log2_block, int row_shift, int W, int slot0, int filled, int T_new,
                                             uint32_t (*s_top)[NT / 64]) {
    const int me = threadIdx.x;
    const int s0 = j << log2_block;
    const int words = min(1 << log2_block, filled - s0) << row_shift;
    const int t = me >> row_shift, slot = slot0 + t < W ? slot0 + t : slot0 + t - W;
    const bool mine = t < T_new && slot >> log2_block == j;
    uint4 *base[2];
    float old_scale[2], old_top[2] = {0.f, 0.f};
    Raw16<T> raw[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        base[x] = reinterpret_cast<uint4 *>(codes[x]) + ((size_t)s0 << row_shift);
        old_scale[x] = scales[x][j];
        raw[x].clear();
        if (mine) raw[x].load(rows[x] + (size_t)me * 16);
    }
    const auto is_old = [&](int i) {
        const int d = s0 + (i >> row_shift) - slot0;
        return (d < 0 ? d + W : d) >= T_new;
    };
    constexpr int kTrip = 2;  // words of each array that a thread requests before it looks at the first
#pragma unroll 1
    for (int i0 = me; i0 < words; i0 += NT * kTrip) {
        uint4 c[2][kTrip];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int u = 0; u < kTrip; ++u) c[x][u] = base[x][min(i0 + u * NT, words - 1)];
#pragma unroll
        for (int u = 0; u < kTrip; ++u) {
            if (i0 + u * NT < words && is_old(i0 + u * NT)) {
#pragma unroll
                for (int x = 0; x < 2; ++x) old_top[x] = fmaxf(old_top[x], F::top16(c[x][u]));
            }
        }
    }
    bool plain[2];  // this thread's new words are finite
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        uint32_t top = raw[x].top();
        plain[x] = top < kInfBits;
        if (!plain[x]) top = raw[x].finite_top();
        top = wave_umax(max(top, old_mag(old_top[x], old_scale[x])));
        if ((me & 63) == 0) s_top[x][me >> 6] = top;
    }
    __syncthreads();
    float scale[2], inv[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) top = max(top, s_top[x][w]);
        const int e = scale_exp<F>(top);
        scale[x] = exp_scale(e);
        inv[x] = exp_inverse(e);
        if (mine) {
            float v[16];
            raw[x].widen(v);
            base[x][((slot - s0) << row_shift) + (me & ((1 << row_shift) - 1))] =
                plain[x] ? pack16<F>(v, inv[x], true) : pack16<F>(v, inv[x], false);
        }
    }
    // Old rows are passed by where no scale moved (where one did, codes of the
    // other array come out as they were).
    if (scale[0] != old_scale[0] || scale[1] != old_scale[1]) {
#pragma unroll 1
        for (int i = me; i < words; i += NT)
            if (is_old(i)) {
#pragma unroll
                for (int x = 0; x < 2; ++x) base[x][i] = repack16<F>(base[x][i], old_scale[x], inv[x]);
            }
    }
    if (me == 0) {
        scales[0][j] = scale[0];
        scales[1][j] = scale[1];
    }
}

}  // namespace cmc
