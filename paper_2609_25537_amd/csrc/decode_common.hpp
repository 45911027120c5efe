// What the decode kernels share (decode.hip: fp32 and bf16 caches, decode8.hip:
// the 8-bit cache, decode4.hip: the 4-bit cache): the ring count's fetch, an
// arrival on a counter, the coherent stores of the partials; and, for the first
// two, the combination of a workgroup's waves and how the splits' merge is cut
// (decode4.hip joins both its own way).
#pragma once

#include <float.h>
#include <limits.h>

#include <type_traits>

#include "device_common.hpp"
#include "kernels.hpp"

namespace cmc {

constexpr float kLog2e = 1.4426950408889634f;

// A running max before any key.  Finite, so that a key whose score is -inf
// weighs exp2(-inf) = 0 also where no other key came before it (from -inf
// the difference would be NaN, and with it the whole head).
constexpr float kNoMax = -FLT_MAX;

typedef float floatx4 __attribute__((ext_vector_type(4)));

// Orders this wave's LDS writes before its following LDS reads (and reads
// before later writes).  LDS operations of one wave execute in order, so only
// the compiler must be kept from moving memory accesses across this point; a
// fence would also wait for every outstanding global load, including the
// next block's prefetch.
__device__ __forceinline__ void wave_lds_sync() { asm volatile("" ::: "memory"); }

// 2^x with the hardware instruction alone: results below 2^-126 are 0 (see
// kSmallWeights; the waves' and splits' weights at the merge always take it).
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// The ring count, fetched by a wave with a vector load issued after its
// first K/V loads (nothing waits for it before they are in flight) and read
// where a mask or a ring slot needs it, and at the end of the walk (stored
// into LDS before the arrival).
struct RingCount {
    int raw;
    bool loaded;  // wave-uniform
    __device__ __forceinline__ void load(const int32_t *win_count, int b) {
        if (!loaded) {
            raw = win_count ? __hip_atomic_load(win_count + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
            loaded = true;
        }
    }
    __device__ __forceinline__ int value() const {  // clamped at 0, wave-uniform
        const int c = __builtin_amdgcn_readfirstlane(raw);
        return c < 0 ? 0 : c;
    }
};

// One arrival on a counter (relaxed, agent scope) that returns the previous
// value.  The address goes through a VGPR so that the compiler keeps it a
// single returning atomic: its atomic optimizer would otherwise turn it into
// a wave-wide scan that reads the result at once, and since loads and atomics
// complete in order, that wait would also cover every load issued before.
// As it is, the result is waited for only where it is used.
__device__ __forceinline__ unsigned arrive_once(unsigned *ctrs, int i, unsigned one) {
    int iv;
    asm volatile("v_mov_b32 %0, %1" : "=v"(iv) : "s"(i));
    return __hip_atomic_fetch_add(ctrs + iv, one, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Cross-workgroup publication without device-scope fences.  The partials are
// written and read with relaxed agent-scope atomic accesses (coherent across
// the XCDs' L2 caches, unlike plain accesses), the writer waits until its
// stores have completed (s_waitcnt) before arriving on the counter, and the
// reader issues its loads only after the arrival count has returned.  An
// agent-scope fence would instead write back and invalidate the whole L2 of
// the XCD for every workgroup, which costs microseconds each.
// Two adjacent floats (8-byte aligned) as one 64-bit coherent access.
__device__ __forceinline__ void coherent_store2(float *p, float a, float b) {
    const uint64_t v = (uint64_t)__float_as_uint(a) | ((uint64_t)__float_as_uint(b) << 32);
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 coherent_load2(const float *p) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// Combine the waves' (m, l, acc) of head g, dim d; returns the joint max.
template <int NW, int G, int DH>
__device__ __forceinline__ float combine_waves(const float (&sm)[NW][G], const float (&sl)[NW][G],
                                               const float (&sa)[NW][G][DH], int g, int d, float &num,
                                               float &den) {
    // Every LDS read issued before the first wait, and no branch on M: with
    // no valid key in any wave (M = kNoMax) the weights are 1 against zeros, so
    // num = den = 0.
    float mw[NW], lw[NW], aw[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        mw[w] = sm[w][g];
        lw[w] = sl[w][g];
        aw[w] = sa[w][g][d];
    }
    float M = mw[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, mw[w]);
    num = 0.f;
    den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float f = fast_exp2(mw[w] - M);
        num = fmaf(f, aw[w], num);
        den = fmaf(f, lw[w], den);
    }
    return M;
}

// How the merge of a pair's splits is cut (decode_finish.hpp).
template <int NW, int DH, int G>
constexpr int merge_pairs = (G * DH / 2 + NW * kWave - 1) / (NW * kWave);  // dim pairs per thread
template <int NW, int DH, int G>
constexpr int merge_batch = merge_pairs<NW, DH, G> >= 4 ? 8 : 16;

}  // namespace cmc
