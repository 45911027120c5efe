// What the decode kernels share (decode.hip: fp32 and bf16 caches, decode8.hip:
// the 8-bit cache): the ring count's fetch, the combination of a workgroup's
// waves, the publication and merge of the splits, and the count's advance.
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

// The end of a workgroup's walk, after the barrier that follows its waves'
// stores of (m, l, acc) and of the count each has read: the output (S == 1), or
// the split's partial, its arrival and, in the last split to arrive, the
// merge.
//
// Ring count.  It may be advanced only after every wave of the
// sequence's workgroups has read it.  Each wave stores the count it read
// into LDS before the barrier that ends its walk (a store of the loaded
// value, so the read has returned by then); after that barrier one
// arrival per (sequence, kv head) pair goes to the sequence's counter:
//   S == 1: thread 0 of the workgroup, right after the barrier;
//   S > 1: each split arrives on its pair counter after that barrier, and
//     the merging workgroup (the last split of the pair) then arrives for
//     the pair, overlapping its merge loads.
// The last of the Hkv arrivals writes the advanced count and re-arms the
// counter, at its workgroup's end (the arrival's value is waited for only
// there).  No data is published through the counter, so no fence is
// needed.
//
// KeepNaN: a head whose attended scores or values hold a NaN gets NaN (else
// its denominator counts as empty and the head gets zeros).  BySplits: the merge
// requests as many splits' partials at a time as there are, 8 to 32, instead of
// always the same number.
template <int NW, int DH, int G, bool KeepNaN, bool BySplits = false>
__device__ __forceinline__ void finish_pair(const DecodeParams &p, int b, int kvh, int s, const float (&s_m)[NW][G],
                                            const float (&s_l)[NW][G], float (&s_acc)[NW][G][DH],
                                            const int (&s_cnt)[NW], int cnt_now) {
    constexpr int kThreads = NW * kWave;
    const bool bump = p.T_new > 0 && p.W > 0;
    unsigned prev = ~0u;  // the sequence counter before this workgroup's arrival (one lane)
    const auto bump_count = [&]() {
        if (bump && prev == (unsigned)(p.Hkv - 1)) { // one lane per sequence
            p.win_count[b] = cnt_now + p.T_new;
            __hip_atomic_store(&p.seq_counter[b], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    };
    const auto holds = [](float den) { return KeepNaN ? !(den == 0.f) : den > 0.f; };
    const size_t head = (size_t)b * p.Hkv + kvh;
    float *outp = p.out + ((size_t)b * p.Hq + (size_t)kvh * G) * DH;
    __shared__ int s_last;
    if (p.S == 1) {
        // every wave's count read returned before the barrier above
        if (bump && threadIdx.x == 0) prev = arrive_once(p.seq_counter, b, (unsigned)(s_cnt[NW - 1] != INT_MIN));
        for (int t = threadIdx.x; t < G * DH; t += kThreads) {
            const int g = t / DH, d = t % DH;
            float num, den;
            combine_waves<NW, G, DH>(s_m, s_l, s_acc, g, d, num, den);
            outp[t] = holds(den) ? num * __builtin_amdgcn_rcpf(den) : 0.f;
        }
        bump_count();
    } else {
        // Publish this split's partial with agent-coherent 64-bit stores (two
        // dims per thread), wait for them to complete, then arrive on the
        // (b, kv head) counter.
        const size_t part = (head * p.S + s) * G;
        for (int t = threadIdx.x; t < G * DH / 2; t += kThreads) {
            const int g = (2 * t) / DH, d = (2 * t) % DH;
            float n0, n1, den;
            const float M = combine_waves<NW, G, DH>(s_m, s_l, s_acc, g, d, n0, den);
            combine_waves<NW, G, DH>(s_m, s_l, s_acc, g, d + 1, n1, den);
            coherent_store2(&p.part_acc[(part + g) * DH + d], n0, n1);
            if (d == 0) coherent_store2(&p.part_ml[(part + g) * 2], M, den);
        }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (threadIdx.x == 0) {
            const unsigned prev = __hip_atomic_fetch_add(&p.pair_counter[head], 1u, __ATOMIC_RELAXED,
                                                         __HIP_MEMORY_SCOPE_AGENT);
            s_last = prev == (unsigned)(p.S - 1);
        }
        __syncthreads();
        if (!s_last) return;  // workgroup-uniform
        // The last split merges all S partials in fixed split order.  Its
        // first batch of acc partials (up to kMB splits per dim pair) and all
        // (m, l) pairs are requested together, so the merge costs one round
        // trip when S <= kMB; the (m, l) pairs are staged in LDS.  The
        // batch's loads are issued unconditionally (splits past S - 1 reload
        // split S - 1 and are never used): as atomic loads they cannot be
        // speculated, and a branch around each cost about a dozen
        // instructions between the arrival and the merge's data.
        constexpr int kPairs = (G * DH / 2 + kThreads - 1) / kThreads;  // dim pairs per thread
        const auto merge = [&](auto batch) {
            constexpr int kMB = decltype(batch)::value;
            const float *ml = p.part_ml + head * p.S * G * 2;
            const float *ac = p.part_acc + head * p.S * G * DH;
            float *s_ml = &s_acc[0][0][0];  // reuse: S*G*2 <= NW*G*DH floats (S <= 2*DH)
            // The (m, l) pairs are requested first (loads complete in issue
            // order, and the max and the weights need only them), and the barrier
            // that publishes them in LDS waits for LDS alone: the acc partials
            // may still be in flight while the weights are computed, and their
            // first use waits for them.
            const bool ml_first = threadIdx.x < p.S * G;  // the first kThreads pairs
            float2 mlv = make_float2(0.f, 0.f);
            if (ml_first) mlv = coherent_load2(&ml[2 * threadIdx.x]);
            float2 a[kPairs][kMB];
#pragma unroll
            for (int pr = 0; pr < kPairs; ++pr) {
                const int t = threadIdx.x + pr * kThreads;
                const int g = (2 * min(t, G * DH / 2 - 1)) / DH, d = (2 * min(t, G * DH / 2 - 1)) % DH;
#pragma unroll
                for (int j = 0; j < kMB; ++j) a[pr][j] = coherent_load2(&ac[(min(j, p.S - 1) * G + g) * DH + d]);
            }
            if (ml_first) {
                s_ml[2 * threadIdx.x] = mlv.x;
                s_ml[2 * threadIdx.x + 1] = mlv.y;
            }
            for (int t = threadIdx.x + kThreads; t < p.S * G; t += kThreads) {
                const float2 v = coherent_load2(&ml[2 * t]);
                s_ml[2 * t] = v.x;
                s_ml[2 * t + 1] = v.y;
            }
            // this workgroup completes the pair; the arrival overlaps the merge loads
            if (bump && threadIdx.x == 0) prev = arrive_once(p.seq_counter, b, (unsigned)(s_cnt[NW - 1] != INT_MIN));
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0) only: vmcnt and expcnt at their maxima
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int pr = 0; pr < kPairs; ++pr) {
                const int t = threadIdx.x + pr * kThreads;
                if (t >= G * DH / 2) continue;
                const int g = (2 * t) / DH, d = (2 * t) % DH;
                // The first batch's (m, l) pairs read together (splits past S - 1
                // read split S - 1 again), and its terms masked by selects rather
                // than branches: no LDS round trip waits for another.  The max
                // is unchanged by the repeats, and the sums take the splits in
                // order as before.
                float mj[kMB], lj[kMB];
#pragma unroll
                for (int j = 0; j < kMB; ++j) {
                    const float2 v = *reinterpret_cast<const float2 *>(&s_ml[(min(j, p.S - 1) * G + g) * 2]);
                    mj[j] = v.x;
                    lj[j] = v.y;
                }
                float M = kNoMax;
#pragma unroll
                for (int j = 0; j < kMB; ++j) M = fmaxf(M, mj[j]);
                for (int q = kMB; q < p.S; ++q) M = fmaxf(M, s_ml[(q * G + g) * 2]);
                float n0 = 0.f, n1 = 0.f, den = 0.f;
                if (KeepNaN || M != kNoMax) {
#pragma unroll
                    for (int j = 0; j < kMB; ++j) {
                        const bool in = j < p.S;
                        const float f = fast_exp2(mj[j] - M);
                        den = in ? fmaf(f, lj[j], den) : den;
                        n0 = in ? fmaf(f, a[pr][j].x, n0) : n0;
                        n1 = in ? fmaf(f, a[pr][j].y, n1) : n1;
                    }
                    for (int q0 = kMB; q0 < p.S; q0 += kMB) {
                        float2 x[kMB];
#pragma unroll
                        for (int j = 0; j < kMB; ++j)
                            x[j] = q0 + j < p.S ? coherent_load2(&ac[((q0 + j) * G + g) * DH + d])
                                                : make_float2(0.f, 0.f);
#pragma unroll
                        for (int j = 0; j < kMB; ++j) {
                            if (q0 + j < p.S) {
                                const int q = q0 + j;
                                const float f = fast_exp2(s_ml[(q * G + g) * 2] - M);
                                den = fmaf(f, s_ml[(q * G + g) * 2 + 1], den);
                                n0 = fmaf(f, x[j].x, n0);
                                n1 = fmaf(f, x[j].y, n1);
                            }
                        }
                    }
                }
                const float inv = holds(den) ? __builtin_amdgcn_rcpf(den) : 0.f;  // within 1 ulp
                *reinterpret_cast<float2 *>(&outp[g * DH + d]) = make_float2(n0 * inv, n1 * inv);
            }
        };
        constexpr int kMost = kPairs >= 4 ? 8 : 16;
        if constexpr (!BySplits) {
            merge(std::integral_constant<int, kMost>{});
        } else if (p.S <= 8 || kMost == 8) {
            merge(std::integral_constant<int, 8>{});
        } else if (p.S <= 16 || kPairs > 1) {
            merge(std::integral_constant<int, kMost>{});
        } else {
            merge(std::integral_constant<int, kPairs == 1 ? 32 : 8>{});
        }
        if (threadIdx.x == 0)
            __hip_atomic_store(&p.pair_counter[head], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        bump_count();
    }
}

}  // namespace cmc
