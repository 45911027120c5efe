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
// This is the text of the decode kernels' last part, to be included in their
// bodies: as a function, inlined, it costs the shortest steps 0.5% (8 pairs,
// 768 keys in bf16 8.15 -> 8.20 us).  It uses their p, b, kvh, s, s_m, s_l, s_acc,
// s_cnt, cnt_now, bump, prev, NW, DH, G and kThreads, and
//   kKeepNaN  a head whose attended scores or values hold a NaN gets NaN (else
//             its denominator counts as empty and the head gets zeros);
//   kBySplits the merge requests as many splits' partials at a time as there are,
//             8 to 32, instead of merge_batch always (the 8-bit decode: 8 pairs in
//             4 splits 8.6 us with 32, 7.4 so).
#define CMC_BUMP()                                                                         \
    do {                                                                                 \
        if (bump && prev == (unsigned)(p.Hkv - 1)) { /* one lane per sequence */       \
            p.win_count[b] = cnt_now + p.T_new;                                          \
            __hip_atomic_store(&p.seq_counter[b], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); \
        }                                                                                \
    } while (0)
    const auto holds = [](float den) { return kKeepNaN ? !(den == 0.f) : den > 0.f; };
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
        CMC_BUMP();
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
        constexpr int kPairs = merge_pairs<NW, DH, G>, kMost = merge_batch<NW, DH, G>;
        if constexpr (!kBySplits) {
            constexpr int kMB = kMost;
#include "decode_merge.hpp"
        } else {
            const auto merge = [&](auto batch) {
                constexpr int kMB = decltype(batch)::value;
#include "decode_merge.hpp"
            };
            if (p.S <= 8 || kMost == 8) merge(std::integral_constant<int, 8>{});
            else if (p.S <= 16 || kPairs > 1) merge(std::integral_constant<int, kMost>{});
            else merge(std::integral_constant<int, kPairs == 1 ? 32 : 8>{});
        }
        if (threadIdx.x == 0)
            __hip_atomic_store(&p.pair_counter[head], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        CMC_BUMP();
    }
#undef CMC_BUMP
