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
//   kMB       how many splits' partials the merge requests at a time.
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
        constexpr int kPairs = merge_pairs<NW, DH, G>;
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
            if (kKeepNaN || M != kNoMax) {
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
        if (threadIdx.x == 0)
            __hip_atomic_store(&p.pair_counter[head], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        CMC_BUMP();
    }
#undef CMC_BUMP
