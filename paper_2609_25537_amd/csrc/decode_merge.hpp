// The merge of a pair's split partials by the last split to arrive: a part of
// decode_finish.hpp's text, with kPairs (dim pairs per thread) and kMB (how many
// splits' partials are requested at a time) besides its names.
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
