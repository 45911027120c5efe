// Two-tier decode attention over the 8-bit cache (format: cache8.hpp): softmax
// attention of one query token over [Tier-1 rows || ring slots], optionally
// fused with the append of this step's rows, in one launch.
//
// Grid (S, Hkv, B), 4 waves.  A wave takes units of 32 rows: with c the codes
// and s_K, s_V the scales of the unit's block (a block is a whole number of
// units), it adds
//   x_t = scale log2(e) s_K <q, c_K[t]>        p_t = 2^(x_t - m)
//   l  += sum_t p_t                            acc += s_V sum_t p_t c_V[t]
// with m a running maximum.  Both products run on MFMA (16x16x32, fp16 in, fp32
// sums): codes of 8 bits are exact in fp16, so only q and p have to be split.
//
// Scores: A = 16 rows' codes, B = q, so that a lane ends with the scores of
// one query head (column lane % 16) for 4 + 4 rows.  q, scaled per head by a
// power of two to a maximum in [2^14, 2^15), is held as fp16 hi + lo (22 bits),
// hi in columns 0 .. 7 and lo in columns 8 .. 15 (head = column % G), so one
// MFMA takes both and a row rotate by 8 adds them.
// P V: the same lanes hold p in the A layout as it stands (rows = columns
// before; k slots = the lane's 4 + 4 rows), hi and lo again in rows 0 .. 7 and 8
// .. 15, so p crosses no lane.  V's rows are loaded to match: lane (c, q4) loads
// Dh/16 consecutive codes of rows 4 q4 .. 4 q4 + 3 and 16 + 4 q4 .., and
// interleaves them in registers to the B layout of Dh/16 MFMAs.  One more MFMA
// against ones gives l from the p that V was multiplied with.  p is scaled by
// 2^13: hi + lo hold weights down to 2^-16 of the largest to 22 bits, and
// below that to 2^-38 of the largest.  Each unit's product starts from zero and
// is added with its block's s_V in fp32, so blocks of any scales mix.
//
// The maximum is moved only when a score passes it by more than 2 (p <= 4),
// which after the first units is rare; that test needs no exchange between
// lanes.  The next unit's K is requested when this unit's scores are done,
// its V when this unit's P V is.
//
// Fused append: the last split (its own where the list is split) brings the
// ring blocks that the appended rows touch up to date (append_block), then
// attends over them; every other split leaves those blocks out.  Publication,
// merge and the count's advance are decode.hip's.
#include "cache8.hpp"
#include "decode_common.hpp"

namespace cmc {

namespace {

constexpr int kWeightExp = 13;   // p is held times 2^13
constexpr float kMaxSlack = 2.f; // how far a score may pass the running maximum

template <int NW, class F, int DH, int G>
struct Walk8 {
    static constexpr int SL = DH / 64;  // 16-byte words of a K row per lane; words of a V row per lane
    static constexpr int D = DH / 16;   // output dims per lane
    uint4 kr[2][SL];
    uint32_t vr[8][SL];
    float ks, vs;
    halfx8 q[2 * SL];
    float qf;                 // scale log2(e) over q's power of two
    float m;                  // of head (lane % 16) % G
    floatx4 l, acc[D];        // rows 4 (lane / 16) + i: heads, hi and lo
    int lane, r16, q4;

    __device__ __forceinline__ void init() {
        lane = threadIdx.x & 63;
        r16 = lane & 15;
        q4 = lane >> 4;
        m = kNoMax;
        l = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < D; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    // Rows past `last` are read as row `last`.
    __device__ __forceinline__ void load_k(const char *k, const float *scale, int last) {
        ks = *scale;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t o = (uint32_t)min(16 * t + r16, last) * DH + 16u * q4;
#pragma unroll
            for (int i = 0; i < SL; ++i) kr[t][i] = *reinterpret_cast<const uint4 *>(k + o + 64 * i);
        }
    }
    __device__ __forceinline__ void load_v(const char *v, const float *scale, int last) {
        vs = *scale;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t o = (uint32_t)min((j >> 2) * 16 + 4 * q4 + (j & 3), last) * DH + (uint32_t)D * r16;
            if constexpr (SL == 1) {
                vr[j][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(v + o));
            } else if constexpr (SL == 2) {
                typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
                const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(v + o));
                vr[j][0] = x[0];
                vr[j][1] = x[1];
            } else {
                const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(v + o));
#pragma unroll
                for (int i = 0; i < 4; ++i) vr[j][i] = x[i];
            }
        }
    }

    __device__ __forceinline__ void load_q(const DecodeParams &p, int b, int kvh) {
        const float *qp = p.q + ((size_t)b * p.Hq + (size_t)kvh * G + (r16 % G)) * DH + 16 * q4;
        float x[16 * SL];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < SL; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 f = *reinterpret_cast<const float4 *>(qp + 64 * i + 4 * e);
                x[16 * i + 4 * e] = f.x;
                x[16 * i + 4 * e + 1] = f.y;
                x[16 * i + 4 * e + 2] = f.z;
                x[16 * i + 4 * e + 3] = f.w;
            }
        }
#pragma unroll
        for (int e = 0; e < 16 * SL; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
        const auto a = __builtin_amdgcn_permlane16_swap(top, top, false, false);
        top = max((uint32_t)a[0], (uint32_t)a[1]);
        const auto c = __builtin_amdgcn_permlane32_swap(top, top, false, false);
        top = max((uint32_t)c[0], (uint32_t)c[1]);
        // times 2^(up - 127): up <= 253 keeps the inverse normal
        const int up = min(127 + 14 + 127 - (int)(top >> 23), 253);
        const float mul = copysignf(__uint_as_float((uint32_t)up << 23), p.qscale);
        qf = fabsf(p.qscale) * __uint_as_float((uint32_t)(254 - up) << 23);
        const bool lo = r16 >= 8;
#pragma unroll
        for (int i = 0; i < 2 * SL; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = x[8 * i + e] * mul;
                const _Float16 h = (_Float16)y;
                q[i][e] = lo ? (_Float16)(y - (float)h) : h;
            }
        }
    }

    __device__ __forceinline__ static halfx8 half8(uint32_t a, uint32_t b) {
        uint32_t w[4];
        F::half4(a, w[0], w[1]);
        F::half4(b, w[2], w[3]);
        return __builtin_bit_cast(halfx8, make_uint4(w[0], w[1], w[2], w[3]));
    }

    // Scores (in units of q's power of two and s_K) of rows 16 t + 4 q4 + i.
    __device__ __forceinline__ void scores(floatx4 (&c)[2]) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                c[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(half8(kr[t][i].x, kr[t][i].y), q[2 * i], c[t], 0, 0, 0);
                c[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(half8(kr[t][i].z, kr[t][i].w), q[2 * i + 1], c[t], 0, 0, 0);
            }
        }
    }

    // The unit's share of l and acc; rows n and up are masked.
    __device__ __forceinline__ void add(const floatx4 (&c)[2], float kscale, int n) {
        const bool full = n >= kUnit8;  // uniform
        float x[8];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * t + i] = c[t][i] + dpp_sum_operand<0x128>(c[t][i]);  // hi + lo
        const float f = kscale * qf;
        if (!full) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (e >> 2) * 16 + 4 * q4 + (e & 3) < n ? x[e] : -FLT_MAX;
        }
        const float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))) * f;
        if (__any(top > m + kMaxSlack)) {
            const float mn = fmaxf(m, combine_xor32<OpMax>(combine_xor16<OpMax>(top)));
            const float alpha = fast_exp2(m - mn);  // 0 from kNoMax, where l and acc are 0
            m = mn;
            float al[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) al[i] = __shfl(alpha, 4 * q4 + i);  // of row 4 q4 + i
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                l[i] *= al[i];
#pragma unroll
                for (int j = 0; j < D; ++j) acc[j][i] *= al[i];
            }
        }
        const float mp = m - (float)kWeightExp;
        const float part = r16 >= 8 ? 1.f : 0.f;
        halfx8 P;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float w = fast_exp2(fmaf(x[e], f, -mp));
            if (!full) w = (e >> 2) * 16 + 4 * q4 + (e & 3) < n ? w : 0.f;
            const _Float16 h = (_Float16)w;
            P[e] = (_Float16)fmaf(-(float)h, part, w);  // hi: w itself; lo: what hi leaves
        }
        if (!full && F::kHasNaN) {  // rows past the list may hold any bits, and 0 NaN is NaN
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((j >> 2) * 16 + 4 * q4 + (j & 3) >= n)
#pragma unroll
                    for (int i = 0; i < SL; ++i) vr[j][i] = 0u;
        }
        constexpr _Float16 one = (_Float16)1.f;
        const halfx8 ones = {one, one, one, one, one, one, one, one};
        l = __builtin_amdgcn_mfma_f32_16x16x32_f16(P, ones, l, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < SL; ++w) {
            uint32_t a[8][2];
#pragma unroll
            for (int j = 0; j < 8; ++j) F::half4(vr[j][w], a[j][0], a[j][1]);
            floatx4 t[4];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                uint32_t y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    y[j] = __builtin_amdgcn_perm(a[2 * j + 1][d >> 1], a[2 * j][d >> 1], d & 1 ? 0x07060302 : 0x05040100);
                t[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    P, __builtin_bit_cast(halfx8, make_uint4(y[0], y[1], y[2], y[3])), floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            }
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[4 * w + d][i] = fmaf(vs, t[d][i], acc[4 * w + d][i]);
        }
    }
};

template <int DH>
constexpr int kMinWaves8 = DH <= 128 ? 4 : 2;

// The leading arguments arrive in SGPRs at wave launch, as decode_kernel's do.
template <int NW, class F, int DH, int G>
__global__ __launch_bounds__(NW * kWave, (kMinWaves8<DH>)) void decode8_kernel(const void *cme_k, const void *cme_v,
                                                                               void *win_k, void *win_v, int k, int W,
                                                                               int N, int Hkv, int chunk, int info,
                                                                               Decode8Params pm) {
    Decode8Params p = pm;
    p.k = k;
    p.W = W;
    p.N = N;
    p.Hkv = Hkv;
    p.S = info & 0xFF;
    const bool own = (info >> 8) & 1;
    const bool has_klen = (info >> 10) & 1;
    p.T_new = (int)((unsigned)info >> 16);
    const int s = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int kb = k;
    if (has_klen) {
        const int v = p.k_len[b];
        kb = v < 0 ? 0 : (v > k ? k : v);
    }
    // Units: the pool's, then the ring's in physical slot order.
    const int pool_units = (kb + kUnit8 - 1) / kUnit8;
    const int units = pool_units + (int)(((unsigned)W + kUnit8 - 1) / kUnit8);
    int u = s * chunk, end = min(u + chunk, units);
    if (s >= p.S - 1 - (own ? 1 : 0)) end = units;
    if (own && s == p.S - 1) u = units;

    const size_t head = (size_t)b * Hkv + kvh;
    const char *pk = static_cast<const char *>(cme_k) + head * (size_t)N * DH;
    const char *pv = static_cast<const char *>(cme_v) + head * (size_t)N * DH;
    const char *rk = static_cast<const char *>(win_k) + head * (size_t)W * DH;
    const char *rv = static_cast<const char *>(win_v) + head * (size_t)W * DH;
    const float *pks = p.cme_ks + head * p.pool_blocks, *pvs = p.cme_vs + head * p.pool_blocks;
    float *rks = p.win_ks + head * p.ring_blocks, *rvs = p.win_vs + head * p.ring_blocks;
    const int unit_shift = p.log2_block - 5;  // units per block

    RingCount cnt{0, false};
    Walk8<NW, F, DH, G> st;
    st.init();
    int filled = 0;  // ring slots that hold a key of this step
    TouchedBlocks tb{0, 0, 1};
    bool ready = false;
    const auto after_first_load = [&]() {
        if (ready) return;
        ready = true;
        cnt.load(W > 0 ? p.win_count : nullptr, b);
        st.load_q(p, b, kvh);
        const int c = cnt.value();
        filled = (int)min((long long)c + p.T_new, (long long)W);
        if (p.T_new > 0 && W > 0) tb.set(c % W, p.T_new, W, p.log2_block);
        end = min(end, pool_units + (filled + kUnit8 - 1) / kUnit8);
    };
    // Rows of unit u that take part (0: none), and its addresses.
    const auto rows_of = [&](int u) {
        if (u < pool_units) return kb - u * kUnit8;
        const int r = u - pool_units;
        return tb.has(r >> unit_shift) && tb.count > 0 ? 0 : filled - r * kUnit8;
    };
    const auto load_k = [&](int u) {
        const bool pool = u < pool_units;
        const int r = pool ? u : u - pool_units;
        st.load_k((pool ? pk : rk) + (size_t)r * (kUnit8 * DH), (pool ? pks : rks) + (r >> unit_shift),
                  min(kUnit8, (pool ? kb : W) - r * kUnit8) - 1);
    };
    const auto load_v = [&](int u) {
        const bool pool = u < pool_units;
        const int r = pool ? u : u - pool_units;
        st.load_v((pool ? pv : rv) + (size_t)r * (kUnit8 * DH), (pool ? pvs : rvs) + (r >> unit_shift),
                  min(kUnit8, (pool ? kb : W) - r * kUnit8) - 1);
    };

    u += wave;
    if (u < end) {
        load_k(u);
        load_v(u);
        after_first_load();
#pragma unroll 1
        while (u < end) {
            const int n = rows_of(u), nu = u + NW;
            const float kscale = st.ks;
            floatx4 c[2];
            st.scores(c);
            __builtin_amdgcn_sched_barrier(0);
            if (nu < end) load_k(nu);
            __builtin_amdgcn_sched_barrier(0);
            if (n > 0) st.add(c, kscale, n);
            __builtin_amdgcn_sched_barrier(0);
            if (nu < end) load_v(nu);
            u = nu;
        }
    }
    if (p.T_new > 0 && W > 0 && s == p.S - 1) {  // workgroup-uniform
        after_first_load();
        const int slot0 = cnt.value() % W;
        for (int w = wave; w < 2 * tb.count; w += NW) {
            const bool is_v = w & 1;
            uint8_t *codes = static_cast<uint8_t *>(is_v ? win_v : win_k) + head * (size_t)W * DH;
            float *scales = is_v ? rvs : rks;
            const char *rows = static_cast<const char *>(is_v ? p.new_v : p.new_k);
            const size_t first = head * (size_t)p.T_new * DH;
            constexpr int shift = DH == 64 ? 2 : DH == 128 ? 3 : 4;
            if (p.new_bf16)
                append_block<uint16_t, F>(reinterpret_cast<const uint16_t *>(rows) + first, codes, scales,
                                          tb.block(w >> 1), p.log2_block, shift, W, slot0, filled, p.T_new);
            else
                append_block<float, F>(reinterpret_cast<const float *>(rows) + first, codes, scales, tb.block(w >> 1),
                                       p.log2_block, shift, W, slot0, filled, p.T_new);
        }
        __syncthreads();  // the blocks are in memory, for this workgroup's loads too
        const int per = 1 << unit_shift;
        for (int i = wave; i < tb.count * per; i += NW) {
            const int r = tb.block(i >> unit_shift) * per + (i & (per - 1));
            const int n = filled - r * kUnit8;
            if (n <= 0) continue;
            load_k(pool_units + r);
            load_v(pool_units + r);
            floatx4 c[2];
            st.scores(c);
            st.add(c, st.ks, n);
        }
    }
    cnt.load(W > 0 ? p.win_count : nullptr, b);  // a wave without rows
    const int cnt_now = cnt.value();

    // hi + lo: rows 0 .. 7 of the accumulators' tile and rows 8 .. 15
    constexpr int NH = G < 4 ? G : 4;
    __shared__ __attribute__((aligned(16))) float s_acc[NW][G][DH];
    __shared__ float s_m[NW][G], s_l[NW][G];
    __shared__ int s_cnt[NW];
    constexpr int D = DH / 16;
#pragma unroll
    for (int i = 0; i < NH; ++i) {
        float t[D];
#pragma unroll
        for (int j = 0; j < D; ++j) t[j] = combine_xor32<OpSum>(st.acc[j][i]);
        const float ls = combine_xor32<OpSum>(st.l[i]);
        const int g = 4 * st.q4 + i;
        if (g < G) {
#pragma unroll
            for (int j = 0; j < D; j += 4)
                *reinterpret_cast<float4 *>(&s_acc[wave][g][D * st.r16 + j]) = make_float4(t[j], t[j + 1], t[j + 2], t[j + 3]);
            if (st.r16 == 0) s_l[wave][g] = ls;
        }
    }
    if (st.lane < G) s_m[wave][st.lane] = st.m;
    if (st.lane == 0) s_cnt[wave] = cnt.raw;  // stored once the wave's count read has returned
    __syncthreads();
    finish_pair<NW, DH, G, true>(p, b, kvh, s, s_m, s_l, s_acc, s_cnt, cnt_now);
}

template <class F, int DH, int G>
hipError_t launch3(const Decode8Params &p, hipStream_t stream) {
    const dim3 grid(p.S, p.Hkv, p.B);
    if (p.S < 1 || p.S > 0xFF || p.T_new < 0 || p.T_new > kMaxAppendRows || p.waves != 4) return hipErrorInvalidValue;
    const int info = p.S | (p.new_split << 8) | ((p.k_len != nullptr) << 10) | (p.T_new << 16);
    decode8_kernel<4, F, DH, G><<<grid, 4 * kWave, 0, stream>>>(p.cme_k, p.cme_v, p.win_k, p.win_v, p.k, p.W, p.N, p.Hkv,
                                                                p.chunk, info, p);
    return hipGetLastError();
}

template <class F, int DH>
hipError_t launch_g(const Decode8Params &p, int G, hipStream_t stream) {
    switch (G) {
        case 1: return launch3<F, DH, 1>(p, stream);
        case 2: return launch3<F, DH, 2>(p, stream);
        case 4: return launch3<F, DH, 4>(p, stream);
        case 8: return launch3<F, DH, 8>(p, stream);
    }
    return hipErrorInvalidValue;
}

template <class F>
hipError_t launch_dh(const Decode8Params &p, int G, int Dh, hipStream_t stream) {
    switch (Dh) {
        case 64: return launch_g<F, 64>(p, G, stream);
        case 128: return launch_g<F, 128>(p, G, stream);
        case 256: return launch_g<F, 256>(p, G, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_decode8(const Decode8Params &p, bool e4m3, int G, int Dh, hipStream_t stream) {
    if (p.B == 0) return hipSuccess;
    return e4m3 ? launch_dh<CodeE4M3>(p, G, Dh, stream) : launch_dh<CodeI8>(p, G, Dh, stream);
}

}  // namespace cmc
