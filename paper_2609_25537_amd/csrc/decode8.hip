// Two-tier decode attention over the 8-bit cache (format: cache8.hpp): softmax
// attention of one query token over [Tier-1 rows || ring slots], optionally
// fused with the append of this step's rows, in one launch.
//
// Grid (S, Hkv, B), 4 or 8 waves.  A wave takes units of 32 rows: with c the codes
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
// is added with its block's s_V in fp32, so blocks of any scales mix; the ones, and
// V's codes or s_V (Down13), take the 2^13 away again, so sums stay within 4 times
// those of the values.
//
// The maximum is moved only when a score passes it by more than 2 (p <= 4),
// which after the first units is rare; that test needs no exchange between
// lanes.  Maxima of 2^22 and more, where fp32 no longer resolves that, move with every
// unit and have their weights' arguments subtracted first.  The next unit's K is
// requested when this unit's scores are done, its V (and its scale before it, which
// the widening of V takes) when this unit's P V is.
//
// Fused append: the last split (one of its own where the plan says so) brings
// the ring blocks that the appended rows touch up to date (append_block), then
// attends over them; every other split leaves them out.  Publication, merge and
// the count's advance are decode.hip's.
//
// Bound by memory where every CU has a full share: 16 sequences of 16 heads of
// 256 (403 MB) 62 us, 6.4 TB/s; 64 of 8 heads of 128, 1536 keys and an append
// (204 MB) 35.5 us, 5.7 TB/s.  Below that by the chain of one workgroup: 9 us
// with 1.6 MB to read (8 pairs), of which the append 1.5.  Vector operations per
// unit of Dh = 128: 189 for e4m3, 280 for int8, which is up to 7% slower (24 sequences
// of 8 heads and 1549 keys in a graph 21.1 / 22.6 us, one sequence of 32808 keys 18.3 /
// 18.8); with the rows' addresses clamped and V widened before its rows are paired
// they were 221 and 317, and times 1 to 2% longer.  The matrix units are busy for less than 10% of the time.
#include <type_traits>

#include "cache8.hpp"
#include "decode_common.hpp"

namespace cmc {

namespace {

constexpr int kWeightExp = 13;   // p is held times 2^13 (Down13 takes it away)
constexpr float kMaxSlack = 2.f; // how far a score may pass a running maximum below 2^22
// Running maxima of 2^22 and more, where fp32 is spaced by a half and more, take the
// weights' argument apart (Walk8::add).
constexpr int kFarExp = 22;

// x f and x f - m with the product rounded on its own: a maximum is such a product,
// so its own difference is 0 (contracted, x f would enter with all its bits).
__device__ __forceinline__ float rounded_product(float x, float f) {
#pragma clang fp contract(off)
    return x * f;
}
__device__ __forceinline__ float product_less(float x, float f, float m) {
#pragma clang fp contract(off)
    const float xf = x * f;
    return xf - m;
}

// Keeps loads after this point from being issued before it, and arithmetic on
// the registers they go to from being moved behind it.
__device__ __forceinline__ void in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

template <int DH>
constexpr int kSets8 = DH == 256 ? 1 : 2;

template <int NW, class F, int DH, int G>
struct Walk8 {
    static constexpr int SL = DH / 64;  // 16-byte words of a K row per lane; words of a V row per lane
    static constexpr int D = DH / 16;   // output dims per lane
    static constexpr int NS = kSets8<DH>;
    // Units on their way or being worked on, each in registers of its own.
    struct Unit {
        uint4 k[2][SL];
        uint32_t v[8][SL];
        float ks, vs;
    } un[NS];
    float4 qx[4 * SL];        // q as loaded
    halfx8 q[2 * SL];
    float qm;                 // scale log2(e) over q's power of two: qm 2^qe
    int qe;
    float m;                  // of head (lane % 16) % G
    float limit;              // the largest score that m may stay for
    floatx4 l, acc[D];        // rows 4 (lane / 16) + i: heads, hi and lo
    int lane, r16, q4;

    __device__ __forceinline__ void init() {
        lane = threadIdx.x & 63;
        r16 = lane & 15;
        q4 = lane >> 4;
        m = kNoMax;
        limit = kNoMax;
        l = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < D; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    // The unit's first `rows` rows, the others as zeros, by the buffer loads'
    // bounds: loads without branches keep the compiler's wait counts exact, and a
    // row costs no address arithmetic (its offset is the lane's and a constant).
    static constexpr int kNonTemporal = 2;
    __device__ __forceinline__ static __amdgpu_buffer_rsrc_t unit_rows(const char *at, int rows) {
        constexpr int untyped = 0x00027000;  // 32-bit elements, addressed by bytes
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, rows * DH, untyped);
    }
    __device__ __forceinline__ void load_k(int set, const char *k, int rows) {
        Unit &n = un[set];
        const __amdgpu_buffer_rsrc_t from = unit_rows(k, rows);
        const int o = r16 * DH + 16 * q4;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(from, o + 16 * t * DH + 64 * i, 0, 0);
                n.k[t][i] = make_uint4(x[0], x[1], x[2], x[3]);
            }
    }
    __device__ __forceinline__ void load_v(int set, const char *v, int rows) {
        Unit &n = un[set];
        const __amdgpu_buffer_rsrc_t from = unit_rows(v, rows);
        const int o = 4 * q4 * DH + D * r16;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = o + ((j >> 2) * 16 + (j & 3)) * DH;
            if constexpr (SL == 1) {
                n.v[j][0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, 0, kNonTemporal);
            } else if constexpr (SL == 2) {
                const auto x = __builtin_amdgcn_raw_buffer_load_b64(from, at, 0, kNonTemporal);
                n.v[j][0] = x[0];
                n.v[j][1] = x[1];
            } else {
                const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, kNonTemporal);
#pragma unroll
                for (int i = 0; i < 4; ++i) n.v[j][i] = x[i];
            }
        }
    }

    // The lane's quarter of its head's q.
    __device__ __forceinline__ void request_q(const DecodeParams &p, int b, int kvh) {
        const float *qp = p.q + ((size_t)b * p.Hq + (size_t)kvh * G + (r16 % G)) * DH + 16 * q4;
#pragma unroll
        for (int i = 0; i < SL; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) qx[4 * i + e] = *reinterpret_cast<const float4 *>(qp + 64 * i + 4 * e);
    }
    __device__ __forceinline__ void split_q(const DecodeParams &p) {
        float x[16 * SL];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4 * SL; ++i) {
            x[4 * i] = qx[i].x;
            x[4 * i + 1] = qx[i].y;
            x[4 * i + 2] = qx[i].z;
            x[4 * i + 3] = qx[i].w;
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
        // Apart: the product of a small scale and a small q's power may be subnormal,
        // and the K scale it meets large.
        const float qs = made_here(p.qscale);
        qm = __builtin_amdgcn_frexp_mantf(fabsf(qs));
        qe = __builtin_amdgcn_frexp_expf(qs) + 127 - up;
        const float part = r16 >= 8 ? 1.f : 0.f;
#pragma unroll
        for (int i = 0; i < 2 * SL; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = x[8 * i + e] * mul;
                const _Float16 h = (_Float16)y;
                q[i][e] = (_Float16)fmaf(-(float)h, part, y);  // hi: y itself; lo: what hi leaves
            }
        }
    }

    // s_K over q's power of two.
    __device__ __forceinline__ float factor(int set) const { return ldexpf(un[set].ks * qm, qe); }

    __device__ __forceinline__ static halfx8 half8(uint32_t a, uint32_t b) {
        uint32_t w[4];
        F::half4(a, w[0], w[1]);
        F::half4(b, w[2], w[3]);
        return __builtin_bit_cast(halfx8, make_uint4(w[0], w[1], w[2], w[3]));
    }

    // Scores (in units of q's power of two and s_K) of rows 16 t + 4 q4 + i.
    __device__ __forceinline__ void scores(int set, floatx4 (&c)[2]) const {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < SL; ++i) {
                c[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(half8(un[set].k[t][i].x, un[set].k[t][i].y), q[2 * i], c[t], 0, 0, 0);
                c[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(half8(un[set].k[t][i].z, un[set].k[t][i].w), q[2 * i + 1], c[t], 0, 0, 0);
            }
        }
    }

    // Has the sums finished here rather than behind the next loads, which would
    // keep this unit's registers and put those loads in others, to be moved (and
    // so waited for) at the end of a turn.
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int j = 0; j < D; ++j) asm volatile("" : "+v"(acc[j]));
        asm volatile("" : "+v"(l));
    }

    // The unit's share of l and acc; f: s_K over q's power of two.  Rows n and up
    // neither count in the maximum nor weigh anything.
    __device__ __forceinline__ void add(int set, const floatx4 (&c)[2], float f, int n) {
        float vs = un[set].vs;
        const typename F::Down13 down(vs);
        float x[8];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * t + i] = c[t][i] + dpp_sum_operand<0x128>(c[t][i]);  // hi + lo
        float top = rounded_product(fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                          fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))), f);
        if (__builtin_expect(__any(f < 0.f), 0))  // a cache made elsewhere may have scales below 0
            top = rounded_product(fminf(fminf(fminf(x[0], x[1]), fminf(x[2], x[3])),
                                        fminf(fminf(x[4], x[5]), fminf(x[6], x[7]))), f);
        const auto live = [&](int e) { return (e >> 2) * 16 + 4 * q4 + (e & 3) < n; };
        if (__builtin_expect(n < kUnit8, 0)) {
            top = made_here(kNoMax);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = live(e) ? fmaxf(top, rounded_product(x[e], f)) : top;
        }
        float mp = m - (float)kWeightExp, by = f;
        if (__builtin_expect(__any(top > limit), 0)) {
            const float mn = fmaxf(m, combine_xor32<OpMax>(combine_xor16<OpMax>(top)));
            const float alpha = fast_exp2(m - mn);  // 0 from kNoMax, where l and acc are 0
            const bool sums = __any(m != made_here(kNoMax));  // not at a wave's first unit
            m = mn;
            const bool far = __builtin_amdgcn_frexp_expf(m) > kFarExp;
            limit = far ? -INFINITY : m + kMaxSlack;  // far maxima come here with every unit
            if (sums) {
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
            mp = far ? 0.f : m - (float)kWeightExp;
            // Below 2^22 the argument x f - mp is off by half the spacing of m and
            // of x f at most, so weights stay under 2^15.6, within fp16.  Above, m - 13
            // may round to m - 16, and the exact product lie far from the rounded one
            // that m is: the largest key's own weight would leave fp16's range at either
            // end.
            if (__builtin_expect(__any(far), 0)) {
                by = far ? 1.f : f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = far ? product_less(x[e], f, m) + (float)kWeightExp : x[e];
            }
        }
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = fast_exp2(fmaf(x[e], by, -mp));
        if (__builtin_expect(n < kUnit8, 0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = live(e) ? w[e] : 0.f;
        }
        const float part = r16 >= 8 ? 1.f : 0.f;
        halfx8 P;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const _Float16 h = (_Float16)w[e];
            P[e] = (_Float16)fmaf(-(float)h, part, w[e]);  // hi: w itself; lo: what hi leaves
        }
        constexpr _Float16 one = (_Float16)(1.f / (1 << kWeightExp));  // a normal fp16 number
        const halfx8 ones = {one, one, one, one, one, one, one, one};
        l = __builtin_amdgcn_mfma_f32_16x16x32_f16(P, ones, l, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < SL; ++w) {
            // Codes of two rows side by side, dim by dim, then widened.
            uint32_t y[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = un[set].v[2 * j][w], b = un[set].v[2 * j + 1][w];
                down.half4(__builtin_amdgcn_perm(b, a, 0x05010400), y[0][j], y[1][j]);
                down.half4(__builtin_amdgcn_perm(b, a, 0x07030602), y[2][j], y[3][j]);
            }
            floatx4 t[4];
#pragma unroll
            for (int d = 0; d < 4; ++d)
                t[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    P, __builtin_bit_cast(halfx8, make_uint4(y[d][0], y[d][1], y[d][2], y[d][3])), floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[4 * w + d][i] = fmaf(vs, t[d][i], acc[4 * w + d][i]);
        }
    }
};

template <int DH>
constexpr int kMinWaves8 = 2;

// decode8_kernel's parameter list as it lies in the kernarg segment: each where its
// alignment puts it, as in a struct.
struct Args8 {
    const void *cme_k, *cme_v;
    void *win_k, *win_v;
    int k, W, N, Hkv, chunk, info;
    Decode8Params p;
};
typedef void (*Kernel8)(const void *, const void *, void *, void *, int, int, int, int, int, int, Decode8Params);
static_assert(sizeof(Args8) == 4 * sizeof(void *) + 6 * sizeof(int) + sizeof(Decode8Params) &&
                  std::is_trivially_copyable_v<Decode8Params>,
              "Args8 holds Kernel8's parameters, in its order and without gaps");

// The last parameter, loaded here and not before (the compiler would load it at
// the kernel's start and wait for it there); fields that nothing uses are not.
__device__ __forceinline__ Decode8Params late_params() {
    typedef const __attribute__((address_space(4))) Args8 *Ptr;
    Ptr at = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    Decode8Params p;
    p.q = at->p.q;
    p.cme_ks = at->p.cme_ks;
    p.cme_vs = at->p.cme_vs;
    p.win_ks = at->p.win_ks;
    p.win_vs = at->p.win_vs;
    p.win_count = at->p.win_count;
    p.new_k = at->p.new_k;
    p.new_v = at->p.new_v;
    p.new_bf16 = at->p.new_bf16;
    p.out = at->p.out;
    p.part_ml = at->p.part_ml;
    p.part_acc = at->p.part_acc;
    p.pair_counter = at->p.pair_counter;
    p.seq_counter = at->p.seq_counter;
    p.Hq = at->p.Hq;
    p.qscale = at->p.qscale;
    p.pool_blocks = at->p.pool_blocks;
    p.ring_blocks = at->p.ring_blocks;
    p.log2_block = at->p.log2_block;
    p.cme_k = at->p.cme_k;
    p.cme_v = at->p.cme_v;
    p.idx = at->p.idx;
    p.k_len = at->p.k_len;
    p.win_k = at->p.win_k;
    p.win_v = at->p.win_v;
    p.k = at->p.k;
    p.W = at->p.W;
    p.B = at->p.B;
    p.Hkv = at->p.Hkv;
    p.N = at->p.N;
    p.T_new = at->p.T_new;
    p.S = at->p.S;
    p.chunk = at->p.chunk;
    p.new_split = at->p.new_split;
    p.waves = at->p.waves;
    return p;
}

// The leading arguments (Args8's, one by one) arrive in SGPRs at wave launch,
// as decode_kernel's do.
template <int NW, class F, int DH, int G>
__global__ __launch_bounds__(NW * kWave, (kMinWaves8<DH>)) void decode8_kernel(const void *cme_k, const void *cme_v,
                                                                               void *win_k, void *win_v, int k, int W,
                                                                               int N, int Hkv, int chunk, int info,
                                                                               Decode8Params pm) {
    const int S = info & 0xFF;
    const bool own = (info >> 8) & 1;
    const int s = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int kb = k;
    if ((info >> 10) & 1) {  // k_len is given
        const int v = pm.k_len[b];
        kb = v < 0 ? 0 : (v > k ? k : v);
    }
    // Units: the pool's, then the ring's in physical slot order.
    const int pool_units = (kb + kUnit8 - 1) / kUnit8;
    const int units = pool_units + (int)(((unsigned)W + kUnit8 - 1) / kUnit8);
    int u = s * chunk, end = min(u + chunk, units);
    if (s >= S - 1 - (own ? 1 : 0)) end = units;
    if (own && s == S - 1) u = units;

    const size_t pair = (size_t)b * Hkv + kvh;
    const char *pk = static_cast<const char *>(cme_k) + pair * (size_t)N * DH;
    const char *pv = static_cast<const char *>(cme_v) + pair * (size_t)N * DH;
    const char *rk = static_cast<const char *>(win_k) + pair * (size_t)W * DH;
    const char *rv = static_cast<const char *>(win_v) + pair * (size_t)W * DH;
    // A unit's place: its first row's codes, its number in its own array, and
    // its live rows.
    struct Place {
        const char *k, *v;
        int r, n;
        bool pool;
    };
    const auto place = [&](int u, int ring_rows) {
        const bool pool = u < pool_units;
        const int r = pool ? u : u - pool_units;
        const size_t o = (size_t)r * (kUnit8 * DH);
        return Place{(pool ? pk : rk) + o, (pool ? pv : rv) + o, r, min(kUnit8, (pool ? kb : ring_rows) - r * kUnit8), pool};
    };
    // The first unit is requested from the leading arguments alone, with all of
    // the ring's slots as live: nothing waits for the others, nor for the count.
    Walk8<NW, F, DH, G> st;
    st.init();
    u += wave;
    const int u0 = u;
    const bool some = u < end;
    Place at{pk, pv, 0, 1, true};
    if (some) {
        at = place(u, W);
        st.load_k(0, at.k, at.n);
        st.load_v(0, at.v, at.n);
    }
    in_order();
    Decode8Params p = late_params();
    p.k = k;
    p.W = W;
    p.N = N;
    p.Hkv = Hkv;
    p.S = S;
    p.T_new = (int)((unsigned)info >> 16);
    const float *pks = p.cme_ks + pair * p.pool_blocks, *pvs = p.cme_vs + pair * p.pool_blocks;
    float *rks = p.win_ks + pair * p.ring_blocks, *rvs = p.win_vs + pair * p.ring_blocks;
    const int unit_shift = p.log2_block - 5;  // units per block
    const auto scale_k = [&](const Place &at) { return (at.pool ? pks : rks)[at.r >> unit_shift]; };
    const auto scale_v = [&](const Place &at) { return (at.pool ? pvs : rvs)[at.r >> unit_shift]; };

    RingCount cnt{0, false};
    int filled = 0;  // ring slots that hold a key of this step
    TouchedBlocks tb{0, 0, 1};
    bool ready = false;
    // q split, and what follows from the count, once both have been requested.
    const auto start = [&]() {
        ready = true;
        st.split_q(p);
        const int c = cnt.value();
        filled = (int)min((long long)c + p.T_new, (long long)W);
        if (p.T_new > 0 && W > 0) tb.set(c % W, p.T_new, W, p.log2_block);
        end = min(end, pool_units + (filled + kUnit8 - 1) / kUnit8);
    };
    const auto touched = [&](int u) { return u >= pool_units && tb.count > 0 && tb.has((u - pool_units) >> unit_shift); };
    const auto after = [&](int u) {  // this wave's next unit, passing by the blocks that are being appended to
        do u += NW;
        while (touched(u) && u < end);
        return u;
    };

    // The units in turn through NS register sets.  In the loop each set's next
    // unit is requested as soon as its registers are free, always: branches
    // around loads would have the waits count for the path without them.  Where
    // there is none left, the last unit is requested again, of which no row
    // counts.  The last NS units are worked off after the loop.
    constexpr int NS = kSets8<DH>;
    if (some) {
        int n[NS];
        st.un[0].ks = scale_k(at);
        st.un[0].vs = scale_v(at);
        in_order();  // before q, whose wait so covers the scales' too
        st.request_q(p, b, kvh);
        cnt.load(W > 0 ? p.win_count : nullptr, b);
        n[0] = at.n;
#pragma unroll
        for (int i = 1; i < NS; ++i) {
            n[i] = 0;
            if (u + NW < end) {
                u += NW;
                at = place(u, W);
                in_order();
                st.load_k(i, at.k, at.n);
                st.un[i].ks = scale_k(at);
                in_order();
                st.un[i].vs = scale_v(at);
                st.load_v(i, at.v, at.n);
                n[i] = at.n;
            }
        }
        start();
        // A unit among them that is being appended to or not filled: once more
        // from the first, as it should have been.
        bool again = false;
        for (int i = 0, v = u0; i < NS; ++i, v += NW)
            again |= v >= pool_units && n[i] > 0 && (touched(v) || v >= end || place(v, filled).n != n[i]);
        if (__builtin_expect(again, 0)) {
            u = u0;
            if (touched(u)) u = after(u);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                if (i > 0 && u < end) u = after(u);
                if (u < end) at = place(u, filled);
                st.load_k(i, at.k, at.n);
                st.un[i].ks = scale_k(at);
                st.load_v(i, at.v, at.n);
                st.un[i].vs = scale_v(at);
                n[i] = u < end ? at.n : 0;
            }
            __builtin_amdgcn_s_waitcnt(0);  // so that the loop's waits need not allow for this path
        }
        u = u < end ? after(u) : u;
#pragma unroll 1
        while (u < end) {
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                floatx4 c[2];
                float f = st.factor(i);
                asm volatile("" : "+v"(f));  // taken here: the scale's register is the next load's
                st.scores(i, c);
                const bool more = u < end;
                if (more) at = place(u, filled);
                in_order();
                st.load_k(i, at.k, at.n);
                st.un[i].ks = scale_k(at);
                in_order();
                st.add(i, c, f, n[i]);
                st.settle();
                in_order();
                st.un[i].vs = scale_v(at);
                st.load_v(i, at.v, at.n);
                n[i] = more ? at.n : 0;
                u = more ? after(u) : u;
            }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            if (n[i] > 0) {
                floatx4 c[2];
                st.scores(i, c);
                st.add(i, c, st.factor(i), n[i]);
            }
        }
    }
    if (p.T_new > 0 && W > 0 && s == p.S - 1) {  // workgroup-uniform
        if (!ready) {
            st.request_q(p, b, kvh);
            cnt.load(p.win_count, b);
            start();
        }
        const int slot0 = cnt.value() % W;
        const size_t src = pair * (size_t)p.T_new * DH, dst = pair * (size_t)W * DH;
        constexpr int shift = DH == 64 ? 2 : DH == 128 ? 3 : 4;
        uint8_t *const codes[2] = {static_cast<uint8_t *>(win_k) + dst, static_cast<uint8_t *>(win_v) + dst};
        float *const scales[2] = {rks, rvs};
        __shared__ uint32_t s_top[2][NW];
#pragma unroll 1
        for (int i = 0; i < tb.count; ++i) {
            if (p.new_bf16)
                append_block<uint16_t, F, NW * kWave>({static_cast<const uint16_t *>(p.new_k) + src,
                                                       static_cast<const uint16_t *>(p.new_v) + src},
                                                      codes, scales, tb.block(i), p.log2_block, shift, W, slot0, filled,
                                                      p.T_new, s_top);
            else
                append_block<float, F, NW * kWave>({static_cast<const float *>(p.new_k) + src,
                                                    static_cast<const float *>(p.new_v) + src},
                                                   codes, scales, tb.block(i), p.log2_block, shift, W, slot0, filled,
                                                   p.T_new, s_top);
            __syncthreads();  // the block is in memory, for this workgroup's loads too
        }
        const int per = 1 << unit_shift;
        for (int i = wave; i < tb.count * per; i += NW) {
            const int r = tb.block(i >> unit_shift) * per + (i & (per - 1));
            if (r * kUnit8 >= filled) continue;
            at = place(pool_units + r, filled);
            st.load_k(0, at.k, at.n);
            st.load_v(0, at.v, at.n);
            st.un[0].ks = scale_k(at);
            st.un[0].vs = scale_v(at);
            floatx4 c[2];
            st.scores(0, c);
            st.add(0, c, st.factor(0), at.n);
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
    constexpr int kThreads = NW * kWave;
    constexpr bool kKeepNaN = true, kBySplits = true;
    const bool bump = p.T_new > 0 && W > 0;
    unsigned prev = ~0u;  // the sequence counter before this workgroup's arrival (one lane)
#include "decode_finish.hpp"
}

template <class F, int DH, int G>
hipError_t launch3(const Decode8Params &p, hipStream_t stream) {
    const dim3 grid(p.S, p.Hkv, p.B);
    static_assert(std::is_same_v<decltype(&decode8_kernel<4, F, DH, G>), Kernel8>, "Args8 is taken from the kernel's list");
    if (p.S < 1 || p.S > 0xFF || p.T_new < 0 || p.T_new > kFusedRows8 || (p.waves != 4 && p.waves != 8)) return hipErrorInvalidValue;
    const int info = p.S | (p.new_split << 8) | ((p.k_len != nullptr) << 10) | (p.T_new << 16);
#define CMC_LAUNCH(NW_)                                                                                          \
    decode8_kernel<NW_, F, DH, G><<<grid, NW_ * kWave, 0, stream>>>(p.cme_k, p.cme_v, p.win_k, p.win_v, p.k, p.W, \
                                                                    p.N, p.Hkv, p.chunk, info, p)
    if (p.waves == 4) CMC_LAUNCH(4);
    else CMC_LAUNCH(8);
#undef CMC_LAUNCH
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
