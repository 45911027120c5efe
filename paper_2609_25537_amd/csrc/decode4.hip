// Two-tier decode attention over the 4-bit cache (format: cache4.hpp): softmax
// attention of one query token over [Tier-1 rows || ring slots], optionally fused
// with the append of this step's rows, in one launch.
//
// Grid (S, Hkv, B), 4 or 8 waves.  A wave takes units of 32 rows and adds
//   x_t = scale log2(e) <q, K_t>     p_t = 2^(x_t - m)
//   l  += sum_t p_t                  acc += sum_t p_t V_t
// with m a running maximum.  Both products run on MFMA (16x16x32, bf16 in, fp32
// sums).  bf16 holds every code times its scale exactly, and the card widens two
// codes with their scale in one instruction, so only q and p have to be split: into
// three bf16 parts of 8 bits each, by cutting, which together are all of fp32's 24.
//
// Scores: A = 16 rows' K, B = q, a lane ends with the scores of one column for 4 + 4
// rows.  Columns are (head, part): column c holds part c / G of head c % G (eight
// heads have room for two parts and take a second MFMA for the third), and rotates
// within the 16 lanes add the parts, from the widest down, so that all columns of a
// head end with the same bits.
// P V: the same lanes hold p in the A layout as it stands (rows = columns before), so
// p crosses no lane.  A code byte holds two dims of one row, and widens to the two k
// slots of a B word: with p in one slot and 0 in the other, a product gives one of
// the two dims.  So rows are (head, dim parity, part), one MFMA takes 16 keys x 32
// dims, and no code moves between bytes.  Lane (c, q4) multiplies Dh / 16 dims of rows 8 q4
// .. 8 q4 + 7, which four lanes exchange from whole 16-byte loads (rows_of_v).
// The same rows against ones give l, from the p that V was multiplied with.
//
// The maximum is moved only when a score passes it by more than 2 (p <= 4), which
// after the first units is rare; that test needs no exchange between lanes.  Maxima
// of 2^22 and more, where fp32 no longer resolves that, move with every unit and have
// their weights' arguments subtracted first.
//
// Fused append: every workgroup requests the appended rows with its first unit; those
// whose part of the ring takes some of them quantise them before their walk, to memory
// and to LDS, and take them from there in the units that hold them: nothing waits for a
// store, and no unit is read twice.
//
// Bound, at 8 kv heads of 128 and 32 heads: full batches by memory between the launch's
// start and end, which take 7 us (64 sequences of 1536 keys, 109 MB, 23.4 to 24 us; of 4608
// keys 59.8, 6.2 TB/s at the slope; 16 x 16 heads of 256 over 3048 keys, 212 MB, 35.5 us, 6.0
// TB/s), few sequences by the chain of one unit's instructions, about 0.65 us for a wave
// alone on its SIMD, and the join of their splits (one sequence of 768 keys 7.4 us, of
// 32808 keys 14.8; 24 ragged sequences of 64 heads 15.3).  Measured and slower: more units
// in flight than two, 12 waves, the next unit's scores between this one's (one workgroup's
// 32768 keys 135 us against 126), K multiplied as codes and scales with q in five parts of 6
// bits (64 sequences 25.7 us against 25.1, with heads of 64 20.1 against 18.0), q split by every
// wave for itself (21 keys of one sequence 5.2 us, 4.2 shared; with heads of 256 7.4 and 5.3).
#include <algorithm>
#include <type_traits>

#include "cache4.hpp"
#include "decode_common.hpp"

namespace cmc {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kMaxSlack = 2.f;  // how far a score may pass a running maximum below 2^22
// Running maxima of 2^22 and more, where fp32 is spaced by a half and more, take the
// weights' argument apart (Walk4::add).
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

// A constant loaded where it is used, on a rare path, instead of kept in a register.
__device__ __forceinline__ float made_here(float c) {
    asm("" : "+v"(c));
    return c;
}

// Keeps loads after this point from being issued before it, and arithmetic on
// the registers they go to from being moved behind it.
__device__ __forceinline__ void in_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A barrier that orders LDS alone: loads and stores to memory stay in flight.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0) only: vmcnt and expcnt at their maxima
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ floatx4 mfma_bf16(const uint4 &a, const uint4 &b, const floatx4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// x's leading 8 bits, as a float.
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// The leading 8 bits of two numbers side by side.
__device__ __forceinline__ uint32_t pair_of(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
}
constexpr uint32_t kNone = 0x0c0c0c0c;  // a permute's selector of zeros

// Units in flight per wave; with eight heads of 256 the registers hold one.
template <int DH, int G>
constexpr int kSets4 = G * DH > 1024 ? 1 : 2;

// The codes and scales of a Tier-1 block's or a ring's rows, bounded by the live ones.
struct Array4 {
    __amdgpu_buffer_rsrc_t k, v, ks, vs;
};
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *at, uint32_t bytes) {
    constexpr int untyped = 0x00027000;  // 32-bit elements, addressed by bytes
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, (int)bytes, untyped);
}

// A word of eight dims of the appended rows for each thread, K's in the first half of the
// workgroup and V's in the second, requested early (fp32 as two loads, bf16 as one and
// one of nothing).
template <int DH, int NT>
struct NewRows {
    static constexpr int kShift = DH == 64 ? 3 : DH == 128 ? 4 : 5;
    uint4 r[2];
    __device__ __forceinline__ static bool is_v() { return threadIdx.x >= NT / 2; }  // whole waves
    __device__ __forceinline__ static int word() { return threadIdx.x & (NT / 2 - 1); }
    __device__ __forceinline__ void request(const Decode4Params &p, int T_new, size_t pair) {
        const int bytes = T_new * DH * (p.new_bf16 ? 2 : 4);
        const char *at = static_cast<const char *>(is_v() ? p.new_v : p.new_k) + pair * (size_t)bytes;
        at = reinterpret_cast<const char *>(uniform(reinterpret_cast<uint64_t>(at)));
        const __amdgpu_buffer_rsrc_t from = buffer_of(at, bytes);
        const int o = word() * (p.new_bf16 ? 16 : 32);
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(from, o, 0, 0);
        const u32x4 y = __builtin_amdgcn_raw_buffer_load_b128(from, p.new_bf16 ? bytes : o + 16, 0, 0);
        r[0] = make_uint4(x[0], x[1], x[2], x[3]);
        r[1] = make_uint4(y[0], y[1], y[2], y[3]);
    }
    __device__ __forceinline__ static uint64_t uniform(uint64_t x) {
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
        return (uint64_t)hi << 32 | lo;
    }
    __device__ __forceinline__ void widen(bool bf16, float (&x)[8]) const {
        float a[4], b[4], c[8];
        Vec16<float>::widen(r[0], a);
        Vec16<float>::widen(r[1], b);
        Vec16<uint16_t>::widen(r[0], c);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = bf16 ? c[e] : e < 4 ? a[e & 3] : b[e & 3];
    }
};

// The appended rows in 4 bits as the ring holds them, [0] K's and [1] V's.
template <int DH>
struct NewCodes {
    uint32_t codes[2][fused_rows4(DH)][DH / 8];
    __attribute__((aligned(16))) uint8_t scales[2][fused_rows4(DH)][DH / 32];
};

// q's parts and the factors of its heads, shared by the workgroup's waves: part p of
// head g, bf16, the last part zeros.  Rows are padded so that a wave's columns lie in
// different banks.
template <int DH, int G>
struct Queries {
    __attribute__((aligned(16))) uint16_t part[4][G][DH + 8];
    float f[G];  // |scale| log2(e) over q's power of two
};

// Exchange between lanes i and i ^ 4 (or i ^ 8) of 16: the lanes with the bit clear keep x
// and take the other's x as y, those with it set keep y and take the other's y as x.  Two of
// these transpose a square of dwords over four lanes.
__device__ __forceinline__ void cross4(uint32_t &x, uint32_t &y) {
    const int a = (int)x, b = (int)y;
    x = (uint32_t)__builtin_amdgcn_update_dpp(a, b, 0x114, 0xF, 0xA, false);  // from lane - 4
    y = (uint32_t)__builtin_amdgcn_update_dpp(b, a, 0x104, 0xF, 0x5, false);  // from lane + 4
}
__device__ __forceinline__ void cross8(uint32_t &x, uint32_t &y) {
    const int a = (int)x, b = (int)y;
    x = (uint32_t)__builtin_amdgcn_update_dpp(a, b, 0x128, 0xF, 0xC, false);
    y = (uint32_t)__builtin_amdgcn_update_dpp(b, a, 0x128, 0xF, 0x3, false);
}
// Of a quad's lane I, to all four.
template <int I>
__device__ __forceinline__ uint32_t of_quad_lane(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, I * 0x55, 0xF, 0xF, true);
}

template <int NW, int DH, int G>
struct Walk4 {
    static constexpr int KW = DH / 32;         // words of a K row per lane, and MFMAs per 16 rows
    static constexpr int VB = DH / 32;         // bytes of a V row per lane (two dims each), and MFMAs per 16 rows
    static constexpr int QP = G == 8 ? 2 : 1;  // MFMAs that q's parts take
    static constexpr int PP = G == 8 ? 3 : G == 4 ? 2 : 1;  // and p's
    static constexpr int NS = kSets4<DH, G>;
    static constexpr int KLoads = DH / 64;     // loads of a unit's K, 16 bytes a lane
    static constexpr int VLoads = DH == 256 ? 4 : 2, VWords = DH == 64 ? 2 : 4;  // and of its V
    // Units on their way or being worked on, each in registers of its own, as loaded.
    struct Unit {
        uint32_t k[KLoads][4], v[VLoads][VWords], ks, vs[DH == 128 ? 8 : DH == 256 ? 4 : 2];
    } un[NS];
    static constexpr int NH = (G + NW - 1) / NW, QE = DH / 64;  // a wave's heads of q, and its lanes' elements of each
    float qx[NH][QE];         // q as loaded
    uint4 q[QP][KW];
    float f;                  // of head r16 % G
    float m;                  // of head r16 % G
    float limit;              // the largest score that m may stay for
    floatx4 l, acc[VB];       // rows 4 q4 + i: (head, dim parity, part)
    int lane, r16, q4;
    int k_turn, v_turn;       // to the lane's scales

    // Where things lie in a unit.  Row x of tile t in both products (its lanes' scores are
    // of rows 4 q4 + i) is row 8 (x / 4) + 4 t + x % 4: a lane group's eight rows follow one
    // another.
    __device__ __forceinline__ int k_row(int t) const { return 8 * (r16 >> 2) + 4 * t + (r16 & 3); }
    __device__ __forceinline__ int v_row(int e) const { return 8 * q4 + e; }  // e = 4 t + i
    // The lane's first dim of q and of a K row, and of a V row.
    __device__ __forceinline__ int k_dim() const { return DH == 64 ? 32 * (q4 & 1) + 16 * (q4 >> 1) : 8 * KW * q4; }
    __device__ __forceinline__ int v_dim() const {
        return DH == 256 ? 32 * (r16 & 7) + 16 * (r16 >> 3) : DH / 4 * (r16 & 3) + DH / 16 * (r16 >> 2);
    }

    __device__ __forceinline__ void init() {
        lane = threadIdx.x & 63;
        r16 = lane & 15;
        q4 = lane >> 4;
        k_turn = turn_for(DH == 64 ? q4 & 1 : DH == 128 ? q4 : 2 * (q4 & 1));
        v_turn = turn_for(DH == 64 ? (r16 & 3) >> 1 : r16 & 3);
        m = kNoMax;
        limit = kNoMax;
        l = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < VB; ++j) acc[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    }

    // Loads.  A unit's rows are at a scalar offset in the buffers of its array, whose bounds
    // are the array's live rows: rows past them come as zeros, and neither a row nor a unit
    // costs address arithmetic per lane.  A load takes the CU's address unit 16 cycles,
    // however little its lanes ask for, and 14 of them a unit (4 bytes of V, the scales of a row
    // each) were what it waited for: so lanes take 16 bytes where they can, of other rows
    // or dims than they need, and exchange them.
    static constexpr int kNonTemporal = 2;
    template <int CACHE = 0>
    __device__ __forceinline__ static void load_words(uint32_t (&to)[4], __amdgpu_buffer_rsrc_t from, int o, int at) {
        const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(from, o, at, CACHE);
        to[0] = x[0];
        to[1] = x[1];
        to[2] = x[2];
        to[3] = x[3];
    }
    template <int CACHE = 0>
    __device__ __forceinline__ static void load_words(uint32_t (&to)[2], __amdgpu_buffer_rsrc_t from, int o, int at) {
        const auto x = __builtin_amdgcn_raw_buffer_load_b64(from, o, at, CACHE);
        to[0] = x[0];
        to[1] = x[1];
    }
    // Heads of 64 as one: half a row for each lane, tile 0's in the lower half of the wave.
    static constexpr int KPer = KLoads == 1 ? 1 : KLoads / 2;  // loads of a tile
    __device__ __forceinline__ int raw_k_row(int j) const { return k_row(DH == 64 ? q4 >> 1 : j / KPer); }
    __device__ __forceinline__ int raw_k_word(int j) const { return DH == 64 ? 4 * (q4 & 1) : KW * q4 + 4 * (j % KPer); }
    __device__ __forceinline__ void load_k(int set, const Array4 &from, int unit) {
        const int at = unit * (kUnit4 * DH / 2), o = raw_k_row(0) * (DH / 2) + 4 * raw_k_word(0);
#pragma unroll
        for (int j = 0; j < KLoads; ++j)
            load_words(un[set].k[j], from.k, o + j / KPer * 4 * (DH / 2) + 16 * (j % KPer), at);
    }
    // Odd lane groups load tile 1's for both.  Scale bytes come with their neighbours (a
    // row's two, or four of them): the compiler clears the other bits of a byte at the end of
    // a loop's turn, for which it waits.
    __device__ __forceinline__ void load_ks(int set, const Array4 &from, int unit) {
        un[set].ks = scales_at(from.ks, k_row(q4 & 1) * (DH / 32) + (DH == 256 ? 4 * (q4 >> 1) : 0), unit * (kUnit4 * DH / 32));
    }
    __device__ __forceinline__ static uint32_t scales_at(__amdgpu_buffer_rsrc_t from, int o, int at) {
        if constexpr (DH == 64) {
            typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
            u16x2 x;  // the other half may hold anything
            x[0] = __builtin_amdgcn_raw_buffer_load_b16(from, o, at, 0);
            return __builtin_bit_cast(uint32_t, x);
        } else {
            return __builtin_amdgcn_raw_buffer_load_b32(from, o, at, 0);
        }
    }
    // A loaded word turned so that byte b is where bf16_pair4 looks for a scale.
    __device__ __forceinline__ static int turn_for(int b) { return (8 * b + 9) & 31; }
    __device__ __forceinline__ static uint32_t turned(uint32_t w, int by) { return __builtin_amdgcn_alignbit(w, w, by); }
    // Four lanes (heads of 256: two, and twice as many loads) hold four (two) rows' chunks of
    // 32 dims (of 64: 16) and want a part of each row's.
    __device__ __forceinline__ int raw_v_row(int j) const { return DH == 256 ? 8 * q4 + 2 * j + (r16 >> 3) : 8 * q4 + 4 * j + (r16 >> 2); }
    __device__ __forceinline__ int raw_v_word() const { return VWords * (r16 & (DH == 256 ? 7 : 3)); }
    __device__ __forceinline__ void load_v(int set, const Array4 &from, int unit) {
        const int o = raw_v_row(0) * (DH / 2) + 4 * raw_v_word(), at = unit * (kUnit4 * DH / 2);
#pragma unroll
        for (int j = 0; j < VLoads; ++j)
            load_words<kNonTemporal>(un[set].v[j], from.v, o + j * (8 / VLoads) * (DH / 2), at);
    }
    // The scales of a lane group's eight rows: of heads of 128 each lane has all of them, else
    // each lane of a quad two rows'.
    __device__ __forceinline__ int raw_vs_row() const { return 8 * q4 + (DH == 128 ? 0 : 2 * (r16 & 3)); }
    __device__ __forceinline__ void load_vs(int set, const Array4 &from, int unit) {
        uint32_t (&to)[DH == 128 ? 8 : DH == 256 ? 4 : 2] = un[set].vs;
        const int o = raw_vs_row() * (DH / 32), at = unit * (kUnit4 * DH / 32);
        if constexpr (DH == 64) {
#pragma unroll
            for (int e = 0; e < 2; ++e) to[e] = scales_at(from.vs, o + e * (DH / 32), at);
        } else {
#pragma unroll
            for (int i = 0; i < (DH == 128 ? 2 : 1); ++i) {
                uint32_t w[4];
                load_words(w, from.vs, o + 16 * i, at);
#pragma unroll
                for (int e = 0; e < 4; ++e) to[4 * i + e] = w[e];
            }
        }
    }

    // A ring unit loaded before it was known which rows it holds: rows that were appended
    // this call from LDS (row `first` of the ring is the unit's first, slot0 the first
    // appended one's), and V's rows from n on, which weigh nothing but may hold NaN, as 0.
    __device__ __forceinline__ void amend(int set, const NewCodes<DH> &fresh, int first, int slot0, int T_new, int W, int n) {
        Unit &x = un[set];
        const auto which = [&](int row) {  // among the appended rows
            const int a = first + row - slot0;
            return a < 0 ? a + W : a;
        };
        const auto codes = [&](auto &to, int kv, int row, int word) {
            const int a = which(row);
            if (a < T_new) {
#pragma unroll
                for (int i = 0; i < (int)(sizeof(to) / 4); ++i) to[i] = fresh.codes[kv][a][word + i];
            }
        };
        const auto scale_word = [&](uint32_t &to, int kv, int row, int at) {
            const int a = which(row);
            if (a < T_new) {
                const uint8_t *from = &fresh.scales[kv][a][at];
                if constexpr (DH == 64) to = *reinterpret_cast<const uint16_t *>(from);
                else to = *reinterpret_cast<const uint32_t *>(from);
            }
        };
#pragma unroll
        for (int j = 0; j < KLoads; ++j) codes(x.k[j], 0, raw_k_row(j), raw_k_word(j));
        scale_word(x.ks, 0, k_row(q4 & 1), DH == 256 ? 4 * (q4 >> 1) : 0);
#pragma unroll
        for (int j = 0; j < VLoads; ++j) codes(x.v[j], 1, raw_v_row(j), raw_v_word());
        constexpr int rows = DH == 128 ? 8 : 2, words = DH == 256 ? 2 : 1;
#pragma unroll
        for (int e = 0; e < rows; ++e)
#pragma unroll
            for (int i = 0; i < words; ++i) {
                uint32_t &to = x.vs[words * e + i];
                scale_word(to, 1, raw_vs_row() + e, 4 * i);
                if (raw_vs_row() + e >= n) to = 0;  // 2^-127 times any code
            }
    }

    // A head of q for each wave (two, where there are eight for four), QE elements a lane.
    __device__ __forceinline__ void request_q(const DecodeParams &p, int b, int kvh, int wave) {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const float *qp = p.q + ((size_t)b * p.Hq + (size_t)kvh * G + min(wave + NW * h, G - 1)) * DH + QE * lane;
            typedef float Run __attribute__((ext_vector_type(QE == 1 ? 2 : QE)));
            if constexpr (QE == 1) {
                qx[h][0] = *qp;
            } else {
                const Run x = *reinterpret_cast<const Run *>(qp);
#pragma unroll
                for (int e = 0; e < QE; ++e) qx[h][e] = x[e];
            }
        }
    }
    // q times a power of two, and its parts.  With 2^sum the size of scale log2(e) q, q
    // is taken to 2^-12, so that a score's sum stays in range for any K, and f makes up
    // for it; past 2^60 and below 2^-100, where it takes tiny or huge K to bring the
    // scores back, q takes a share, so that neither f nor the products are subnormal.
    __device__ __forceinline__ void split_q(const DecodeParams &p, int wave, Queries<DH, G> &to_all) {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const int g = wave + NW * h;
            if (g >= G) break;  // wave-uniform
            float x[QE], top = 0.f;
#pragma unroll
            for (int e = 0; e < QE; ++e) {
                x[e] = qx[h][e];
                top = fmaxf(top, fabsf(x[e]));
            }
            top = lane_reduce<OpMax, 1, 64>(top);
            const int qe = (int)(__float_as_uint(top) >> 23) - 127, se = __builtin_amdgcn_frexp_expf(p.qscale);
            const int sum = qe + se;
            const int to = sum > 60 ? min(sum - 72, 60) : sum < -100 ? max(sum + 88, -72) : -12;
            const float factor = ldexpf(__builtin_amdgcn_frexp_mantf(fabsf(p.qscale)), sum - to);
            const int by = to - qe, most = min(max(by, -126), 127);
            const float mul = ldexpf(copysignf(1.f, p.qscale), most);
            uint32_t y[3][QE];
#pragma unroll
            for (int e = 0; e < QE; ++e) {
                x[e] *= mul;
                if (__builtin_expect(by != most, 0)) x[e] = ldexpf(x[e], by - most);
                const float r = x[e] - cut(x[e]);
                y[0][e] = __float_as_uint(x[e]);
                y[1][e] = __float_as_uint(r);
                y[2][e] = __float_as_uint(r - cut(r));
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                uint16_t *const at = &to_all.part[s][g][QE * lane];
                if constexpr (QE == 1) {
                    *at = s < 3 ? (uint16_t)(y[s % 3][0] >> 16) : (uint16_t)0;
                } else {
#pragma unroll
                    for (int e = 0; e < QE; e += 2)
                        *reinterpret_cast<uint32_t *>(at + e) =
                            s < 3 ? pair_of(__uint_as_float(y[s % 3][e]), __uint_as_float(y[s % 3][e + 1])) : 0u;
                }
            }
            if (lane == 0) to_all.f[g] = factor;
        }
    }
    // The lane's columns: part r16 / G of head r16 % G, the third of eight heads for itself.
    __device__ __forceinline__ void take_q(const Queries<DH, G> &from) {
        const int head = r16 % G, part = r16 / G;
#pragma unroll
        for (int s = 0; s < QP; ++s)
#pragma unroll
            for (int i = 0; i < KW; ++i)
                q[s][i] = *reinterpret_cast<const uint4 *>(&from.part[s ? 2 + part : min(part, 3)][head][k_dim() + 8 * i]);
        f = from.f[head];
    }

    // Scores (over f) of rows 8 q4 + 4 t + i.
    __device__ __forceinline__ void scores(int set, floatx4 (&c)[2]) const {
        const Unit &x = un[set];
        const auto ks = __builtin_amdgcn_permlane16_swap(x.ks, x.ks, false, false);
        uint32_t k[2][KW];
        if constexpr (DH == 64) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const auto w = __builtin_amdgcn_permlane32_swap(x.k[0][i], x.k[0][2 + i], false, false);
                k[0][i] = w[0];
                k[1][i] = w[1];
            }
        } else {
#pragma unroll
            for (int j = 0; j < KLoads; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) k[j / KPer][4 * (j % KPer) + e] = x.k[j][e];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            c[t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                const uint32_t s = turned(ks[t], DH == 256 && i >= KW / 2 ? k_turn + 8 & 31 : k_turn);
                const uint4 w = bf16_word4(k[t][i], s);
#pragma unroll
                for (int j = 0; j < QP; ++j) c[t] = mfma_bf16(w, q[j][i], c[t]);
            }
        }
    }

    // V's codes of tile t: a row's in a word (of heads of 256 two, of 64 a half: rows 2 h and
    // 2 h + 1 in word h).
    __device__ __forceinline__ void rows_of_v(int set, int t, uint32_t (&w)[DH == 256 ? 8 : DH == 128 ? 4 : 2]) const {
        const auto &x = un[set].v;
        if constexpr (DH == 64) {
            uint32_t a = x[t][0], b = x[t][1];
            cross8(a, b);  // the lane's words of rows r, 2 + r, with r the lane's bit 2
            const uint32_t take = r16 & 4 ? 0x03020706u : 0x05040100u;  // the upper halves or the lower
            const auto halves = [&](uint32_t own) {
                int o = __builtin_amdgcn_update_dpp(0, (int)own, 0x114, 0xF, 0xA, false);
                o = __builtin_amdgcn_update_dpp(o, (int)own, 0x104, 0xF, 0x5, false);
                return __builtin_amdgcn_perm((uint32_t)o, own, take);
            };
            w[0] = halves(a);
            w[1] = halves(b);
        } else if constexpr (DH == 128) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = x[t][i];
            cross4(w[0], w[1]);
            cross4(w[2], w[3]);
            cross8(w[0], w[2]);
            cross8(w[1], w[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {  // rows 2 j and 2 j + 1
                uint32_t a[4] = {x[2 * t + j][0], x[2 * t + j][1], x[2 * t + j][2], x[2 * t + j][3]};
                cross8(a[0], a[2]);
                cross8(a[1], a[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[4 * j + e] = a[2 * (e >> 1) + (e & 1)];
            }
        }
    }
    // V's scale of row 8 q4 + E, turned.
    template <int E>
    __device__ __forceinline__ uint32_t scale_of_v(const uint32_t (&two)[2], int set) const {
        if constexpr (DH == 128) return turned(un[set].vs[E], v_turn);
        else return turned(of_quad_lane<(E >> 1)>(two[E & 1]), v_turn);
    }

    // Has the sums finished here rather than behind the next loads, which would
    // keep this unit's registers and put those loads in others, to be moved (and
    // so waited for) at the end of a turn.
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int j = 0; j < VB; ++j) asm volatile("" : "+v"(acc[j]));
        asm volatile("" : "+v"(l));
    }

    // The unit's share of l and acc.  Rows n and up neither count in the maximum nor
    // weigh anything.
    __device__ __forceinline__ void add(int set, const floatx4 (&c)[2], int n) {
        float x[8];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float y = c[t][i];
                y += dpp_sum_operand<0x128>(y);
                if constexpr (G <= 4) y += dpp_sum_operand<0x124>(y);
                if constexpr (G <= 2) y += dpp_sum_operand<0x122>(y);
                if constexpr (G == 1) y += dpp_sum_operand<0x121>(y);
                x[4 * t + i] = y;
            }
        float top = rounded_product(fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                                          fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7]))), f);
        const auto live = [&](int e) { return v_row(e) < n; };
        if (__builtin_expect(n < kUnit4, 0)) {
            top = made_here(kNoMax);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = live(e) ? fmaxf(top, rounded_product(x[e], f)) : top;
        }
        float mp = m, by = f;
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
                    for (int j = 0; j < VB; ++j) acc[j][i] *= al[i];
                }
            }
            mp = far ? 0.f : m;
            // Below 2^22 the argument x f - m is off by half the spacing of x f at most.
            // Above, the exact product may lie far from the rounded one that m is.
            if (__builtin_expect(__any(far), 0)) {
                by = far ? 1.f : f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = far ? product_less(x[e], f, m) : x[e];
            }
        }
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = fast_exp2(fmaf(x[e], by, -mp));
        if (__builtin_expect(n < kUnit4, 0)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = live(e) ? w[e] : 0.f;
        }
        // p's parts: the top of what the leading ones leave, in the half of the word that the
        // row's dim parity has, or nothing.
        const int part = r16 / (2 * G);
        const uint32_t half = (r16 / G) & 1 ? 0x03020c0cu : 0x0c0c0302u;
        const uint32_t take = part < 3 ? half : kNone, take_lo = part == 1 ? half : kNone;
        const float less1 = part >= 1 ? 1.f : 0.f, less2 = part >= 2 ? 1.f : 0.f;
        const auto slot = [](float y, uint32_t take) { return __builtin_amdgcn_perm(0u, __float_as_uint(y), take); };
        uint32_t P[PP][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (G == 8) {
                const float r = w[e] - cut(w[e]);
                P[0][e] = slot(w[e], half);
                P[1][e] = slot(r, half);
                P[2][e] = slot(r - cut(r), half);
            } else if constexpr (G == 4) {  // the second part's rows take the third too
                const float r = fmaf(-less1, cut(w[e]), w[e]);
                P[0][e] = slot(r, half);
                P[1][e] = slot(r - cut(r), take_lo);
            } else {
                const float r = fmaf(-less1, cut(w[e]), w[e]);
                P[0][e] = slot(fmaf(-less2, cut(r), r), take);
            }
        }
        constexpr uint32_t one = 0x3f803f80u;
        const uint4 ones = make_uint4(one, one, one, one);
        uint32_t two[2] = {};  // the scales of rows 2 (r16 % 4) and the next, of the lane's dims
        if constexpr (DH == 64) {
            two[0] = un[set].vs[0];
            two[1] = un[set].vs[1];
        } else if constexpr (DH == 256) {
            const uint32_t w0 = un[set].vs[0], w1 = un[set].vs[1], w2 = un[set].vs[2], w3 = un[set].vs[3];
            two[0] = r16 & 4 ? w1 : w0;
            two[1] = r16 & 4 ? w3 : w2;
        }
        const auto tile = [&](auto which) {
            constexpr int t = decltype(which)::value;
            const uint32_t s[4] = {scale_of_v<4 * t>(two, set), scale_of_v<4 * t + 1>(two, set), scale_of_v<4 * t + 2>(two, set),
                                   scale_of_v<4 * t + 3>(two, set)};
            uint32_t v[DH == 256 ? 8 : DH == 128 ? 4 : 2];
            rows_of_v(set, t, v);
#pragma unroll
            for (int h = 0; h < PP; ++h) {
                const uint4 p = make_uint4(P[h][4 * t], P[h][4 * t + 1], P[h][4 * t + 2], P[h][4 * t + 3]);
                l = mfma_bf16(p, ones, l);
            }
            const auto product = [&](auto byte) {
                constexpr int J = decltype(byte)::value;
                uint4 y;
                if constexpr (DH == 64)
                    y = make_uint4(bf16_pair4<J>(v[0], s[0]), bf16_pair4<2 + J>(v[0], s[1]), bf16_pair4<J>(v[1], s[2]),
                                   bf16_pair4<2 + J>(v[1], s[3]));
                else if constexpr (DH == 128)
                    y = make_uint4(bf16_pair4<J>(v[0], s[0]), bf16_pair4<J>(v[1], s[1]), bf16_pair4<J>(v[2], s[2]),
                                   bf16_pair4<J>(v[3], s[3]));
                else
                    y = make_uint4(bf16_pair4<J & 3>(v[J >> 2], s[0]), bf16_pair4<J & 3>(v[2 + (J >> 2)], s[1]),
                                   bf16_pair4<J & 3>(v[4 + (J >> 2)], s[2]), bf16_pair4<J & 3>(v[6 + (J >> 2)], s[3]));
#pragma unroll
                for (int h = 0; h < PP; ++h) {
                    const uint4 p = make_uint4(P[h][4 * t], P[h][4 * t + 1], P[h][4 * t + 2], P[h][4 * t + 3]);
                    acc[J] = mfma_bf16(p, y, acc[J]);
                }
            };
            product(std::integral_constant<int, 0>{});
            product(std::integral_constant<int, 1>{});
            if constexpr (VB >= 4) {
                product(std::integral_constant<int, 2>{});
                product(std::integral_constant<int, 3>{});
            }
            if constexpr (VB == 8) {
                product(std::integral_constant<int, 4>{});
                product(std::integral_constant<int, 5>{});
                product(std::integral_constant<int, 6>{});
                product(std::integral_constant<int, 7>{});
            }
        };
        tile(std::integral_constant<int, 0>{});
        tile(std::integral_constant<int, 1>{});
    }

    // A row-tile value (rows 4 q4 + i) summed over the parts: put(g, parity, value)
    // on the lanes that hold one.
    template <class Put>
    __device__ __forceinline__ void over_parts(const floatx4 &a, Put &&put) const {
        if constexpr (G == 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) put(4 * (q4 & 1) + i, q4 >> 1, a[i]);
        } else if constexpr (G == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float t = combine_xor32<OpSum>(a[i]);
                if (q4 < 2) put(i, q4, t);
            }
        } else if constexpr (G == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float t = combine_xor32<OpSum>(combine_xor16<OpSum>(a[i]));
                if (q4 == 0) put(i & 1, i >> 1, t);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float t = combine_xor32<OpSum>(combine_xor16<OpSum>(a[i] + a[i + 2]));
                if (q4 == 0) put(0, i, t);
            }
        }
    }
};

// Two dims of head g over the waves' (m, l, acc); returns the joint maximum.  Without a
// key in any wave (m = kNoMax) the weights are 1 against zeros.
template <int NW, int DH, int G>
__device__ __forceinline__ float joined(const float (&sm)[NW][G], const float (&sl)[NW][G], const float (&sa)[NW][G][DH],
                                        int g, int d, float2 &num, float &den) {
    float mw[NW], lw[NW];
    float2 aw[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        mw[w] = sm[w][g];
        lw[w] = sl[w][g];
        aw[w] = *reinterpret_cast<const float2 *>(&sa[w][g][d]);
    }
    float M = mw[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, mw[w]);
    num = make_float2(0.f, 0.f);
    den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float f = fast_exp2(mw[w] - M);
        num.x = fmaf(f, aw[w].x, num.x);
        num.y = fmaf(f, aw[w].y, num.y);
        den = fmaf(f, lw[w], den);
    }
    return M;
}

// The partials of a pair's S splits into the waves' (m, l, acc), as if each wave had
// walked every NW-th split's rows (with fewer than 256 sums a split, groups of its lanes
// every NW-th or so): each split is read by one wave, 16 bytes a lane, all of them
// requested at once for up to 8 NW splits.  Loads are coherent across the XCDs, and
// bounded: splits past the last come as zeros, with kNoMax for m.  Against each thread
// reading two dims of every split: 8 pairs in 29 splits of four heads of 128 15.3 -> 15.1
// us, one of eight heads in 33 15.7 -> 14.7, one of two pairs of a head of 64 in 59 14.6 -> 11.7;
// 8 pairs in 6 splits 7.4 both.
template <int NW, int DH, int G, int MOST, class Arrive>
__device__ __forceinline__ void merge_splits(const float *part_ml, const float *part_acc, int S, int wave, int lane,
                                             float (&s_m)[NW][G], float (&s_l)[NW][G], float (&s_acc)[NW][G][DH], Arrive arrive) {
    constexpr int kWords = G * DH / 4;                        // of 16 bytes, a split's sums
    constexpr int L = kWords < 64 ? kWords : 64, NG = 64 / L;  // lanes to a split, splits at a time
    constexpr int NV = kWords / L;                            // words a lane
    constexpr int NJ = std::min(MOST, NV >= 8 ? 2 : NV >= 4 ? 4 : 8);  // turns requested at a time
    constexpr int kCoherent = 16;                             // sc1
    const __amdgpu_buffer_rsrc_t ml = buffer_of(part_ml, S * G * 8), ac = buffer_of(part_acc, S * G * DH * 4);
    const int turns = (S + NW * NG - 1) / (NW * NG), group = lane / L;
    // The wave's i-th split is wave + NW i; in turn j a group takes i = group + NG j.
    float *const own = &s_acc[wave][0][0];  // (m, l) of its splits: 2 G turns NG <= G DH floats
    const int mls = turns * NG * G;
    const auto ml_at = [&](int x) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b64(ml, ((wave + NW * (x / G)) * G + x % G) * 8, 0, kCoherent);
        return make_uint2(v[0], v[1]);
    };
    const auto keep = [&](int x, const uint2 &v) {
        const bool in = wave + NW * (x / G) < S;
        *reinterpret_cast<float2 *>(own + 2 * x) = make_float2(in ? __uint_as_float(v.x) : kNoMax, in ? __uint_as_float(v.y) : 0.f);
    };
    const uint2 first = ml_at(lane);
    u32x4 a[NJ][NV];
    const auto request = [&](int j0) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int v = 0; v < NV; ++v)
                a[j][v] = __builtin_amdgcn_raw_buffer_load_b128(
                    ac, (wave + NW * (group + NG * (j0 + j))) * (G * DH * 4) + 16 * (lane % L + L * v), 0, kCoherent);
    };
    in_order();  // (m, l) first: the weights need only them
    request(0);
    in_order();
    if (lane < mls) keep(lane, first);
    for (int x = lane + 64; x < mls; x += 64) keep(x, ml_at(x));
    arrive();
    int g[NV];
    float M[NV], den[NV], sum[NV][4];
    float2 x[NV][NJ];
    const auto take = [&](int v, int j0) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)  // past the last turn that one again
            x[v][j] = *reinterpret_cast<const float2 *>(own + 2 * ((group + NG * min(j0 + j, turns - 1)) * G + g[v]));
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        g[v] = 4 * (lane % L + L * v) / DH;
        take(v, 0);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        M[v] = kNoMax;
#pragma unroll
        for (int j = 0; j < NJ; ++j) M[v] = fmaxf(M[v], x[v][j].x);
        for (int j = NJ; j < turns; ++j) M[v] = fmaxf(M[v], own[2 * ((group + NG * j) * G + g[v])]);
        if constexpr (L <= 16) M[v] = combine_xor16<OpMax>(M[v]);
        if constexpr (L <= 32) M[v] = combine_xor32<OpMax>(M[v]);
        den[v] = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[v][e] = 0.f;
    }
    for (int j0 = 0;;) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            if (j0 + j < turns) {  // wave-uniform
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    const float f = fast_exp2(x[v][j].x - M[v]);
                    den[v] = fmaf(f, x[v][j].y, den[v]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[v][e] = fmaf(f, __uint_as_float(a[j][v][e]), sum[v][e]);
                }
            }
        }
        j0 += NJ;
        if (j0 >= turns) break;
        request(j0);
#pragma unroll
        for (int v = 0; v < NV; ++v) take(v, j0);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const auto over_groups = [&](float x) {
            if constexpr (L <= 16) x = combine_xor16<OpSum>(x);
            if constexpr (L <= 32) x = combine_xor32<OpSum>(x);
            return x;
        };
        den[v] = over_groups(den[v]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[v][e] = over_groups(sum[v][e]);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int at = 4 * (lane % L + L * v);
        if (group == 0) {
            *reinterpret_cast<float4 *>(own + at) = make_float4(sum[v][0], sum[v][1], sum[v][2], sum[v][3]);
            if (at % DH == 0) {
                s_m[wave][g[v]] = M[v];
                s_l[wave][g[v]] = den[v];
            }
        }
    }
}

template <int DH, int G>
constexpr int kMinWaves4 = 2;

// decode4_kernel's parameter list as it lies in the kernarg segment: each where its
// alignment puts it, as in a struct.
struct Args4 {
    const void *cme_k, *cme_v;
    void *win_k, *win_v;
    int k, W, N, Hkv, chunk, info;
    Decode4Params p;
};
typedef void (*Kernel4)(const void *, const void *, void *, void *, int, int, int, int, int, int, Decode4Params);
static_assert(sizeof(Args4) == 4 * sizeof(void *) + 6 * sizeof(int) + sizeof(Decode4Params) &&
                  std::is_trivially_copyable_v<Decode4Params>,
              "Args4 holds Kernel4's parameters, in its order and without gaps");

// The last parameter, loaded here and not before (the compiler would load it at
// the kernel's start and wait for it there); fields that nothing uses are not.
__device__ __forceinline__ Decode4Params late_params() {
    typedef const __attribute__((address_space(4))) Args4 *Ptr;
    Ptr at = (Ptr)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    Decode4Params p;
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
    p.waves = at->p.waves;
    return p;
}

// The ring units that an append of T_new rows at slot0 writes: consecutive from
// first, round the ring's nu units.
struct TouchedUnits {
    int first, count, nu;
    __device__ __forceinline__ void set(int slot0, int T_new, int W) {
        nu = (int)(((unsigned)W + kUnit4 - 1u) / kUnit4);
        first = slot0 / kUnit4;
        const int room = W - slot0;  // slots up to the ring's end
        if (T_new <= room) count = (slot0 + T_new - 1) / kUnit4 - first + 1;
        else count = min(nu, nu - first + (T_new - room - 1) / kUnit4 + 1);
    }
    __device__ __forceinline__ int unit(int i) const { return first + i < nu ? first + i : first + i - nu; }
    __device__ __forceinline__ bool has(int j) const {
        const int d = j - first;
        return (d < 0 ? d + nu : d) < count;
    }
};

// The leading arguments (Args4's, one by one) arrive in SGPRs at wave launch,
// as decode_kernel's do.
template <int NW, int DH, int G>
__global__ __launch_bounds__(NW * kWave, (kMinWaves4<DH, G>)) void decode4_kernel(const void *cme_k, const void *cme_v,
                                                                                  void *win_k, void *win_v, int k,
                                                                                  int W, int N, int Hkv, int chunk,
                                                                                  int info, Decode4Params pm) {
    const int S = info & 0xFF;
    const int s = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int kb = k;
    if ((info >> 10) & 1) {  // k_len is given
        const int v = pm.k_len[b];
        kb = v < 0 ? 0 : (v > k ? k : v);
    }
    // Units: the pool's, then the ring's in physical slot order.
    const int pool_units = (kb + kUnit4 - 1) / kUnit4;
    const int units = pool_units + (int)(((unsigned)W + kUnit4 - 1) / kUnit4);
    int u = s * chunk, end = s == S - 1 ? units : min(u + chunk, units);
    const int from = u;

    const size_t pair = (size_t)b * Hkv + kvh;
    const uint8_t *pk = static_cast<const uint8_t *>(cme_k) + pair * (size_t)N * (DH / 2);
    const uint8_t *pv = static_cast<const uint8_t *>(cme_v) + pair * (size_t)N * (DH / 2);
    uint8_t *rk = static_cast<uint8_t *>(win_k) + pair * (size_t)W * (DH / 2);
    uint8_t *rv = static_cast<uint8_t *>(win_v) + pair * (size_t)W * (DH / 2);
    // Wave w takes units w, w + NW, ...: unit u is number u - first of its array `a`, of
    // `rows` live rows.  The first unit's codes are requested from the leading arguments
    // alone, with all of the ring's slots as live: nothing waits for the others, nor for
    // the count.
    Walk4<NW, DH, G> st;
    st.init();
    u += wave;
    bool ring = u >= pool_units;
    int first = ring ? pool_units : 0, rows = ring ? W : kb;
    Array4 a;
    const auto codes = [&](int rows) {
        a.k = buffer_of(ring ? rk : pk, (uint32_t)rows * (DH / 2));  // 2^31 at most
        a.v = buffer_of(ring ? rv : pv, (uint32_t)rows * (DH / 2));
    };
    codes(u < end ? rows : 0);
    int at = u < end ? u - first : 0;  // in range, or at the start of an empty buffer
    st.load_k(0, a, at);
    st.load_v(0, a, at);
    in_order();
    const int T_new = (int)((unsigned)info >> 16);
    const Decode4Params early = late_params();
    const uint8_t *pks = early.cme_ks + pair * (size_t)N * (DH / 32), *pvs = early.cme_vs + pair * (size_t)N * (DH / 32);
    uint8_t *rks = early.win_ks + pair * (size_t)W * (DH / 32), *rvs = early.win_vs + pair * (size_t)W * (DH / 32);
    const auto scales = [&](int rows) {
        a.ks = buffer_of(ring ? rks : pks, (uint32_t)rows * (DH / 32));
        a.vs = buffer_of(ring ? rvs : pvs, (uint32_t)rows * (DH / 32));
    };

    // The units in turn through NS register sets.  Loads are requested always, of no
    // rows where there is nothing to load: branches around them would have the waits
    // count for the path without them.  In the loop each set's next unit is requested as
    // soon as its registers are free; where there is none left, the last unit again, of
    // which no row counts.  The last NS units are worked off after the loop.
    constexpr int NS = kSets4<DH, G>;
    int n[NS], mine[NS];  // a set's live rows, its unit
    RingCount cnt{0, false};
    NewRows<DH, NW * kWave> fresh;
    scales(u < end ? rows : 0);
    st.load_ks(0, a, at);
    st.load_vs(0, a, at);
    fresh.request(early, T_new, pair);
    in_order();  // before q, whose wait so covers the scales' and the new rows' too
    st.request_q(early, b, kvh, wave);
    cnt.load(W > 0 ? early.win_count : nullptr, b);
    n[0] = u < end ? min(kUnit4, rows - at * kUnit4) : 0;
    mine[0] = u;
#pragma unroll
    for (int i = 1; i < NS; ++i) {
        u += NW;
        ring = u >= pool_units;
        first = ring ? pool_units : 0;
        rows = ring ? W : kb;
        codes(u < end ? rows : 0);
        scales(u < end ? rows : 0);
        at = u < end ? u - first : 0;
        n[i] = u < end ? min(kUnit4, rows - at * kUnit4) : 0;
        mine[i] = u;
        in_order();
        st.load_k(i, a, at);
        st.load_ks(i, a, at);
        in_order();
        st.load_v(i, a, at);
        st.load_vs(i, a, at);
    }
    __shared__ Queries<DH, G> s_q;
    st.split_q(early, wave, s_q);
    // What follows from the count: the ring slots that hold a key of this step, and the
    // units that take appended rows.
    const int count = cnt.value();
    const int filled = (int)min((long long)count + T_new, (long long)W);
    end = min(end, pool_units + (filled + kUnit4 - 1) / kUnit4);
    const bool appends = T_new > 0 && W > 0;
    const int slot0 = appends ? count % W : 0;
    TouchedUnits tu{0, 0, 1};
    if (appends) tu.set(slot0, T_new, W);
    const auto touched = [&](int u) { return u >= pool_units && tu.has(u - pool_units); };
    bool amends[NS];
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        const int live = mine[i] < pool_units ? n[i] : mine[i] < end ? min(kUnit4, filled - (mine[i] - pool_units) * kUnit4) : 0;
        amends[i] = touched(mine[i]) || live != n[i];
        n[i] = live;
    }
    // The appended rows that fall into this workgroup's units, to memory and to LDS.
    __shared__ NewCodes<DH> s_new;
    bool some_here = false;
    const auto here = [&](int ring_unit) { return pool_units + ring_unit >= from && pool_units + ring_unit < end; };
    for (int i = 0; i < tu.count; ++i) some_here |= here(tu.unit(i));
    if (some_here) {  // workgroup-uniform
        const int i = fresh.word(), row = i >> fresh.kShift, word = i & ((1 << fresh.kShift) - 1);
        float x[8];
        fresh.widen(early.new_bf16, x);
        uint32_t byte;
        const uint32_t w = quantise4(x, byte);
        const int slot = slot0 + row < W ? slot0 + row : slot0 + row - W;
        if (row < T_new && here(slot / kUnit4)) {
            const bool v = fresh.is_v();
            Row4{v ? rv : rk, v ? rvs : rks}.store(slot, word, fresh.kShift, w, byte);
            s_new.codes[v][row][word] = w;
            if ((word & 3) == 0) s_new.scales[v][row][word >> 2] = (uint8_t)byte;
        }
    }
    lds_barrier();
    st.take_q(s_q);
    const auto amend = [&](int i) {
        if (__builtin_expect(amends[i], 0))
            st.amend(i, s_new, (mine[i] - pool_units) * kUnit4, slot0, T_new, W, n[i]);
    };
    u += NW;
    const auto enter = [&](bool in_ring) {
        ring = in_ring;
        first = ring ? pool_units : 0;
        rows = ring ? filled : kb;
        codes(rows);
        scales(rows);
    };
    if (u < end) enter(u >= pool_units);
    at = u - first;
    int left = 0;
#pragma unroll 1
    while (u < end) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            floatx4 c[2];
            amend(i);
            st.scores(i, c);
            const bool more = u < end;
            if (more) {
                if (__builtin_expect(!ring && u >= pool_units, 0)) enter(true);
                at = u - first;
            }
            left = more ? rows - at * kUnit4 : 0;
            in_order();
            st.load_k(i, a, at);
            st.load_ks(i, a, at);
            in_order();
            st.add(i, c, n[i]);
            st.settle();
            in_order();
            st.load_v(i, a, at);
            st.load_vs(i, a, at);
            n[i] = min(kUnit4, left);
            mine[i] = u;
            amends[i] = more && touched(u);
            u += NW;
        }
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        if (n[i] > 0) {
            floatx4 c[2];
            amend(i);
            st.scores(i, c);
            st.add(i, c, n[i]);
        }
    }
    // The rest of the arguments, which so take no registers during the walk.
    Decode4Params p = late_params();
    p.k = k;
    p.W = W;
    p.N = N;
    p.Hkv = Hkv;
    p.S = S;
    p.T_new = T_new;

    __shared__ __attribute__((aligned(16))) float s_acc[NW][G][DH];
    __shared__ float s_m[NW][G], s_l[NW][G];
    __shared__ int s_cnt[NW];
#pragma unroll
    for (int j = 0; j < DH / 32; ++j)
        st.over_parts(st.acc[j], [&](int g, int odd, float x) { s_acc[wave][g][st.v_dim() + 2 * j + odd] = x; });
    st.over_parts(st.l, [&](int g, int odd, float x) {
        if (st.r16 == 0 && odd == 0) s_l[wave][g] = x;
    });
    if (st.lane < G) s_m[wave][st.lane] = st.m;
    if (st.lane == 0) s_cnt[wave] = cnt.raw;  // stored once the wave's count read has returned
    __syncthreads();
    constexpr int kThreads = NW * kWave;
    const bool bump = p.T_new > 0 && W > 0;
    unsigned prev = ~0u;  // the sequence counter before this pair's arrival (one lane)
    // A pair arrives for its sequence once all of its waves have read the count: each stored
    // what it read before the barrier above.
    const auto arrive = [&] {
        if (bump && threadIdx.x == 0) prev = arrive_once(p.seq_counter, b, (unsigned)(s_cnt[NW - 1] != INT_MIN));
    };
    float *const outp = p.out + ((size_t)b * p.Hq + (size_t)kvh * G) * DH;
    const auto output = [&] {
        for (int t = threadIdx.x; t < G * DH / 2; t += kThreads) {
            float2 num;
            float den;
            joined<NW, DH, G>(s_m, s_l, s_acc, 2 * t / DH, 2 * t % DH, num, den);
            const float inv = den == 0.f ? 0.f : __builtin_amdgcn_rcpf(den);  // a NaN stays one
            *reinterpret_cast<float2 *>(outp + 2 * t) = make_float2(num.x * inv, num.y * inv);
        }
    };
    if (S == 1) {
        arrive();
        output();
    } else {
        // Publication: the split's partial by coherent stores, which have completed when it
        // arrives on the pair's counter; the last one to arrive merges them all.
        __shared__ int s_last;
        const size_t part = (pair * S + s) * G;
        for (int t = threadIdx.x; t < G * DH / 2; t += kThreads) {
            const int g = 2 * t / DH, d = 2 * t % DH;
            float2 num;
            float den;
            const float M = joined<NW, DH, G>(s_m, s_l, s_acc, g, d, num, den);
            coherent_store2(&p.part_acc[part * DH + 2 * t], num.x, num.y);
            if (d == 0) coherent_store2(&p.part_ml[(part + g) * 2], M, den);
        }
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (threadIdx.x == 0)
            s_last = __hip_atomic_fetch_add(&p.pair_counter[pair], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(S - 1);
        __syncthreads();
        if (!s_last) return;  // workgroup-uniform
        const auto merge = [&](auto most) {
            merge_splits<NW, DH, G, decltype(most)::value>(p.part_ml + pair * S * G * 2, p.part_acc + pair * S * G * DH, S, wave,
                                                           st.lane, s_m, s_l, s_acc, arrive);
        };
        if (S <= 2 * NW) merge(std::integral_constant<int, 2>{});
        else merge(std::integral_constant<int, 8>{});
        lds_barrier();
        output();
        if (threadIdx.x == 0) __hip_atomic_store(&p.pair_counter[pair], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    if (bump && prev == (unsigned)(p.Hkv - 1)) {  // one lane of the sequence's last pair
        p.win_count[b] = count + p.T_new;
        __hip_atomic_store(&p.seq_counter[b], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

template <int DH, int G>
hipError_t launch2(const Decode4Params &p, hipStream_t stream) {
    const dim3 grid(p.S, p.Hkv, p.B);
    static_assert(std::is_same_v<decltype(&decode4_kernel<4, DH, G>), Kernel4>, "Args4 is taken from the kernel's list");
    if (p.S < 1 || p.S > 0xFF || p.T_new < 0 || p.T_new > fused_rows4(DH) || (p.waves != 4 && p.waves != 8)) return hipErrorInvalidValue;
    const int info = p.S | ((p.k_len != nullptr) << 10) | (p.T_new << 16);
#define CMC_LAUNCH(NW_)                                                                                      \
    decode4_kernel<NW_, DH, G><<<grid, NW_ * kWave, 0, stream>>>(p.cme_k, p.cme_v, p.win_k, p.win_v, p.k, p.W, \
                                                                 p.N, p.Hkv, p.chunk, info, p)
    if (p.waves == 4) CMC_LAUNCH(4);
    else CMC_LAUNCH(8);
#undef CMC_LAUNCH
    return hipGetLastError();
}

template <int DH>
hipError_t launch_g(const Decode4Params &p, int G, hipStream_t stream) {
    switch (G) {
        case 1: return launch2<DH, 1>(p, stream);
        case 2: return launch2<DH, 2>(p, stream);
        case 4: return launch2<DH, 4>(p, stream);
        case 8: return launch2<DH, 8>(p, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_decode4(const Decode4Params &p, int G, int Dh, hipStream_t stream) {
    if (p.B == 0) return hipSuccess;
    switch (Dh) {
        case 64: return launch_g<64>(p, G, stream);
        case 128: return launch_g<128>(p, G, stream);
        case 256: return launch_g<256>(p, G, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace cmc
