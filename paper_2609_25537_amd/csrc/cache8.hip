// Writing the 8-bit cache and reading it back (the format: cache8.hpp).
//
// The Tier-1 gather and the ring append take one workgroup per block of rows,
// for K and V together: half of its threads hold the block's K in registers,
// half its V, so every row is read once; the block's largest magnitude is
// reduced over the half, and the codes go out as 16-byte stores.  All of it is
// bound by memory (a gather of fp32 rows to int8, 229 MB, 43 us; an append of
// 1024 bf16 rows to 64 x 8 rings 72.9 us, 5.5 TB/s), the small calls by latency
// (3.7 us for a gather of 256 rows of one sequence).
#include <algorithm>
#include <type_traits>

#include "cache8.hpp"
#include "kernels.hpp"

namespace cmc {

namespace {

// One block of rows of one (sequence, kv head): the rows of a Tier-1 block,
// read from the pool through the index list, or (RING) a ring block that the
// appended rows touch, its other live rows read back from their codes.  NP:
// 16-element words per thread, for blockDim.x / 2 threads on each of K and V.
template <typename T, class F, bool RING, int NP>
__global__ __launch_bounds__(1024) void write_blocks_kernel(Write8Params p) {
    const int h = blockIdx.y, b = blockIdx.z;
    const size_t head = (size_t)b * p.Hkv + h;
    const int half = (int)(blockDim.x >> 1);  // whole waves
    const bool is_v = (int)threadIdx.x >= half;
    const int t0 = (int)threadIdx.x - (is_v ? half : 0);
    const int shift = p.row_shift, lb = p.log2_block;
    int j = blockIdx.x, slot0 = 0, live;
    if constexpr (RING) {
        const int count = max(p.count[b], 0);
        slot0 = count % p.R;
        TouchedBlocks tb;
        tb.set(slot0, p.T_new, p.R, lb);
        if (j >= tb.count) return;  // uniform
        j = tb.block(j);
        live = (int)min((long long)count + p.T_new, (long long)p.R) - (j << lb);
    } else {
        live = (p.count ? min(max(p.count[b], 0), p.R) : p.R) - (j << lb);
        if (live <= 0) return;  // uniform
    }
    const int s0 = j << lb;
    const int words = min(live, 1 << lb) << shift;
    const T *src = static_cast<const T *>(is_v ? p.src_v : p.src_k) + ((head * p.src_rows) << shift) * 16;
    uint4 *dst = static_cast<uint4 *>(is_v ? p.v : p.k) + ((head * p.R + s0) << shift);
    float *scale_at = (is_v ? p.vs : p.ks) + head * p.blocks + j;
    float old_scale = 0.f;
    if constexpr (RING) old_scale = *scale_at;

    // A word holds elements to be rounded (fresh) or a ring's old codes.
    Raw16<T> raw[NP];
    uint4 code[RING ? NP : 1];
    bool fresh[NP];
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        const int i = t0 + u * half;
        int row = s0 + (i >> shift);
        bool in = i < words;
        raw[u].clear();
        if constexpr (RING) {
            row -= slot0;
            row += row < 0 ? p.R : 0;
            fresh[u] = in && row < p.T_new;
            code[u] = make_uint4(0, 0, 0, 0);
            if (in && !fresh[u]) code[u] = dst[i];
        } else {
            fresh[u] = in;
            if (in && p.idx) row = min(max(p.idx[(size_t)b * p.idx_stride + row], 0), p.src_rows - 1);
        }
        if (fresh[u]) raw[u].load(src + (((size_t)row << shift) + (i & ((1 << shift) - 1))) * 16);
    }
    uint32_t top = 0, old = 0;
#pragma unroll
    for (int u = 0; u < NP; ++u) top = max(top, raw[u].top());
    if constexpr (RING) {
        float t = 0.f;
#pragma unroll
        for (int u = 0; u < NP; ++u) t = fmaxf(t, F::top16(code[u]));
        old = old_mag(t, old_scale);
    }
    __shared__ uint32_t s_top[2][2][8];
    const int wave = t0 >> 6, waves = half >> 6;
    top = wave_umax(max(top, old));
    if ((threadIdx.x & 63) == 0) s_top[0][is_v][wave] = top;
    __syncthreads();
    for (int w = 0; w < waves; ++w) top = max(top, s_top[0][is_v][w]);
    // Infinities or NaN in the block, known to the whole half: the maximum is
    // taken anew without them.
    const bool plain = top < kInfBits;
    if (!plain) {
        top = old;
#pragma unroll
        for (int u = 0; u < NP; ++u) top = max(top, raw[u].finite_top());
        top = wave_umax(top);
        if ((threadIdx.x & 63) == 0) s_top[1][is_v][wave] = top;
    }
    __syncthreads();
    if (!plain) {
        for (int w = 0; w < waves; ++w) top = max(top, s_top[1][is_v][w]);
    }
    const int e = scale_exp<F>(top);
    const float scale = exp_scale(e), inv = exp_inverse(e);
    if (t0 == 0) *scale_at = scale;
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        const int i = t0 + u * half;
        if (fresh[u]) {
            float x[16];
            raw[u].widen(x);
            st16_nt(&dst[i], pack16<F>(x, inv, plain));
        } else if constexpr (RING) {
            if (i < words && scale != old_scale) st16_nt(&dst[i], repack16<F>(code[u], old_scale, inv));
        }
    }
}

// One row appended, of up to 8 kv heads, to blocks of up to 256 words: one
// workgroup per sequence, a wave for K and for V of each head.  A lane looks at
// every 64th word of the block's codes, all of them requested together with the
// new row; they are written again only where the scale moves.
template <typename T, class F>
__global__ __launch_bounds__(1024) void append_row_kernel(Write8Params p) {
    const int b = blockIdx.x, lane = threadIdx.x & 63;
    const int count = max(p.count[b], 0);
    const int slot = count % p.R, shift = p.row_shift;
    const int filled = min(count, p.R - 1) + 1;  // live after the append
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_v = w & 1;
    const size_t head = (size_t)b * p.Hkv + (w >> 1);
    const int j = slot >> p.log2_block, s0 = j << p.log2_block;
    const int words = min(filled - s0, 1 << p.log2_block) << shift;
    const T *src = static_cast<const T *>(is_v ? p.src_v : p.src_k) + (head << shift) * 16;
    uint4 *dst = static_cast<uint4 *>(is_v ? p.v : p.k) + ((head * p.R + s0) << shift);
    float *scale_at = (is_v ? p.vs : p.ks) + head * p.blocks + j;
    const float old_scale = *scale_at;
    const int first = (slot - s0) << shift;  // word of the new row
    const auto is_old = [&](int i) { return i < words && (i >> shift) != slot - s0; };
    Raw16<T> raw;
    raw.clear();
    const bool mine = lane < 1 << shift;
    if (mine) raw.load(src + (size_t)lane * 16);
    uint4 code[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) code[u] = dst[min(lane + u * 64, words - 1)];
    float t_old = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u)
        if (is_old(lane + u * 64)) t_old = fmaxf(t_old, F::top16(code[u]));
    uint32_t top = raw.top();
    const bool plain = top < kInfBits;
    if (!plain) top = raw.finite_top();
    const int e = scale_exp<F>(wave_umax(max(top, old_mag(t_old, old_scale))));
    const float scale = exp_scale(e), inv = exp_inverse(e);
    if (scale != old_scale) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (is_old(lane + u * 64)) dst[lane + u * 64] = repack16<F>(code[u], old_scale, inv);
        if (lane == 0) *scale_at = scale;
    }
    if (mine) {
        float x[16];
        raw.widen(x);
        dst[first + lane] = pack16<F>(x, inv, plain);
    }
    __syncthreads();
    if (threadIdx.x == 0) p.count[b] = count + 1;
}

// Sixteen bytes of values of 8 (bf16) or 4 codes.
template <typename T, class F, typename Codes>
__device__ __forceinline__ uint4 values16(const Codes &c, float scale) {
    uint32_t w[4];
    if constexpr (sizeof(T) == 2) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float f[4];
            F::widen4(q ? c.y : c.x, f);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                w[2 * q + e] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(f[2 * e] * scale), (__bf16)(f[2 * e + 1] * scale)});
        }
    } else {
        float f[4];
        F::widen4(c, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(f[e] * scale);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Rows r < min(count, R) of the cache in the order they were written, oldest
// first: row (first + r) mod R, first = count mod R where the ring has
// wrapped.  A thread makes 16 bytes of K and of V from 8 (bf16) or 4 codes, so
// that every load and store of a wave takes a whole run.  Bound by memory: 64
// sequences x 8 heads x 1000 rows of 128 to bf16 (393 MB) 64.6 us, 6.1 TB/s;
// with 16 codes a thread, whose stores leave gaps for the next one, 96.4 us (to
// fp32 446 against 85).
template <typename T, class F>
__global__ __launch_bounds__(256) void read_kernel(Read8Params p, int group0) {
    constexpr int E = Vec16<T>::N;  // codes a thread takes
    typedef std::conditional_t<E == 8, uint2, uint32_t> Codes;
    const int h = blockIdx.y, b = blockIdx.z;
    const size_t head = (size_t)b * p.Hkv + h;
    const int shift = p.row_shift + (E == 8 ? 1 : 2);  // log2 of the threads to a row
    const int count = p.count ? p.count[b] : p.R;
    const long long i = (long long)(group0 + (int)blockIdx.x) * 256 + threadIdx.x;
    const long long r = i >> shift;
    if (r >= min(count, p.R)) return;
    long long row = r + (count > p.R ? count % p.R : 0);
    row -= row >= p.R ? p.R : 0;
    const size_t from = ((head * p.R + row) << shift) + (i & ((1 << shift) - 1));
    const size_t to = ((head * p.R) << shift) + i;
    const size_t at = head * p.blocks + (row >> p.log2_block);
    const Codes k = static_cast<const Codes *>(p.k)[from], v = static_cast<const Codes *>(p.v)[from];
    const float ks = p.ks[at], vs = p.vs[at];
    st16_nt(static_cast<uint4 *>(p.out_k) + to, values16<T, F>(k, ks));
    st16_nt(static_cast<uint4 *>(p.out_v) + to, values16<T, F>(v, vs));
}

template <typename T, class F, bool RING>
hipError_t launch_blocks(const Write8Params &p, int items, hipStream_t stream) {
    const int words = 1 << (p.log2_block + p.row_shift);  // of a whole block: 128 to 2048
    // Two words a thread, four where the workgroup would pass 1024 threads.  One
    // word a thread: an append of 1024 rows to 64 x 8 rings of 128 in blocks of
    // 32 takes 80.6 us against 72.9, of one row 7.8 against 6.1, a gather of 512
    // rows for them 39.8 against 39.1; four: 73.5, 6.8 and 41.6.
    const int half = std::min(words / 2, 512);
    const dim3 grid(items, p.Hkv, p.B);
    if (words / half == 2) write_blocks_kernel<T, F, RING, 2><<<grid, 2 * half, 0, stream>>>(p);
    else write_blocks_kernel<T, F, RING, 4><<<grid, 2 * half, 0, stream>>>(p);
    return hipGetLastError();
}

// Ring blocks that an append of T rows can touch at most: two that it fills
// in part, those between and a short last block on the way, each by a row.
int touched_most(int T, int blocks, int log2_block) {
    return std::min({T, blocks, ((T - 1) >> log2_block) + 3});
}

// Every workgroup of write_blocks_kernel reads the counts, so a launch of its own
// raises them.  One row of a small block goes by append_row_kernel, which does
// both: for 1 / 8 / 64 / 256 sequences of 8 heads of 128 in a graph 4.1 / 4.7 / 5.3 /
// 6.6 us against 5.1 / 5.2 / 5.8 / 9.1 (the one that lost of those measured: the append
// case of perf/operators.py, 64 sequences, 6.1 against 5.9), called from the host 7.6
// against 10.6 at every size.  Past a word in each of four registers and a wave for every head, rounds add up:
// 8 sequences of 16 heads in blocks of 64 took 11.5 us in two rounds against 5.8.
template <typename T, class F>
hipError_t launch_append(const Write8Params &p, hipStream_t stream) {
    const int most = touched_most(p.T_new, p.blocks, p.log2_block);
    if (p.T_new == 1 && p.Hkv <= 8 && p.log2_block + p.row_shift <= 8) {
        append_row_kernel<T, F><<<p.B, 128 * p.Hkv, 0, stream>>>(p);
        return hipGetLastError();
    }
    if (hipError_t e = launch_blocks<T, F, true>(p, most, stream); e != hipSuccess) return e;
    return launch_window_count(p.count, p.B, p.T_new, stream);
}

template <typename T, class F>
hipError_t launch_read(const Read8Params &p, hipStream_t stream) {
    const long long threads = (long long)p.R << (p.row_shift + (sizeof(T) == 2 ? 1 : 2));
    const int groups = (int)((threads + 255) / 256);  // 2^24 at most
    // A grid holds less than 2^32 threads a dimension, which 2^26 rows of 256 in fp32
    // reach: those take two launches.
    constexpr int kMost = (1 << 24) - 1;
    for (int at = 0; at < groups; at += kMost) {
        read_kernel<T, F><<<dim3(std::min(groups - at, kMost), p.Hkv, p.B), 256, 0, stream>>>(p, at);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_gather8(const Write8Params &p, bool bf16, bool e4m3, hipStream_t stream) {
    if (bf16) return e4m3 ? launch_blocks<uint16_t, CodeE4M3, false>(p, p.blocks, stream)
                          : launch_blocks<uint16_t, CodeI8, false>(p, p.blocks, stream);
    return e4m3 ? launch_blocks<float, CodeE4M3, false>(p, p.blocks, stream)
                : launch_blocks<float, CodeI8, false>(p, p.blocks, stream);
}

hipError_t launch_append8(const Write8Params &p, bool bf16, bool e4m3, hipStream_t stream) {
    if (bf16) return e4m3 ? launch_append<uint16_t, CodeE4M3>(p, stream) : launch_append<uint16_t, CodeI8>(p, stream);
    return e4m3 ? launch_append<float, CodeE4M3>(p, stream) : launch_append<float, CodeI8>(p, stream);
}

hipError_t launch_read8(const Read8Params &p, bool bf16, bool e4m3, hipStream_t stream) {
    if (bf16) return e4m3 ? launch_read<uint16_t, CodeE4M3>(p, stream) : launch_read<uint16_t, CodeI8>(p, stream);
    return e4m3 ? launch_read<float, CodeE4M3>(p, stream) : launch_read<float, CodeI8>(p, stream);
}

}  // namespace cmc
