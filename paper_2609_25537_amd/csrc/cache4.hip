// Writing the 4-bit cache and reading it back (the format: cache4.hpp).
//
// Rows are independent, so a thread takes eight dims of a K row and the same of
// its V row, 16-byte loads of bf16; four neighbouring lanes hold the 32 dims of a
// scale and find their maximum with two lane exchanges.
//
// Bound by memory: a gather of 350 of 4096 fp32 rows for each of 64 x 8 heads, 207 MB,
// 44.3 us, 4.7 TB/s (the same rows side by side 5.1); reading these back as bf16, 117 MB,
// 18.4 us.  Small calls are bound by latency: 2.3 us for a gather of 256 rows of one
// sequence, 2.9 for an append of a row to 64 x 8 rings, 2.1 for 256 rows read back.
#include <algorithm>

#include "cache4.hpp"
#include "kernels.hpp"

namespace cmc {

namespace {

// Words of each array that a thread requests at once, and whether past the caches.  A
// gather waits for an index first and is quickest with many threads: 256 rows of one
// sequence 2.3 us (two words 2.8, four 3.7), 64 sequences 44.3 (45.4, 46.5), not faster past the
// caches (45.2).  An append of 1024 rows to 8 x 8 rings 11.9 us (one word 12.4, through the
// caches 12.7).
template <bool RING>
constexpr int kWriteTrip = RING ? 2 : 1;

// Rows of one (sequence, kv head): a Tier-1 block's, from the pool through the
// index list, or (RING) the appended ones, to their ring slots.
template <typename T, bool RING>
__global__ __launch_bounds__(256) void write_rows4_kernel(Write4Params p) {
    const int h = blockIdx.y, b = blockIdx.z;
    const size_t head = (size_t)b * p.Hkv + h;
    const int shift = p.row_shift;
    int rows, slot0 = 0;
    if constexpr (RING) {
        rows = p.T_new;
        slot0 = max(p.count[b], 0) % p.R;
    } else {
        rows = p.count ? min(max(p.count[b], 0), p.R) : p.R;
    }
    const uint32_t words = (uint32_t)rows << shift;
    const uint32_t i0 = blockIdx.x * (256u * kWriteTrip<RING>) + threadIdx.x;
    if (i0 - threadIdx.x >= words) return;  // uniform
    const T *src[2] = {static_cast<const T *>(p.src_k) + ((head * p.src_rows) << shift) * 8,
                       static_cast<const T *>(p.src_v) + ((head * p.src_rows) << shift) * 8};
    const Row4 dst[2] = {{p.k + ((head * p.R) << shift) * 4, p.ks + ((head * p.R) << (shift - 2))},
                         {p.v + ((head * p.R) << shift) * 4, p.vs + ((head * p.R) << (shift - 2))}};
    Raw8<T> raw[kWriteTrip<RING>][2];
    uint32_t row[kWriteTrip<RING>];
    int word[kWriteTrip<RING>];
#pragma unroll
    for (int u = 0; u < kWriteTrip<RING>; ++u) {
        const uint32_t i = min(i0 + u * 256u, words - 1);  // a row is whole quads, so quads stay together
        row[u] = i >> shift;
        word[u] = (int)(i & ((1u << shift) - 1));
        size_t from = row[u];
        if constexpr (!RING) {
            if (p.idx) from = (size_t)min(max(p.idx[(size_t)b * p.idx_stride + row[u]], 0), p.src_rows - 1);
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) raw[u][x].template load<RING>(src[x] + ((from << shift) + word[u]) * 8);
    }
#pragma unroll
    for (int u = 0; u < kWriteTrip<RING>; ++u) {
        size_t to = row[u];
        if constexpr (RING) {
            to += slot0;
            to -= to >= (size_t)p.R ? p.R : 0;
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) dst[x].put(to, word[u], shift, raw[u][x], i0 + u * 256u < words);
    }
}

// A few appended rows: one workgroup per sequence, which raises the count too.
template <typename T>
__global__ __launch_bounds__(1024) void append_rows4_kernel(Write4Params p) {
    const int b = blockIdx.x, shift = p.row_shift;
    const int count = max(p.count[b], 0);
    const int slot0 = count % p.R;
    const size_t head0 = (size_t)b * p.Hkv;
    const int words = (p.Hkv * p.T_new) << shift;
    for (int i = threadIdx.x; i < words; i += blockDim.x) {  // whole quads: words and blockDim.x are multiples of 4
        const int n = i >> shift, word = i & ((1 << shift) - 1);
        const int h = n / p.T_new, t = n - h * p.T_new;
        const size_t at = (head0 + h) * p.R;
        const size_t from = (((head0 << shift) * p.T_new) + i) * 8;
        Raw8<T> k, v;
        k.template load<false>(static_cast<const T *>(p.src_k) + from);
        v.template load<false>(static_cast<const T *>(p.src_v) + from);
        const int slot = slot0 + t < p.R ? slot0 + t : slot0 + t - p.R;
        Row4{p.k + (at << shift) * 4, p.ks + (at << (shift - 2))}.put(slot, word, shift, k, true);
        Row4{p.v + (at << shift) * 4, p.vs + (at << (shift - 2))}.put(slot, word, shift, v, true);
    }
    __syncthreads();  // every wave has read the count
    if (threadIdx.x == 0) p.count[b] = count + p.T_new;
}

// Values, in the order the rows were written: a thread takes eight dims of K and
// of V.
template <typename T>
__global__ __launch_bounds__(256) void read_rows4_kernel(Read4Params p) {
    const int h = blockIdx.y, b = blockIdx.z;
    const size_t head = (size_t)b * p.Hkv + h;
    const int shift = p.row_shift;
    const int count = p.count ? p.count[b] : p.R;
    const int n = min(max(count, 0), p.R), m = min(n, p.rows);
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t r = i >> shift;
    if (r >= (uint32_t)m) return;
    const int word = (int)(i & ((1u << shift) - 1));
    size_t row = (size_t)(count > p.R ? count % p.R : 0) + (n - m) + r;
    row -= row >= (size_t)p.R ? p.R : 0;
    row += head * p.R;
    const size_t at = (row << shift) + word, sat = (row << (shift - 2)) + (word >> 2);
    const uint32_t k = reinterpret_cast<const uint32_t *>(p.k)[at], v = reinterpret_cast<const uint32_t *>(p.v)[at];
    const uint32_t ks = (uint32_t)p.ks[sat] << 23, vs = (uint32_t)p.vs[sat] << 23;
    const size_t to = (((head * p.rows) << shift) + i) * 8;
    const auto out = [](T *o, uint32_t w, uint32_t s) {
        const uint4 y = bf16_word4(w, s);
        if constexpr (sizeof(T) == 2) {
            st16_nt(o, y);
        } else {
            float f[8];
            Vec16<uint16_t>::widen(y, f);
            st16_nt(o, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
            st16_nt(o + 4, make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])));
        }
    };
    out(static_cast<T *>(p.out_k) + to, k, ks);
    out(static_cast<T *>(p.out_v) + to, v, vs);
}

// Words of one (sequence, kv head)'s rows of 256: 2^29.  The kernels number words, and those
// of a last trip past them, in 32 bits, and a grid dimension holds less than 2^32 threads.
constexpr long long kMostWords = (long long)kCache4MaxRows * (256 / 8);
static_assert(kMostWords + 256 * kWriteTrip<true> <= 1LL << 31, "32-bit word numbers");

template <typename T, bool RING>
hipError_t launch_rows(const Write4Params &p, int rows, hipStream_t stream) {
    const long long words = (long long)rows << p.row_shift;  // kMostWords at most
    const dim3 grid((unsigned)((words + 256 * kWriteTrip<RING> - 1) / (256 * kWriteTrip<RING>)), p.Hkv, p.B);
    write_rows4_kernel<T, RING><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_append(const Write4Params &p, hipStream_t stream) {
    const long long words = ((long long)p.Hkv * p.T_new) << p.row_shift;
    if (words <= kAppendOneGroup4) {
        const int threads = std::min(1024, ((int)words + 63) / 64 * 64);
        append_rows4_kernel<T><<<p.B, threads, 0, stream>>>(p);
        return hipGetLastError();
    }
    if (hipError_t e = launch_rows<T, true>(p, p.T_new, stream); e != hipSuccess) return e;
    return launch_window_count(p.count, p.B, p.T_new, stream);
}

}  // namespace

hipError_t launch_gather4(const Write4Params &p, bool bf16, hipStream_t stream) {
    return bf16 ? launch_rows<uint16_t, false>(p, p.R, stream) : launch_rows<float, false>(p, p.R, stream);
}

hipError_t launch_append4(const Write4Params &p, bool bf16, hipStream_t stream) {
    return bf16 ? launch_append<uint16_t>(p, stream) : launch_append<float>(p, stream);
}

hipError_t launch_read4(const Read4Params &p, bool bf16, hipStream_t stream) {
    const long long words = (long long)p.rows << p.row_shift;  // kMostWords at most
    const dim3 grid((unsigned)((words + 255) / 256), p.Hkv, p.B);
    if (bf16) read_rows4_kernel<uint16_t><<<grid, 256, 0, stream>>>(p);
    else read_rows4_kernel<float><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace cmc
