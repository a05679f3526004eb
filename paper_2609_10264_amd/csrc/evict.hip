// Eviction from a paged cache by collected attention weight.
//
// Per (sequence, kv head) of n entries: keep the first `sinks`, the last
// `recent` and the r = m - sinks - recent heaviest others, m = min(n, budget),
// in order.  Two launches: evict_select finds the r-th largest weight by a
// radix descent over order-preserving 32-bit keys and writes the kept indices;
// evict_copy moves the kept rows.  Ties at the threshold go to the lowest
// indices, counted in order, so the choice does not depend on timing.
#include "kv.h"
#include "mvk_internal.h"

namespace mvk {

namespace {

constexpr uint32_t kSelThreads = 1024, kSelWaves = kSelThreads / 64;

// Unsigned keys in the order of the floats: -0 and 0 alike, not-a-numbers below all.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct EvictArgs {
    const float* w;
    size_t w_seq, w_head;
    float* wo;
    size_t o_seq, o_head;
    uint32_t budget, recent, sinks, shift;  // shift: of src
    int32_t* kept;
    int32_t* lens_out;
};

// Exclusive rank of this thread among the set flags of the workgroup, and their count.
__device__ __forceinline__ uint32_t block_rank(bool f, uint32_t* sm, uint32_t& total) {
    const uint64_t b = __ballot(f);
    const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    __syncthreads();
    if (lane == 0) sm[wave] = (uint32_t)__popcll(b);
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (uint32_t i = 0; i < kSelWaves; ++i) {
        const uint32_t c = sm[i];
        if (i < wave) before += c;
        sum += c;
    }
    total = sum;
    return before + (uint32_t)__popcll(b & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs a, SeqView sq) {
    __shared__ uint32_t hist[256], sm[2 * kSelWaves], pick[2];
    const uint32_t h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x;
    const uint32_t n = seq_entries(sq, a.shift, s), m = min(n, a.budget);
    const float* w = a.w + (size_t)s * a.w_seq + (size_t)h * a.w_head;
    float* wo = a.wo ? a.wo + (size_t)s * a.o_seq + (size_t)h * a.o_head : nullptr;
    int32_t* kept = a.kept + ((size_t)s * gridDim.x + h) * a.budget;
    if (h == 0 && tid == 0) a.lens_out[s] = (int32_t)m;
    for (uint32_t i = m + tid; i < a.budget; i += kSelThreads) kept[i] = -1;
    if (n <= a.budget) {
        for (uint32_t i = tid; i < n; i += kSelThreads) {
            kept[i] = (int32_t)i;
            if (wo) wo[i] = w[i];
        }
        return;
    }
    // here n > budget >= sinks + recent
    const uint32_t c0 = a.sinks, c1 = n - a.recent;
    uint32_t want = m - a.sinks - a.recent, prefix = 0;  // the want-th largest of the keys that begin with prefix
    if (want) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (uint32_t i = c0 + tid; i < c1; i += kSelThreads) {
                const uint32_t k = weight_key(w[i]);
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                uint32_t left = want, d = 255;
                while (left > hist[d]) left -= hist[d--];  // the digits' counts sum to at least want
                pick[0] = d;
                pick[1] = left;
            }
            __syncthreads();
            prefix |= pick[0] << shift;
            want = pick[1];
        }
    }
    // keys above prefix are kept, and the first `want` keys equal to it
    uint32_t base = 0, ties = 0;
    for (uint32_t i0 = 0; i0 < n; i0 += kSelThreads) {
        const uint32_t i = i0 + tid;
        const float x = i < n ? w[i] : 0.f;
        const bool fixed = i < c0 || i >= c1;
        const uint32_t k = weight_key(x);
        const bool other = i < n && !fixed && m > a.sinks + a.recent;
        uint32_t nt, nk;
        const bool tie = other && k == prefix;
        const uint32_t rt = block_rank(tie, sm, nt);
        const bool keep = i < n && (fixed || (other && (k > prefix || (tie && ties + rt < want))));
        const uint32_t rk = block_rank(keep, sm + kSelWaves, nk);
        if (keep) {
            kept[base + rk] = (int32_t)i;
            if (wo) wo[base + rk] = x;
        }
        base += nk;
        ties += nt;
    }
}

struct CopyArgs {
    KvView src, dst;
    SeqView sq;             // of src
    const int32_t* dtable;
    size_t dts;
    uint32_t dwidth, budget;
    const int32_t* kept;
};

// One thread per element (T: the element's size) or 16-byte granule of a kept row.
template <typename T>
__global__ __launch_bounds__(256) void evict_copy(CopyArgs a, uint32_t per) {
    const uint32_t h = blockIdx.y, s = blockIdx.z;
    const uint32_t m = min(seq_entries(a.sq, a.src.shift, s), a.budget);
    const size_t count = (size_t)m * per;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (size_t)gridDim.x * 256) {
        const uint32_t r = (uint32_t)(i / per), c = (uint32_t)(i % per);
        const uint32_t e = (uint32_t)a.kept[((size_t)s * gridDim.y + h) * a.budget + r];
        if ((r >> a.dst.shift) >= a.dwidth) continue;
        const int32_t dp = a.dtable[(size_t)s * a.dts + (r >> a.dst.shift)];
        if (dp < 0 || (uint32_t)dp >= a.dst.pages) continue;
        const uint32_t sp = seq_page(a.sq, a.src, s, e);
        const uint32_t se = e & ((1u << a.src.shift) - 1), de = r & ((1u << a.dst.shift) - 1);
        ((T*)a.dst.K)[dp * a.dst.kp + h * a.dst.kh + de * a.dst.ke + c] =
            ((const T*)a.src.K)[sp * a.src.kp + h * a.src.kh + se * a.src.ke + c];
        ((T*)a.dst.V)[dp * a.dst.vp + h * a.dst.vh + de * a.dst.ve + c] =
            ((const T*)a.src.V)[sp * a.src.vp + h * a.src.vh + se * a.src.ve + c];
    }
}

}  // namespace

hipError_t launch_evict(const KvView& src, const SeqView& sq, size_t elem, const float* w, size_t w_seq, size_t w_head,
                        uint32_t budget, uint32_t recent, uint32_t sinks, const KvView& dst, const int32_t* dtable,
                        size_t dts, uint32_t dwidth, float* wo, size_t o_seq, size_t o_head, int32_t* kept,
                        int32_t* lens_out, hipStream_t s) {
    const EvictArgs e = {w, w_seq, w_head, wo, o_seq, o_head, budget, recent, sinks, src.shift, kept, lens_out};
    hipLaunchKernelGGL(evict_select, dim3(src.heads, sq.count), dim3(kSelThreads), 0, s, e, sq);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const CopyArgs c = {src, dst, sq, dtable, dts, dwidth, budget, kept};
    const uint64_t cap = (uint64_t)sq.width << src.shift;
    const uint64_t most = (cap < budget ? cap : budget) * src.dim;
    const uint32_t grid = (uint32_t)(most / 256 + 1 < 4096 ? most / 256 + 1 : 4096);
    if (elem == 2)
        hipLaunchKernelGGL(evict_copy<uint16_t>, dim3(grid, src.heads, sq.count), dim3(256), 0, s, c, src.dim);
    else
        hipLaunchKernelGGL(evict_copy<uint32_t>, dim3(grid, src.heads, sq.count), dim3(256), 0, s, c, src.dim);
    return hipGetLastError();
}

}  // namespace mvk
