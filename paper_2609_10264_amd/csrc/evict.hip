// Eviction from a paged cache by collected attention weight.
//
// Per (sequence, kv head) of n entries: keep the first `sinks`, the last
// `recent` and the r = m - sinks - recent heaviest others, m = min(n, budget),
// in order.  Two launches: evict_select finds the r-th largest weight, as an
// order-preserving 32-bit key, and writes the kept indices; evict_copy moves
// the kept rows.  Ties at the threshold go to the lowest indices, counted in
// order, so the choice does not depend on timing.
//
// The search is a chain of compares, counts and barriers on one compute unit a row:
// 12.7 us for 32 rows of 4096, 43 for 96 rows of up to 32768.  The copy is bound by
// memory: 138 us for 660 MB (8191 kept of each of those rows), 4.8 TB/s.
#include <algorithm>

#include "kv.h"
#include "mvk_internal.h"

namespace mvk {

namespace {

constexpr uint32_t kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr uint32_t kListKeys = 4096;  // keys of a list in LDS

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
};

// Where a search stands: the want-th largest of the candidates' keys lies in
// [x, x + 2^bit); lo keys are >= x, hi are >= x + 2^bit (hi < want <= lo).
struct Search {
    uint32_t x, bit, lo, hi, want;
    __device__ __forceinline__ bool done() const { return bit == 0 || lo == want; }
    __device__ __forceinline__ bool holds(uint32_t k) const { return k && k >= x && (bit == 32 || (k - x) >> bit == 0); }
};

// One step of kBits bits.  count(c): this wave's keys >= c.
template <uint32_t kBits, typename Count>
__device__ __forceinline__ void search_step(Search& s, Count count, uint32_t (*sm)[3][kSelWaves], uint32_t& turn) {
    const uint32_t bits = min(kBits, s.bit), unit = 1u << (s.bit - bits), wave = threadIdx.x >> 6;
    uint32_t(*c)[kSelWaves] = sm[turn];  // two in turn: one barrier a step
    turn ^= 1;
    constexpr uint32_t kCands = (1u << kBits) - 1;
#pragma unroll
    for (uint32_t i = 0; i < kCands; ++i) {
        const uint32_t n = count(s.x + (i + 1) * unit);
        if ((threadIdx.x & 63) == 0) c[i][wave] = n;
    }
    __syncthreads();
    const uint32_t x0 = s.x;
    s.bit -= bits;
#pragma unroll
    for (uint32_t i = 0; i < kCands; ++i) {
        if (i + 1 >= 1u << bits) break;
        uint32_t sum = 0;
#pragma unroll
        for (uint32_t w = 0; w < kSelWaves; ++w) sum += c[i][w];
        if (sum >= s.want) s.x = x0 + (i + 1) * unit, s.lo = sum;
        else if (sum > s.hi) s.hi = sum;
    }
}

// The rest of a search among the `n` keys of a list in LDS (those in its range), two
// bits a step.
template <uint32_t kMost>
__device__ __forceinline__ void search_list(Search& s, const uint32_t* list, uint32_t n, uint32_t (*sm)[3][kSelWaves],
                                            uint32_t& turn) {
    constexpr uint32_t kEach = kMost / kSelThreads;
    uint32_t k[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = i * kSelThreads + threadIdx.x;
        k[i] = e < n ? list[e] : 0u;
    }
    const uint32_t above = s.hi;  // keys beyond the range are not in the list
    s.want -= above, s.lo -= above, s.hi = 0;
    while (!s.done())
        search_step<2>(
            s,
            [&](uint32_t c) {
                uint32_t m = 0;
#pragma unroll
                for (uint32_t i = 0; i < kEach; ++i) m += (uint32_t)__popcll(__ballot(k[i] >= c));
                return m;
            },
            sm, turn);
    s.want += above, s.lo += above, s.hi += above;
}

// Appends the keys that the search's range holds to the list (in any order: only their values count).
__device__ __forceinline__ void append(uint32_t* list, uint32_t* size, bool f, uint32_t k) {
    const uint64_t b = __ballot(f);
    if (!b) return;
    const uint32_t lane = threadIdx.x & 63;
    uint32_t at = 0;
    if (lane == 0) at = atomicAdd(size, (uint32_t)__popcll(b));
    at = (uint32_t)__shfl((int)at, 0);
    if (f) list[at + (uint32_t)__popcll(b & ((1ull << lane) - 1))] = k;
}

// Exclusive prefix sums of sm[0, kCount), in place, and the total (wave 0 scans).
template <uint32_t kCount>
__device__ __forceinline__ uint32_t scan_counts(uint32_t* sm, uint32_t* total) {
    __syncthreads();
    if (threadIdx.x < 64) {
        constexpr uint32_t kPer = (kCount + 63) / 64;
        const uint32_t lane = threadIdx.x;
        uint32_t c[kPer], sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i) {
            const uint32_t at = lane * kPer + i;
            c[i] = at < kCount ? sm[at] : 0u;
            sum += c[i];
        }
        uint32_t incl = sum;
#pragma unroll
        for (uint32_t s = 1; s < 64; s <<= 1) {
            const uint32_t y = (uint32_t)__shfl_up((int)incl, s);
            if (lane >= s) incl += y;
        }
        uint32_t run = incl - sum;
#pragma unroll
        for (uint32_t i = 0; i < kPer; ++i) {
            const uint32_t at = lane * kPer + i;
            if (at < kCount) sm[at] = run;
            run += c[i];
        }
        if (lane == 63) *total = incl;
    }
    __syncthreads();
    return *total;
}

// Rows of up to kEach * kSelThreads entries: the keys stay in registers, entry
// i * kSelThreads + tid in register i, so a step of the search is a compare and
// the count of a lane mask for each.
template <uint32_t kEach>
__device__ __forceinline__ void select_in_registers(const EvictArgs& a, const float* w, float* wo, int32_t* kept,
                                                    uint32_t n, uint32_t want, uint32_t (*sm)[3][kSelWaves],
                                                    uint32_t* counts, uint32_t* tied, uint32_t* total, uint32_t* list) {
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c0 = a.sinks, c1 = n - a.recent;
    uint32_t k[kEach];
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = i * kSelThreads + tid;
        k[i] = __float_as_uint(e < n ? w[e] : 0.f);
    }
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t e = i * kSelThreads + tid;
        // 0 stands for what is no candidate, so the least candidate key is 1
        k[i] = e >= c0 && e < c1 ? max(weight_key(__uint_as_float(k[i])), 1u) : 0u;
    }
    Search s = {0, 32, c1 - c0, 0, want};
    uint32_t turn = 0;
    auto count = [&](uint32_t c) {
        uint32_t m = 0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) m += (uint32_t)__popcll(__ballot(k[i] >= c));
        return m;
    };
    if (want) {
        if (kEach * kSelThreads <= kListKeys) {
            while (!s.done()) search_step<2>(s, count, sm, turn);
        } else {
            // until few keys are left in the range, then among those alone
            while (!s.done() && s.lo - s.hi > kListKeys) search_step<1>(s, count, sm, turn);
            if (!s.done()) {
                if (tid == 0) *total = 0;
                __syncthreads();
#pragma unroll
                for (uint32_t i = 0; i < kEach; ++i) append(list, total, s.holds(k[i]), k[i]);
                __syncthreads();
                search_list<kListKeys>(s, list, s.lo - s.hi, sm, turn);
            }
        }
    }
    const uint32_t thr = want ? s.x : 0xffffffffu;
    const bool exact = !want || s.lo == want;
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
    uint32_t ties = 0xffffffffu;  // how many of the keys equal to thr are kept
    if (!exact) {
        // keys above thr are kept, and the first of those equal to it
        uint32_t more = 0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
            more += (uint32_t)__popcll(__ballot(k[i] > thr));
            const uint32_t c = (uint32_t)__popcll(__ballot(k[i] == thr));
            if (lane == 0) tied[i * kSelWaves + wave] = c;
        }
        if (lane == 0) sm[0][0][wave] = more;
        scan_counts<kEach * kSelWaves>(tied, total);
        uint32_t sum = 0;
#pragma unroll
        for (uint32_t i = 0; i < kSelWaves; ++i) sum += sm[0][0][i];
        ties = want - sum;
    }
    auto keep = [&](uint32_t i) {
        const uint32_t e = i * kSelThreads + tid;
        bool f = want && (exact ? k[i] >= thr : k[i] > thr);
        if (!exact) {
            const uint64_t b = __ballot(k[i] == thr);
            f |= k[i] == thr && tied[i * kSelWaves + wave] + (uint32_t)__popcll(b & below) < ties;
        }
        return e < n && (e < c0 || e >= c1 || f);
    };
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t c = (uint32_t)__popcll(__ballot(keep(i)));
        if (lane == 0) counts[i * kSelWaves + wave] = c;
    }
    scan_counts<kEach * kSelWaves>(counts, total);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const bool f = keep(i);
        const uint64_t b = __ballot(f);
        if (f) {
            const uint32_t e = i * kSelThreads + tid;
            const uint32_t r = counts[i * kSelWaves + wave] + (uint32_t)__popcll(b & below);
            kept[r] = (int32_t)e;
            if (wo) wo[r] = w[e];
        }
    }
}

__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs a, SeqView sq) {
    __shared__ uint32_t sm[2][3][kSelWaves], counts[32 * kSelWaves], tied[32 * kSelWaves], total, list[kListKeys];
    const uint32_t h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const uint32_t n = seq_entries(sq, a.shift, s), m = min(n, a.budget);
    const float* w = a.w + (size_t)s * a.w_seq + (size_t)h * a.w_head;
    float* wo = a.wo ? a.wo + (size_t)s * a.o_seq + (size_t)h * a.o_head : nullptr;
    int32_t* kept = a.kept + ((size_t)s * gridDim.x + h) * a.budget;
    for (uint32_t i = m + tid; i < a.budget; i += kSelThreads) kept[i] = -1;
    if (n <= a.budget) {
        for (uint32_t i = tid; i < n; i += kSelThreads) {
            kept[i] = (int32_t)i;
            if (wo) wo[i] = w[i];
        }
        return;
    }
    // here n > budget >= sinks + recent
    const uint32_t want = m - a.sinks - a.recent;
    if (n <= kListKeys) return select_in_registers<kListKeys / kSelThreads>(a, w, wo, kept, n, want, sm, counts, tied, &total, list);
    if (n <= 32 * kSelThreads) return select_in_registers<32>(a, w, wo, kept, n, want, sm, counts, tied, &total, list);
    // longer rows: each step reads the weights again (they stay in L2)
    const uint32_t c0 = a.sinks, c1 = n - a.recent;
    auto key = [&](uint32_t e) { return e >= c0 && e < c1 ? max(weight_key(w[e]), 1u) : 0u; };
    auto count_if = [&](auto pick) {
        uint32_t c = 0;
        for (uint32_t e0 = 0; e0 < n; e0 += kSelThreads) {
            const uint32_t e = e0 + tid;
            c += (uint32_t)__popcll(__ballot(e < n && pick(key(min(e, n - 1)))));
        }
        return c;
    };
    Search s_ = {0, 32, c1 - c0, 0, want};
    uint32_t turn = 0, ties = 0xffffffffu;
    if (want) {
        while (!s_.done() && s_.lo - s_.hi > kListKeys)
            search_step<1>(s_, [&](uint32_t c) { return count_if([c](uint32_t k) { return k >= c; }); }, sm, turn);
        if (!s_.done()) {
            if (tid == 0) total = 0;
            __syncthreads();
            for (uint32_t e0 = 0; e0 < n; e0 += kSelThreads) {
                const uint32_t k = e0 + tid < n ? key(e0 + tid) : 0u;
                append(list, &total, s_.holds(k), k);
            }
            __syncthreads();
            search_list<kListKeys>(s_, list, s_.lo - s_.hi, sm, turn);
        }
    }
    const uint32_t thr = want ? s_.x : 0xffffffffu;
    const bool exact = !want || s_.lo == want;
    __syncthreads();
    if (!exact) {
        const uint32_t more = count_if([thr](uint32_t k) { return k > thr; });
        if (lane == 0) sm[0][0][wave] = more;
        __syncthreads();
        uint32_t sum = 0;
        for (uint32_t i = 0; i < kSelWaves; ++i) sum += sm[0][0][i];
        ties = want - sum;
        __syncthreads();
    }
    uint32_t base = 0, seen = 0;  // kept entries and ties before this block of entries
    const uint64_t below = (1ull << lane) - 1;
    for (uint32_t e0 = 0; e0 < n; e0 += kSelThreads) {
        const uint32_t e = e0 + tid;
        const uint32_t k = e < n ? key(e) : 0u;
        const bool fixed = e < n && (e < c0 || e >= c1);
        uint32_t rank = 0;
        if (!exact) {
            const uint64_t b = __ballot(k == thr);
            if (lane == 0) counts[wave] = (uint32_t)__popcll(b);
            const uint32_t nt = scan_counts<kSelWaves>(counts, &total);
            rank = seen + counts[wave] + (uint32_t)__popcll(b & below);
            seen += nt;
            __syncthreads();
        }
        const bool f = fixed || (want && k && (exact ? k >= thr : k > thr || (k == thr && rank < ties)));
        const uint64_t b = __ballot(f);
        if (lane == 0) counts[wave] = (uint32_t)__popcll(b);
        const uint32_t nk = scan_counts<kSelWaves>(counts, &total);
        if (f) {
            const uint32_t r = base + counts[wave] + (uint32_t)__popcll(b & below);
            kept[r] = (int32_t)e;
            if (wo) wo[r] = w[e];
        }
        base += nk;
        __syncthreads();
    }
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct CopyArgs {
    KvView src, dst;
    SeqView sq;             // of src
    const int32_t* dtable;
    size_t dts;
    uint32_t dwidth, budget, most;  // most: rows that a sequence may keep
    const int32_t* kept;
    int32_t* lens_out;
};

// kRowsEach rows a group of threads that holds one, T (an element or a 16-byte
// granule) a thread; their loads are in flight together.  dims: T's a row.
// How many rows there are is read from `kept` (-1 beyond them), not from the
// lengths: lens_out, written here, may be their place.
constexpr uint32_t kRowsEach = 4;
template <typename T>
__global__ __launch_bounds__(256) void evict_copy(CopyArgs a, uint32_t dims, uint32_t per) {
    const uint32_t h = blockIdx.y, s = blockIdx.z;
    const uint32_t group = threadIdx.x / per, rows = 256 / per;  // rows at once: per threads each
    if (group >= rows) return;
    const int32_t* kept = a.kept + ((size_t)s * gridDim.y + h) * a.budget;
    for (uint32_t r0 = blockIdx.x * rows * kRowsEach + group; r0 < a.most; r0 += gridDim.x * rows * kRowsEach) {
        int32_t at[kRowsEach];
#pragma unroll
        for (uint32_t u = 0; u < kRowsEach; ++u) {
            const uint32_t r = r0 + u * rows;
            at[u] = r < a.most ? kept[r] : -1;
        }
        if (h == 0 && threadIdx.x % per == 0) {
            // of each sequence one thread finds the last row, or that there is none
#pragma unroll
            for (uint32_t u = 0; u < kRowsEach; ++u) {
                const uint32_t r = r0 + u * rows;
                if (at[u] >= 0 && (r + 1 == a.most || kept[r + 1] < 0)) a.lens_out[s] = (int32_t)(r + 1);
                if (at[u] < 0 && r == 0) a.lens_out[s] = 0;
            }
        }
        if (at[0] < 0) return;  // (none of the later rows has one)
        size_t ks[kRowsEach], vs[kRowsEach], kd[kRowsEach], vd[kRowsEach];
        bool on[kRowsEach];
#pragma unroll
        for (uint32_t u = 0; u < kRowsEach; ++u) {
            const uint32_t r = at[u] < 0 ? r0 : r0 + u * rows, e = (uint32_t)(at[u] < 0 ? at[0] : at[u]);
            const uint32_t slot = r >> a.dst.shift;
            const uint32_t sp = seq_page(a.sq, a.src, s, e), se = e & ((1u << a.src.shift) - 1);
            const int32_t dp = slot < a.dwidth ? a.dtable[(size_t)s * a.dts + slot] : -1;
            on[u] = at[u] >= 0 && dp >= 0 && (uint32_t)dp < a.dst.pages;
            const uint32_t de = r & ((1u << a.dst.shift) - 1);
            ks[u] = sp * a.src.kp + h * a.src.kh + se * a.src.ke;
            vs[u] = sp * a.src.vp + h * a.src.vh + se * a.src.ve;
            kd[u] = dp * a.dst.kp + h * a.dst.kh + de * a.dst.ke;
            vd[u] = dp * a.dst.vp + h * a.dst.vh + de * a.dst.ve;
        }
        for (uint32_t c = threadIdx.x % per; c < dims; c += per) {
            T k[kRowsEach], v[kRowsEach];
#pragma unroll
            for (uint32_t u = 0; u < kRowsEach; ++u) {
                k[u] = ((const T*)a.src.K)[ks[u] + c];
                v[u] = ((const T*)a.src.V)[vs[u] + c];
            }
#pragma unroll
            for (uint32_t u = 0; u < kRowsEach; ++u)
                if (on[u]) {
                    ((T*)a.dst.K)[kd[u] + c] = k[u];
                    ((T*)a.dst.V)[vd[u] + c] = v[u];
                }
        }
    }
}

// The view with strides in granules of `per` values; false where they are not whole.
bool in_granules(KvView& v, uint32_t per) {
    if ((uintptr_t)v.K % 16 || (uintptr_t)v.V % 16 || v.dim % per || (v.kp | v.kh | v.ke | v.vp | v.vh | v.ve) % per)
        return false;
    v.kp /= per, v.kh /= per, v.ke /= per, v.vp /= per, v.vh /= per, v.ve /= per;
    return true;
}

}  // namespace

hipError_t launch_evict(const KvView& src, const SeqView& sq, size_t elem, const float* w, size_t w_seq, size_t w_head,
                        uint32_t budget, uint32_t recent, uint32_t sinks, const KvView& dst, const int32_t* dtable,
                        size_t dts, uint32_t dwidth, float* wo, size_t o_seq, size_t o_head, int32_t* kept,
                        int32_t* lens_out, hipStream_t s) {
    const EvictArgs e = {w, w_seq, w_head, wo, o_seq, o_head, budget, recent, sinks, src.shift, kept};
    hipLaunchKernelGGL(evict_select, dim3(src.heads, sq.count), dim3(kSelThreads), 0, s, e, sq);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    const uint64_t cap = (uint64_t)sq.width << src.shift;
    const uint32_t most = (uint32_t)(cap < budget ? cap : budget);
    CopyArgs c = {src, dst, sq, dtable, dts, dwidth, budget, most, kept, lens_out};
    auto go = [&](auto kernel, uint32_t dims) {
        uint32_t per = 1;
        while (per < dims && per < 256) per *= 2;
        const uint32_t each = 256 / per * kRowsEach;
        // (one launch takes fewer than 2^32 threads an axis)
        const dim3 grid(std::min((most + each - 1) / each, 1u << 22), src.heads, sq.count);
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, c, dims, per);
        return hipGetLastError();
    };
    const uint32_t per = (uint32_t)(16 / elem);
    if (in_granules(c.src, per) && in_granules(c.dst, per)) return go(evict_copy<u32x4>, src.dim / per);
    c.src = src, c.dst = dst;
    return elem == 2 ? go(evict_copy<uint16_t>, src.dim) : go(evict_copy<uint32_t>, src.dim);
}

}  // namespace mvk
