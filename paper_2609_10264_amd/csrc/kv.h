// Device views of the client's attention calls: rows of heads, the paged
// cache, the sequences, and the conversions of their values.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "field.h"
#include "mvk.h"

namespace mvk {

struct Rows {
    void* p;
    size_t token, head;  // strides in elements
    int type;
};

struct KvView {
    void *K, *V;
    size_t kp, kh, ke, vp, vh, ve;  // strides in elements: page, head, entry
    uint32_t pages, heads, shift, dim;  // 2^shift entries a page
};

struct SeqView {
    const int32_t *table, *lens, *q_start;
    size_t ts;
    uint32_t count, width;
};

// Entries of sequence s: within what its row of the table can hold.
__device__ __forceinline__ uint32_t seq_entries(const SeqView& sq, uint32_t shift, uint32_t s) {
    const int32_t n = sq.lens[s];
    const uint64_t cap = (uint64_t)sq.width << shift;
    return n <= 0 ? 0u : (uint64_t)n < cap ? (uint32_t)n : (uint32_t)cap;
}

// The token rows [q0, q0 + c) of sequence s (of T) and its entries n.
struct SeqSpan {
    uint32_t q0, c, n;
};
__device__ __forceinline__ SeqSpan seq_span(const SeqView& sq, uint32_t shift, uint32_t s, uint32_t T) {
    const int32_t a = sq.q_start[s], b = sq.q_start[s + 1];
    const uint32_t q0 = a < 0 ? 0u : min((uint32_t)a, T), q1 = b < 0 ? 0u : min((uint32_t)b, T);
    return {q0, q1 > q0 ? q1 - q0 : 0u, seq_entries(sq, shift, s)};
}

// The sequence of token row t: the last one that begins at or before it (0 if none does).
__device__ __forceinline__ uint32_t seq_of(const SeqView& sq, uint32_t t) {
    uint32_t lo = 0, hi = sq.count;  // q_start[lo] <= t (or lo == 0), q_start[hi] > t (or hi == count)
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (sq.q_start[mid] <= (int32_t)t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Page of entry j of sequence s (j within the table's width), for reading.
__device__ __forceinline__ uint32_t seq_page(const SeqView& sq, const KvView& kv, uint32_t s, uint32_t j) {
    const int32_t pg = sq.table[(size_t)s * sq.ts + (j >> kv.shift)];
    return pg < 0 ? 0u : min((uint32_t)pg, kv.pages - 1);
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__bf16 x) { return (float)x; }
__device__ __forceinline__ float to_float(_Float16 x) { return (float)x; }
template <typename T>
__device__ __forceinline__ T from_float(float x) { return (T)x; }

// A field element as the centred residue.  (The conversion rounds: 31 bits into 24.)
struct Field {
    uint32_t v;
};
__device__ __forceinline__ float field_lift(uint32_t y) {
    return (float)(y > kP / 2 ? (int32_t)(y - kP) : (int32_t)y);
}

// The field element of the integer nearest to x (ties to even; clamped to the
// centred residues; a not-a-number is 0).
__device__ __forceinline__ uint32_t field_of(float x) {
    constexpr int32_t half = (int32_t)((kP - 1) / 2);
    const float r = fminf(fmaxf(x == x ? rintf(x) : 0.f, -1.5e9f), 1.5e9f);
    const int32_t i = max(-half, min(half, (int32_t)r));
    return i < 0 ? kP + (uint32_t)i : (uint32_t)i;
}

// Element i of row data of a type known at run time.
__device__ __forceinline__ void store_as(void* p, int type, size_t i, float x, float inv_scale) {
    if (type == MVK_TYPE_BF16) ((__bf16*)p)[i] = (__bf16)x;
    else if (type == MVK_TYPE_F16) ((_Float16*)p)[i] = (_Float16)x;
    else if (type == MVK_TYPE_F32) ((float*)p)[i] = x;
    else ((uint32_t*)p)[i] = field_of(x * inv_scale);
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

}  // namespace mvk
