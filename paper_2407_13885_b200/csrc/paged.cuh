// The paged cache of keys and values as the kernels see it, and the rules by which all of them read it.
//
// A sequence's keys lie in the pages that its row of the table names, page by page in order.  Table, lengths and starts are device
// data that the host has not seen, so nothing in them may lead a kernel out of bounds: a length counts as at least 0 and at most the
// table's capacity, and a place whose page lies outside the cache is neither read nor written.
#pragma once
#include <climits>
#include <cstdint>

#include "ptx.cuh"

namespace attnw {
namespace paged {

struct Cache {
    __nv_bfloat16 *K, *V;     // [pages, kv_heads, page, d]
    const int* table;         // [sequences, table_width]
    const int* lengths;       // [sequences], new tokens included
    int pages, kv_heads, page_shift, d, sequences, table_width;
};

__device__ __forceinline__ int length_of(const Cache& c, int b) {
    const long long capacity = static_cast<long long>(c.table_width) << c.page_shift;  // at most 2^31 - 1 (checked on the host)
    const int n = c.lengths[b];
    return n < 0 ? 0 : n > capacity ? static_cast<int>(capacity) : n;
}

// The page of key `at` (in [0, capacity)) of sequence `b`; -1 where the table names none of the cache.
__device__ __forceinline__ int page_of(const int* table, const Cache& c, int b, int at) {
    const int p = table[static_cast<size_t>(b) * c.table_width + (at >> c.page_shift)];
    return static_cast<unsigned>(p) < static_cast<unsigned>(c.pages) ? p : -1;
}

// Element offset of key `at`'s row in the cache, given its page.
__device__ __forceinline__ size_t row_offset(const Cache& c, int page, int h, int at) {
    const int in_page = at & ((1 << c.page_shift) - 1);
    return (((static_cast<size_t>(page) * c.kv_heads + h) << c.page_shift) + in_page) * c.d;
}

// The sequence that owns token `t` of the packed new tokens, whose sequence b has [starts[b], starts[b + 1]); -1 if none.  `starts` has
// been sampled to shared memory every `stride` entries (sample(starts)), so that most of the dependent loads are short ones.
constexpr int kSamples = 256;

struct Samples {
    int value[kSamples];
};

__device__ __forceinline__ int sample_stride(int sequences) { return (sequences + kSamples) / kSamples; }

// By all threads of the block; the caller synchronises it.
__device__ __forceinline__ void sample_starts(Samples* s, const int* starts, int sequences, int threads) {
    const int stride = sample_stride(sequences);
    for (int i = static_cast<int>(threadIdx.x); i < kSamples; i += threads) {
        const long long at = static_cast<long long>(i) * stride;
        s->value[i] = at <= sequences ? starts[at] : INT_MAX;
    }
}

__device__ __forceinline__ int owner_of(const Samples* s, const int* starts, int sequences, int t, int* end) {
    const int stride = sample_stride(sequences);
    int lo = 0;  // the last sample at or below t
#pragma unroll
    for (int step = kSamples / 2; step > 0; step >>= 1)
        if (s->value[lo + step] <= t) lo += step;
    lo *= stride;
    int hi = lo + stride < sequences ? lo + stride : sequences;  // starts[lo] <= t, and (where they ascend) t < starts[hi] or hi is the last
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= t) lo = mid; else hi = mid;
    }
    if (lo >= sequences) return -1;  // behind the last sequence
    *end = starts[lo + 1];
    return starts[lo] <= t && t < *end ? lo : -1;
}

}  // namespace paged
}  // namespace attnw
