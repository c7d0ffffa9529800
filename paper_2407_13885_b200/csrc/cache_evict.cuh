// Eviction from a paged cache by accumulated attention weight: of a sequence that is longer than its budget, each key head keeps the
// latest `recent` keys and, of the others, those of most weight; they move together, in their order.
//
// evict_select: one CTA a row (sequence, key head).  The weights become integers of the same order; three passes of 11 bits find the
// smallest one that stays (a radix select: 11 bits, because the weights of a cache share their exponents' upper bits and a histogram of
// them would be one long queue of atomics at a few addresses), a fourth pass numbers the keys that stay.  Of equal weights at the
// border the lowest indices stay.  The passes read the row again, out of L2: three quarters of a microsecond each at 16384 keys.
//
// evict_move: to pages of their own, any CTA takes any keys.  In place, key t comes from index kept[t] >= t, so a row can be moved in
// ascending steps - all of a step read before any of it is written - and nothing is overwritten that a later step reads.  The steps of
// a row are one CTA's; for enough CTAs the row's features are dealt out, down to 32 bytes (a sector of DRAM) each, since the features of a key
// move alike.
#pragma once
#include <cstdint>

#include "paged.cuh"

namespace attnw {
namespace evict {

constexpr int kSelectThreads = 1024;
constexpr int kBins = 2048;

// Larger weight, larger integer; both zeros alike; a NaN is below every number.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct SelectSmem {
    uint32_t bins[kBins];
    uint32_t warp_sum[32];
    uint32_t digit, above;  // the chosen bin and the keys above it
};

// Inclusive sum over the block's threads; `total` to all.  One use between two __syncthreads of the caller's.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* warp_sum, uint32_t* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    uint32_t w = warp_sum[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    *total = __shfl_sync(0xffffffffu, w, 31);
    const uint32_t before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return x + (warp > 0 ? before : 0u);
}

__global__ void __launch_bounds__(kSelectThreads)
evict_select_kernel(paged::Cache cache, const float* mass, float* mass_out, int* kept, int* lengths_out, int budget, int recent, int capacity,
                    int capacity_out) {
    __shared__ SelectSmem sm;
    const int tid = static_cast<int>(threadIdx.x);
    const int b = static_cast<int>(blockIdx.x) / cache.kv_heads;
    ptx::grid_dependency_wait();
    const float* row = mass + static_cast<size_t>(blockIdx.x) * capacity;
    float* out = mass_out + static_cast<size_t>(blockIdx.x) * capacity_out;
    int* keep = kept + static_cast<size_t>(blockIdx.x) * budget;
    const int length = paged::length_of(cache, b);
    const int left = min(length, budget);
    if (tid == 0 && blockIdx.x % cache.kv_heads == 0) lengths_out[b] = left;
    const int old = length > budget ? length - recent : 0;  // the keys to choose from; the others up to `length` stay
    const int chosen = length > budget ? budget - recent : 0;

    if (chosen > 0) {
        uint32_t prefix = 0, mask = 0, need = static_cast<uint32_t>(chosen);
        constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = kShift[pass], bins = 1 << kBits[pass];
            for (int i = tid; i < kBins; i += kSelectThreads) sm.bins[i] = 0;
            __syncthreads();
            for (int i0 = 0; i0 < old; i0 += kSelectThreads) {
                const int i = i0 + tid;
                const uint32_t key = i < old ? order_of(row[i]) : 0u;
                const bool in = i < old && (key & mask) == prefix;
                const uint32_t bin = (key >> shift) & static_cast<uint32_t>(bins - 1);
                // (a row of equal weights would be one queue: a warp of equals adds once)
                int same;
                __match_all_sync(0xffffffffu, in ? bin : 0xffffffffu, &same);
                if (same) {
                    if (in && (tid & 31) == 0) atomicAdd(&sm.bins[bin], 32u);
                } else if (in) {
                    atomicAdd(&sm.bins[bin], 1u);
                }
            }
            __syncthreads();
            // from the largest bin down: the one in which the sum reaches `need`
            const int hi = bins - 1 - 2 * tid;  // this thread's bins hi and hi - 1
            const uint32_t c0 = hi >= 1 ? sm.bins[hi] : 0u, c1 = hi >= 1 ? sm.bins[hi - 1] : 0u;
            uint32_t total;
            const uint32_t upto = block_scan(c0 + c1, sm.warp_sum, &total), before = upto - c0 - c1;
            if (before < need && need <= upto) {
                const bool first = need <= before + c0;
                sm.digit = static_cast<uint32_t>(first ? hi : hi - 1);
                sm.above = first ? before : before + c0;
            }
            __syncthreads();
            prefix |= sm.digit << shift;
            mask |= static_cast<uint32_t>(bins - 1) << shift;
            need -= sm.above;
        }
        // `prefix` is the smallest weight that stays; of those equal to it the first `need`.
        uint32_t done_above = 0, done_equal = 0;
        for (int i0 = 0; i0 < old; i0 += 4 * kSelectThreads) {
            float x[4];
            uint32_t counts = 0;  // above in the low half, equal in the high half
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + 4 * tid + e;
                x[e] = i < old ? row[i] : 0.0f;
                const uint32_t key = i < old ? order_of(x[e]) : 0u;
                counts += i < old && key > prefix ? 1u : i < old && key == prefix ? 0x10000u : 0u;
            }
            uint32_t total;
            const uint32_t before = block_scan(counts, sm.warp_sum, &total) - counts;  // (its barriers: all have read before any writes)
            uint32_t above = done_above + (before & 0xffffu), equal = done_equal + (before >> 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = i0 + 4 * tid + e;
                if (i >= old) break;
                const uint32_t key = order_of(x[e]);
                if (key > prefix || (key == prefix && equal < need)) {
                    const uint32_t at = above + min(equal, need);
                    keep[at] = i;
                    out[at] = x[e];
                }
                above += key > prefix ? 1u : 0u;
                equal += key == prefix ? 1u : 0u;
            }
            done_above += total & 0xffffu;
            done_equal += total >> 16;
        }
    }
    // the keys that stay anyway; nothing behind them
    for (int t0 = chosen; t0 < left; t0 += kSelectThreads) {
        const int t = t0 + tid;
        const float x = t < left ? row[old + t - chosen] : 0.0f;
        __syncthreads();
        if (t < left) {
            keep[t] = old + t - chosen;
            out[t] = x;
        }
        __syncthreads();
    }
    for (int t = left + tid; t < budget; t += kSelectThreads) keep[t] = -1;
    for (int t = left + tid; t < capacity_out; t += kSelectThreads) out[t] = 0.0f;
}

constexpr int kMoveThreads = 256;
constexpr int kFlight = 8;  // 16-byte pieces of a thread in flight

// Grid: x over (steps of keys, if they go to pages of their own) x slices of the features, y over rows, z over keys and values.
template <bool IN_PLACE>
__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(paged::Cache cache, const int* table_out, int table_out_width, const int* kept, int budget, int slices) {
    ptx::grid_dependency_wait();
    const int pieces = cache.d / 8 / slices;  // of a key, this CTA's: a power of two
    const int slice = static_cast<int>(blockIdx.x) % slices;
    const int row = static_cast<int>(blockIdx.y), b = row / cache.kv_heads, h = row % cache.kv_heads;
    const int left = min(paged::length_of(cache, b), budget);
    const int* keep = kept + static_cast<size_t>(row) * budget;
    uint4* data = reinterpret_cast<uint4*>(blockIdx.z == 0 ? cache.K : cache.V);
    const int keys = kMoveThreads * kFlight / pieces;  // of a step
    const int piece = static_cast<int>(threadIdx.x) % pieces + slice * pieces, first = static_cast<int>(threadIdx.x) / pieces;
    const int stride = kMoveThreads / pieces;
    // the target's page comes from its own table, which may be narrower
    auto target_page = [&](int t) {
        const int p = table_out[static_cast<size_t>(b) * table_out_width + (t >> cache.page_shift)];
        return static_cast<unsigned>(p) < static_cast<unsigned>(cache.pages) ? p : -1;
    };
    uint4 v[kFlight];
    long long to[kFlight];
    auto load = [&](int t0) {
        int from[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int t = t0 + first + i * stride;
            from[i] = t < left ? keep[t] : -1;
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int t = t0 + first + i * stride;
            to[i] = -1;
            if (from[i] < 0 || (IN_PLACE && from[i] == t)) continue;
            const int page = paged::page_of(cache.table, cache, b, from[i]), page_to = target_page(t);
            if (page < 0 || page_to < 0) continue;
            to[i] = static_cast<long long>(paged::row_offset(cache, page_to, h, t) / 8 + piece);
            v[i] = __ldcs(data + paged::row_offset(cache, page, h, from[i]) / 8 + piece);
        }
    };
    auto store = [&]() {
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (to[i] >= 0) data[to[i]] = v[i];
    };
    if constexpr (IN_PLACE) {
        for (int t0 = 0; t0 < left; t0 += keys) {
            load(t0);
            __syncthreads();  // all of a step is read before any of it is written
            store();
        }
    } else {
        load(static_cast<int>(blockIdx.x) / slices * keys);
        store();
    }
}

}  // namespace evict
}  // namespace attnw
