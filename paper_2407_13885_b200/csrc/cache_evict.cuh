// Eviction from a paged cache by accumulated attention weight: of a sequence that is longer than its budget, each key head keeps the
// latest `recent` keys and, of the others, those of most weight; they move together, in their order.
//
// evict_select: one CTA a row (sequence, key head).  The weights become integers of the same order; a histogram of their upper 13 bits (sign, exponent
// and four digits: the weights of a cache share their exponents' upper bits, and few bins would be a queue of atomics at each) tells which stay, but for
// those of one bin, of which the largest have room.  If that bin has at most kList weights, each counts those in front of it; if not, another 11 and 8
// bits, and of weights that are equal to the last bit the first ones stay.  Who stays is a bit a key in shared memory; a sum over the words' bits gives
// the new places.  Up to 16384 keys are read once, into registers; longer rows in turns of as many, again for each step (out of L2).
//
// evict_move: to pages of their own, any CTA takes any keys.  In place, key t comes from index kept[t] >= t, so a row can be moved in
// ascending steps - all of a step read before any of it is written - and nothing is overwritten that a later step reads.  The steps of
// a row are one CTA's; for enough CTAs the row's features are dealt out, down to 32 bytes (a sector of DRAM) each, since the features of a key
// move alike.
//
// Bound by HBM where rows are many: 128 rows of up to 16384 keys of 128 features to 4096 take 100 us to other pages and 109 in place (the bytes 73), 17 of them
// evict_select, whose one CTA a row works through its histogram, the others evict_move.  In place a step's reads end before its writes begin; to other pages
// reads and writes of all CTAs mix, and what keeps them at 5.7 TB/s has not been found.  8 rows of 4096 to 2048: 13.1 us to other pages, 17.0 in place, two
// launches' latency and one CTA a row.  More than 16384 keys a row: 32 rows of 40000 to 8000 87 and 113 us (the bytes 41).
#pragma once
#include <cstdint>

#include "paged.cuh"

namespace attnw {
namespace evict {

constexpr int kSelectThreads = 1024;
constexpr int kBins = 8192, kBinsEach = kBins / kSelectThreads;
constexpr int kHeld = 16;                             // weights that a thread holds
constexpr int kRound = kSelectThreads * kHeld;        // keys of a turn
constexpr int kList = 1024;

// Larger weight, larger integer; both zeros alike; a NaN is below every number.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);  // (-0 + 0 is +0)
    const uint32_t k = u ^ (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u);
    return x == x ? k : 0u;
}

struct SelectSmem {
    uint32_t bins[kBins];
    uint32_t warp_sum[32];
    uint32_t digit, above, in_bin;  // the chosen bin, the keys above it, and in it
    uint32_t listed;
    unsigned long long list[kList];  // weight's integer << 32 | ~index: the larger, the earlier
    // then dynamic: words of bits, [turns' words] and the sums in front of them
};

// Inclusive sum over the block's threads; `total` to all.
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
    __shared__ uint32_t words[kRound / 32], equals[kRound / 32], before[kRound / 32];  // of a turn
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = tid >> 5;
    const int b = static_cast<int>(blockIdx.x) / cache.kv_heads;
    ptx::grid_dependency_wait();
    const float* row = mass + static_cast<size_t>(blockIdx.x) * capacity;
    float* out = mass_out + static_cast<size_t>(blockIdx.x) * capacity_out;
    int* keep = kept + static_cast<size_t>(blockIdx.x) * budget;
    // This thread's weights of a turn, as integers: word (e * 32 + warp) of the turn's, bit `lane`.
    uint32_t key[kHeld];
    auto index_of = [&](int turn0, int e) { return turn0 + (e * 32 + warp) * 32 + lane; };
    auto values = [&](int turn0, int end, float (&x)[kHeld]) {  // (all loads, then what is made of them: one latency)
#pragma unroll
        for (int e = 0; e < kHeld; ++e) {
            const int i = index_of(turn0, e);
            x[e] = i < end ? row[i] : 0.0f;
        }
    };
    auto load = [&](int turn0, int end) {
        float x[kHeld];
        values(turn0, end, x);
#pragma unroll
        for (int e = 0; e < kHeld; ++e) key[e] = order_of(x[e]);
    };
    load(0, capacity);  // (beside the length)
    const int length = paged::length_of(cache, b);
    const int left = min(length, budget);
    if (tid == 0 && blockIdx.x % cache.kv_heads == 0) lengths_out[b] = left;
    const int old = length > budget ? length - recent : 0;  // the keys to choose from; the others up to `length` stay
    const int chosen = length > budget ? budget - recent : 0;

    if (chosen > 0) {
        const bool once = old <= kRound;
        for (int i = tid; i < kBins; i += kSelectThreads) sm.bins[i] = 0;
        if (tid == 0) sm.listed = 0;
        __syncthreads();
        // ---- the smallest weight that stays, as far as needed: all bits of `mask` ----
        uint32_t prefix = 0, mask = 0, need = static_cast<uint32_t>(chosen), shift = 19, bits = 13;
        for (;;) {
            for (int turn0 = 0; turn0 < old; turn0 += kRound) {
                if (!once) load(turn0, old);
#pragma unroll
                for (int e = 0; e < kHeld; ++e) {
                    const int i = index_of(turn0, e);
                    if (i - lane >= old) break;  // (the whole warp)
                    if (i < old && (key[e] & mask) == prefix) atomicAdd(&sm.bins[(key[e] >> shift) & ((1u << bits) - 1u)], 1u);
                }
            }
            __syncthreads();
            // from the largest bin down: the one in which the sum reaches `need`
            const int hi = (1 << bits) - 1 - kBinsEach * tid;  // this thread's bins hi ... hi - kBinsEach + 1
            uint32_t c[kBinsEach], own = 0;
#pragma unroll
            for (int k = 0; k < kBinsEach; ++k) {
                c[k] = hi - k >= 0 ? sm.bins[hi - k] : 0u;
                own += c[k];
            }
            uint32_t total, in_front = block_scan(own, sm.warp_sum, &total) - own;
            if (in_front < need && need <= in_front + own) {
#pragma unroll
                for (int k = 0; k < kBinsEach; ++k) {
                    if (in_front < need && need <= in_front + c[k]) {
                        sm.digit = static_cast<uint32_t>(hi - k);
                        sm.above = in_front;
                        sm.in_bin = c[k];
                    }
                    in_front += c[k];
                }
            }
            __syncthreads();
            prefix |= sm.digit << shift;
            mask |= ((1u << bits) - 1u) << shift;
            need -= sm.above;
            if (sm.in_bin <= kList || shift == 0) break;
            bits = shift == 19 ? 11 : 8;
            shift = shift == 19 ? 8 : 0;
            for (int i = tid; i < kBins; i += kSelectThreads) sm.bins[i] = 0;
            __syncthreads();
        }
        // Of those with the prefix the first `need` stay, by weight, then by index: all weights above `border`, and those equal to it up to index
        // `last` (by_list) or the first `need` (then mask has all bits).
        const bool by_list = sm.in_bin <= kList;
        uint32_t border = prefix;
        int last = -1;
        if (by_list) {
            for (int turn0 = 0; turn0 < old; turn0 += kRound) {
                if (!once) load(turn0, old);
#pragma unroll
                for (int e = 0; e < kHeld; ++e) {
                    const int i = index_of(turn0, e);
                    if (i - lane >= old) break;
                    if (i < old && (key[e] & mask) == prefix)
                        sm.list[atomicAdd(&sm.listed, 1u)] = static_cast<unsigned long long>(key[e]) << 32 | static_cast<uint32_t>(~i);
                }
            }
            __syncthreads();
            const int n = static_cast<int>(sm.listed);
            if (tid < n) {
                const unsigned long long mine = sm.list[tid];
                uint32_t in_front = 0;
#pragma unroll 8
                for (int i = 0; i < n; ++i) in_front += sm.list[i] > mine ? 1u : 0u;
                if (in_front + 1u == need) {  // one of them
                    sm.digit = static_cast<uint32_t>(mine >> 32);
                    sm.above = ~static_cast<uint32_t>(mine);
                }
            }
            __syncthreads();
            border = sm.digit;
            last = static_cast<int>(sm.above);
        }
        // ---- the new places ----
        uint32_t done = 0, done_equal = 0;
        for (int turn0 = 0; turn0 < old; turn0 += kRound) {
            if (!once) load(turn0, old);
#pragma unroll
            for (int e = 0; e < kHeld; ++e) {
                const int i = index_of(turn0, e);
                if (i - lane >= old) break;
                const bool equal = i < old && key[e] == border;
                const uint32_t word = __ballot_sync(0xffffffffu, i < old && (key[e] > border || (equal && i <= last)));
                const uint32_t same = by_list ? 0u : __ballot_sync(0xffffffffu, equal);
                if (lane == 0) {
                    words[e * 32 + warp] = word;
                    equals[e * 32 + warp] = same;
                }
            }
            __syncthreads();
            static_assert(kRound / 32 <= kSelectThreads, "a thread a word");
            const bool has_word = tid < kRound / 32 && turn0 + tid * 32 < old;
            uint32_t word = has_word ? words[tid] : 0u, total;
            if (!by_list) {  // the first `need` of the equal ones
                const uint32_t same = has_word ? equals[tid] : 0u, count = static_cast<uint32_t>(__popc(same));
                const uint32_t in_front = done_equal + block_scan(count, sm.warp_sum, &total) - count;
                uint32_t some = same;
                if (in_front + count > need) {
                    some = 0;
                    for (uint32_t k = in_front, rest = same; k < need; ++k) {
                        some |= rest & (0u - rest);
                        rest &= rest - 1u;
                    }
                }
                word |= some;
                if (has_word) words[tid] = word;
                done_equal += total;
            }
            const uint32_t count = static_cast<uint32_t>(__popc(word));
            const uint32_t in_front = done + block_scan(count, sm.warp_sum, &total) - count;
            if (has_word) before[tid] = in_front;
            done += total;
            // the weights themselves, where their integers do not tell (zeros, NaN), before any is written
            float odd[kHeld];
#pragma unroll
            for (int e = 0; e < kHeld; ++e) {
                const int i = index_of(turn0, e);
                odd[e] = i < old && (key[e] == 0u || key[e] == 0x80000000u) ? row[i] : 0.0f;
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kHeld; ++e) {
                const int i = index_of(turn0, e);
                if (i - lane >= old) break;
                const uint32_t w = words[e * 32 + warp];
                if (w >> lane & 1u) {
                    const uint32_t at = before[e * 32 + warp] + static_cast<uint32_t>(__popc(w & ((1u << lane) - 1u)));
                    keep[at] = i;
                    out[at] = key[e] == 0u || key[e] == 0x80000000u ? odd[e] : __uint_as_float(key[e] & 0x80000000u ? key[e] ^ 0x80000000u : ~key[e]);
                }
            }
            __syncthreads();
        }
    }
    // the keys that stay anyway; nothing behind them
    for (int t0 = chosen; t0 < left; t0 += kSelectThreads) {
        const int t = t0 + tid;
        const float v = t < left ? row[old + t - chosen] : 0.0f;
        __syncthreads();
        if (t < left) {
            keep[t] = old + t - chosen;
            out[t] = v;
        }
        __syncthreads();
    }
    for (int t = left + tid; t < budget; t += kSelectThreads) keep[t] = -1;
    for (int t = left + tid; t < capacity_out; t += kSelectThreads) out[t] = 0.0f;
}

// The place that key t comes from, by what evict_select wrote; -1: none that the sequence has (the two kernels are two launches, and what lies
// between them is the caller's memory: a place out of it is looked up in the table only where the table has it).
__host__ __device__ __forceinline__ int source_of(int kept, int t, int length) { return kept >= t && kept < length ? kept : -1; }

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
    const int length = paged::length_of(cache, b), left = min(length, budget);
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
            if (source_of(from[i], t, length) < 0 || (IN_PLACE && from[i] == t)) continue;
            const int page = paged::page_of(cache.table, cache, b, from[i]), page_to = target_page(t);
            if (page_to < 0) continue;
            to[i] = static_cast<long long>(paged::row_offset(cache, page_to, h, t) / 8 + piece);
            v[i] = page >= 0 ? __ldcs(data + paged::row_offset(cache, page, h, from[i]) / 8 + piece) : make_uint4(0u, 0u, 0u, 0u);  // (reads as zeros)
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
