// Attention of few new tokens over a paged cache: decoding over caches that are short, or where each key is wanted once.
//
// The operation is attn_paged_kernel's (attn_paged.cuh), which spends some 12 us on its way through tensor memory however little there is to do, 8 more
// where blocks are cut and joined, and reads the keys a second time for their weights.  Here a cluster of up to 8 CTAs has one token's (or one
// sequence's) key head: each takes a range of the keys, multiplies them with the queries of the group, keeps the scores in shared
// memory, turns them into 2^(c s - m) with its own maximum m, adds up the values, and the CTAs join their parts through distributed shared
// memory.  What a key weighs is then there to be added to `mass`: one launch in all.
//
// Groups of 3 to 8 heads: a warp takes 16 keys (of one page: pages are multiples of 16) at a time, and both products are m16n8k16 products of a warp, whose
// operands are 16-byte vectors just as they were loaded: neither the order of the features of a score nor that of the keys of a sum matters, so a lane's
// vector is its share of the operand.  (tcgen05 wants its operands in shared memory and 64 rows at least, and its results take a way of 12 us.)  One or two
// heads: FMA pipes, four vectors a lane and turn, the dot products reduced over a key's lanes by halves, heads first.  Eight heads' products for one
// head's cost more than they save: one token over 500 keys, 12 heads on 12, d = 64 the same, 8 tokens over 4000 27 us -> 30.
// us per call before (FMA pipes for all) -> now: 32 heads on 8, 8 tokens over 4095 keys 35 -> 30.9, 16 over 1000 19.6 -> 16.9, with weights 21.6 -> 19.6,
// 64 heads on 8, 8 over 4000 71 -> 46, with weights 81 -> 57; 14 heads on 2, d = 64, 32 over 2000 19.3 -> 13.3.
// Bound: the latency of a chain of loads (lengths, table, keys, values) for small calls (one token over 500 keys, 12 heads, d = 64: 5.2 us); for larger
// ones the loads that a warp has on their way, 4 KB (8 sequences of up to 4096 keys, 32 heads on 8, d = 128, with weights: 30.6 us, where the 65 MB take 9.9
// and half of the CTAs have long been done: a cluster is as slow as the longest sequence).  More clusters than fit at once were slower at every length.
#pragma once
#include "attnw_fused.cuh"
#include "paged.cuh"

namespace attnw {
namespace few {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kUnit = 16;          // keys that a warp takes at a time
constexpr int kMaxCluster = 8;
constexpr int kMaxScores = 12288;  // floats of scores that a CTA keeps

struct Shape {
    int tokens, heads, group;
    int cluster;    // CTAs of an item
    int max_keys;   // that a CTA may have, a multiple of kUnit
    int turns;      // with weights: tokens of a sequence, at most; those with more are attn_paged_kernel's
};

template <int D, int GP>
struct Smem {
    static constexpr int kPartOff = 0;                                   // float [warps][GP][D]: the warps' parts of O
    static constexpr int kStatOff = kPartOff + kWarps * GP * D * 4;       // float2 [kMaxCluster][GP]: (maximum, sum) of each CTA
    static constexpr int kWarpOff = kStatOff + kMaxCluster * GP * 8;      // float [2][warps][GP]: the warps' maxima and sums
    static constexpr int kOutOff = kWarpOff + 2 * kWarps * GP * 4;        // float [GP][D]: this CTA's O, for its peers
    static constexpr int kScoreOff = kOutOff + GP * D * 4;                // float [keys][GP], and with weights float [keys]
    static constexpr int bytes(int max_keys, bool weigh) { return kScoreOff + max_keys * (GP + (weigh ? 1 : 0)) * 4; }
};

// Eight bfloat16 as four pairs of float32.
__device__ __forceinline__ void unpack_pairs(uint4 v, uint64_t* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = ptx::pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}

// x[GP], one part in each of LANES neighbouring lanes -> in each lane the whole sum of one: head_of(lane).
template <int GP, int LANES>
__device__ __forceinline__ float reduce_heads(float (&x)[GP], int lane) {
    int n = GP;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        if (n > 1) {
            n >>= 1;
            const bool upper = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < GP / 2; ++i) {
                if (i >= n) break;
                const float send = upper ? x[i] : x[i + n], keep = upper ? x[i + n] : x[i];
                x[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
            }
        } else {
            x[0] += __shfl_xor_sync(0xffffffffu, x[0], o);
        }
    }
    return x[0];
}
template <int GP, int LANES>
__device__ __forceinline__ int head_of(int lane) {
    int head = 0, n = GP;
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1)
        if (n > 1) {
            n >>= 1;
            head += (lane & o) != 0 ? n : 0;
        }
    return head;
}

// D (16 x 8, float32) += A (16 x 16) B (16 x 8), bfloat16, by one warp.  Lane (r, c) = (lane / 4, lane % 4) has of A rows r and r + 8 at k = 2c, 2c + 1
// (a[0], a[1]) and 2c + 8, 2c + 9 (a[2], a[3]), of B column r at the same k (b0, b1), of D rows r (d[0], d[1]) and r + 8 (d[2], d[3]) in columns 2c, 2c + 1.
__device__ __forceinline__ void multiply(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Item: without weights (token, key head), with weights (sequence, key head) and its tokens one after the other.
template <int D, int GP, bool WEIGH>
__global__ void __launch_bounds__(kThreads, 1)
attn_few_kernel(const __nv_bfloat16* Q, long long q_token, long long q_head, const __grid_constant__ paged::Cache cache, const __grid_constant__ Shape shape,
                const int* starts, float scale_log2e, __nv_bfloat16* O, float* lse, const float* mass, float* mass_out) {
    using L = Smem<D, GP>;
    constexpr bool kTensor = GP >= 4;
    // FMA pipes:
    constexpr int kKeyLanes = 8, kVecs = D / 8 / kKeyLanes;  // keys: lanes of a key, vectors of a lane
    constexpr int kRowLanes = D / 8;                                            // values: lanes of a key
    constexpr int kKeys = 4 * (32 / kRowLanes);                                  // that a warp takes at a time, four vectors a lane
    constexpr int kTurns = kUnit / kKeys;                                        // of a unit
    constexpr int kHeadLanes = kKeyLanes / GP > 0 ? kKeyLanes / GP : 1;          // lanes that end up with the same sum
    static_assert(kKeys * kKeyLanes * kVecs == 32 * 4 && kKeyLanes >= GP, "four vectors a lane");
    // Tensor cores:
    constexpr int kSteps = D / 32;   // of a unit's keys: 32 features, two vectors a lane
    constexpr int kHalves = D / 64;  // of a unit's values: 64 features, four vectors a lane
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ paged::Samples samples;
    float* part = reinterpret_cast<float*>(smem + L::kPartOff);
    float2* stats = reinterpret_cast<float2*>(smem + L::kStatOff);
    float* of_warps = reinterpret_cast<float*>(smem + L::kWarpOff);
    float* out = reinterpret_cast<float*>(smem + L::kOutOff);
    float* scores = reinterpret_cast<float*>(smem + L::kScoreOff);
    float* weights = scores + shape.max_keys * GP;
    const int tid = static_cast<int>(threadIdx.x), warp = tid >> 5, lane = tid & 31;
    const int S = shape.cluster, rank = S > 1 ? static_cast<int>(ptx::cluster_ctarank()) : 0;
    const int item = static_cast<int>(blockIdx.x) / S, h = item % cache.kv_heads;
    auto cluster_sync = [&]() {
        if (S > 1) {
            ptx::cluster_arrive_release();
            ptx::cluster_wait_acquire();
        } else {
            __syncthreads();
        }
    };
    ptx::grid_dependency_wait();
    int b, t0, t1, end, length;
    if (WEIGH) {
        b = item / cache.kv_heads;
        const int s0 = starts[b];
        end = starts[b + 1];
        length = paged::length_of(cache, b);
        t0 = min(max(s0, 0), shape.tokens);
        t1 = min(max(end, 0), shape.tokens);
        if (t1 - t0 > shape.turns) return;  // (all CTAs of the cluster)
    } else {
        t0 = item / cache.kv_heads;
        t1 = t0 + 1;
        if (cache.sequences <= 32) {  // a lane a sequence: one latency for all that is asked
            const bool there = lane < cache.sequences;
            const int from = there ? starts[lane] : 0, to = there ? starts[lane + 1] : 0, of_lane = there ? paged::length_of(cache, lane) : 0;
            const uint32_t owners = __ballot_sync(0xffffffffu, there && from <= t0 && t0 < to);
            if (owners == 0u) return;  // (all CTAs of the cluster)
            b = 31 - __clz(owners);
            end = __shfl_sync(0xffffffffu, to, b);
            length = __shfl_sync(0xffffffffu, of_lane, b);
        } else {
            paged::sample_starts(&samples, starts, cache.sequences, kThreads);
            __syncthreads();
            b = paged::owner_of(&samples, starts, cache.sequences, t0, &end);
            if (b < 0) return;
            length = paged::length_of(cache, b);
        }
    }
    const int capacity = cache.table_width << cache.page_shift;
    const size_t mass_row = (static_cast<size_t>(b) * cache.kv_heads + h) * capacity;
    // This CTA's units of the sequence's keys, the same for all its tokens.
    const int units = (length + kUnit - 1) / kUnit, unit0 = static_cast<int>(static_cast<long long>(units) * rank / S),
              unit1 = static_cast<int>(static_cast<long long>(units) * (rank + 1) / S), key0 = unit0 * kUnit;
    if (WEIGH) {
        for (int i = tid; i < (unit1 - unit0) * kUnit; i += kThreads) weights[i] = 0.0f;
        if (mass != mass_out)  // what no token sees
            for (int j = (t1 > t0 ? length : 0) + rank * kThreads + tid; j < capacity; j += S * kThreads) mass_out[mass_row + j] = mass[mass_row + j];
    }
    // (A peer's shared memory is written to only when the peer runs: the other half of this is in front of the first such store.)
    if (S > 1 && t0 < t1) ptx::cluster_arrive_relaxed();
    // The pages of this warp's first 32 units, one a lane; -1: none that the cache has.  (kMaxScores allows it 24.  Without the question for more, compiled
    // otherwise, calls with weights took longer: 16 sequences of 256 keys 9.8 -> 10.2 us, 8 of up to 4096 31.1 -> 31.9.)
    const int my_first = unit0 + warp + kWarps * lane;
    const int page_mine = my_first < unit1 ? paged::page_of(cache.table, cache, b, my_first * kUnit) : -1;
    // Turn i of this warp: kKeys keys as four vectors a lane, `lanes` lanes a key; zeros where there is no key that the token sees, or no page.
    auto fetch = [&](const __nv_bfloat16* data, int i, int seen, int lanes, uint4 (&v)[4]) {
        const int n = i / kTurns, unit = unit0 + warp + kWarps * n;
        const int page = n < 32 ? __shfl_sync(0xffffffffu, page_mine, n & 31) : unit < unit1 ? paged::page_of(cache.table, cache, b, unit * kUnit) : -1;
        const int key = unit * kUnit + i % kTurns * kKeys;
        const __nv_bfloat16* rows = data + (page >= 0 ? paged::row_offset(cache, page, h, key) : 0);
        const int vecs = D / 8 / lanes;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int row = x / vecs * (32 / lanes) + lane / lanes, column = x % vecs * lanes + lane % lanes;
            v[x] = page >= 0 && key + row < seen ? __ldcs(reinterpret_cast<const uint4*>(rows + row * D + column * 8)) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    const int my_turns = max(0, unit1 - unit0 - warp + kWarps - 1) / kWarps * kTurns;  // of this warp
    auto turn_begin = [&](int i) { return (warp + kWarps * (i / kTurns)) * kUnit + i % kTurns * kKeys; };  // its first key, from key0 on
    const int my_units = max(0, unit1 - unit0 - warp + kWarps - 1) / kWarps;  // of this warp
    const int r = lane >> 2, c = lane & 3;
    // Unit i of this warp: its page (below 0: none), and the first of its rows.
    auto rows_of = [&](const __nv_bfloat16* data, int i, int* key) {
        const int unit = unit0 + warp + kWarps * i;
        const int page = i < 32 ? __shfl_sync(0xffffffffu, page_mine, i & 31) : unit < unit1 ? paged::page_of(cache.table, cache, b, unit * kUnit) : -1;
        *key = unit * kUnit;
        return page >= 0 ? data + paged::row_offset(cache, page, h, *key) : nullptr;
    };
    auto vector_of = [&](const __nv_bfloat16* rows, bool there, int at) {
        return rows != nullptr && there ? __ldcs(reinterpret_cast<const uint4*>(rows + at)) : make_uint4(0u, 0u, 0u, 0u);
    };
    // Keys r and r + 8 of the unit, features 8c ... 8c + 7 of each 32; zeros where there is no key that the token sees.
    auto fetch_keys = [&](int i, int seen, uint4 (&v)[2 * kSteps]) {
        int key;
        const __nv_bfloat16* rows = rows_of(cache.K, i, &key);
#pragma unroll
        for (int x = 0; x < 2 * kSteps; ++x) v[x] = vector_of(rows, key + r + (x & 1) * 8 < seen, (r + (x & 1) * 8) * D + (x >> 1) * 32 + c * 8);
    };
    // Values c, c + 4, c + 8, c + 12 of the unit, features 8r ... 8r + 7 of 64.
    auto fetch_values = [&](int i, int half, int seen, uint4 (&v)[4]) {
        int key;
        const __nv_bfloat16* rows = rows_of(cache.V, i, &key);
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = vector_of(rows, key + c + 4 * x < seen, (c + 4 * x) * D + half * 64 + r * 8);
    };
    // The values `ahead` units behind unit i of that half, all units of one half in front of the next.
    auto fetch_next = [&](int i, int half, int ahead, int seen, uint4 (&v)[4]) {
        int n = i + ahead, y = half;
        while (n >= my_units && y < kHalves) {
            n -= my_units;
            ++y;
        }
        if (y < kHalves) fetch_values(n, y, seen, v);
    };
    auto unit_begin = [&](int i) { return (warp + kWarps * i) * kUnit; };  // its first key, from key0 on
    const float c2 = scale_log2e;

    for (int t = t0; t < t1; ++t) {
        const long long seen_by = static_cast<long long>(length) - (static_cast<long long>(end) - t) + 1;
        const int seen = static_cast<int>(min(max(seen_by, 0ll), static_cast<long long>(length)));
        uint4 next[4], values[2][4];  // (of either path; loaded in front of the weights)
        if constexpr (kTensor) {
            uint4 q[kSteps];  // head r, features 8c ... 8c + 7 of each 32
#pragma unroll
            for (int x = 0; x < kSteps; ++x)
                q[x] = r < shape.group ? *reinterpret_cast<const uint4*>(Q + t * q_token + (h * shape.group + r) * q_head + x * 32 + c * 8) : make_uint4(0u, 0u, 0u, 0u);
            // ---- scores, and their maximum: keys are the rows, heads the columns; the order of the features is the same for both ----
            float top[2] = {-3.0e38f, -3.0e38f};  // of heads 2c, 2c + 1
            uint4 keys[2 * kSteps];
            if (my_units > 0) fetch_keys(0, seen, keys);
            for (int i = 0; i < my_units; ++i) {
                uint4 v[2 * kSteps];
#pragma unroll
                for (int x = 0; x < 2 * kSteps; ++x) v[x] = keys[x];
                if (i + 1 < my_units) fetch_keys(i + 1, seen, keys);
                float z[2][4] = {};  // (two sums: half the chain)
#pragma unroll
                for (int x = 0; x < kSteps; ++x) {
                    multiply(z[0], v[2 * x].x, v[2 * x + 1].x, v[2 * x].y, v[2 * x + 1].y, q[x].x, q[x].y);
                    multiply(z[1], v[2 * x].z, v[2 * x + 1].z, v[2 * x].w, v[2 * x + 1].w, q[x].z, q[x].w);
                }
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int key = unit_begin(i) + r + (y >> 1) * 8, head = 2 * c + (y & 1);
                    const float s = key0 + key < seen ? (z[0][y] + z[1][y]) * c2 : __int_as_float(0xff800000);
                    top[y & 1] = fmaxf(top[y & 1], s);
                    if (head < GP) scores[key * GP + head] = s;
                }
            }
            // the first values are on their way while the scores are turned into weights
            if (my_units > 0) fetch_values(0, 0, seen, values[0]);
            if (my_units > 0) fetch_next(0, 0, 1, seen, values[1]);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int o = 16; o >= 4; o >>= 1) top[y] = fmaxf(top[y], __shfl_xor_sync(0xffffffffu, top[y], o));
                if (r == 0 && 2 * c + y < GP) of_warps[warp * GP + 2 * c + y] = top[y];
            }
        } else {
            uint64_t q[GP][4 * kVecs];  // pairs of features
#pragma unroll
            for (int g = 0; g < GP; ++g)
#pragma unroll
                for (int i = 0; i < kVecs; ++i) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (g < shape.group)
                        v = *reinterpret_cast<const uint4*>(Q + t * q_token + (h * shape.group + g) * q_head + (i * kKeyLanes + lane % kKeyLanes) * 8);
                    unpack_pairs(v, q[g] + 4 * i);
                }
            // ---- scores, and their maximum ----
            const int head = head_of<GP, kKeyLanes>(lane);
            float top = -3.0e38f;
            if (my_turns > 0) fetch(cache.K, 0, seen, kKeyLanes, next);
            for (int i = 0; i < my_turns; ++i) {
                uint4 v[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = next[x];
                if (i + 1 < my_turns) fetch(cache.K, i + 1, seen, kKeyLanes, next);
                const int at = turn_begin(i) + lane / kKeyLanes;
#pragma unroll
                for (int x = 0; x < 4; x += kVecs) {
                    uint64_t k[4 * kVecs];
#pragma unroll
                    for (int y = 0; y < kVecs; ++y) unpack_pairs(v[x + y], k + 4 * y);
                    float dot[GP];
#pragma unroll
                    for (int g = 0; g < GP; ++g) {
                        uint64_t sum = ptx::mul2(q[g][0], k[0]);
#pragma unroll
                        for (int e = 1; e < 4 * kVecs; ++e) sum = ptx::fma2(q[g][e], k[e], sum);
                        float lo, hi;
                        ptx::unpack2(sum, lo, hi);
                        dot[g] = lo + hi;
                    }
                    const int key = at + x / kVecs * (32 / kKeyLanes);
                    const float z = reduce_heads<GP, kKeyLanes>(dot, lane), s = key0 + key < seen ? z * c2 : __int_as_float(0xff800000);
                    top = fmaxf(top, s);
                    if (lane % kHeadLanes == 0) scores[key * GP + head] = s;
                }
            }
            // (as above)
            if (my_turns > 0) fetch(cache.V, 0, seen, kRowLanes, next);
#pragma unroll
            for (int o = 16; o >= kKeyLanes; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (lane < kKeyLanes && lane % kHeadLanes == 0) of_warps[warp * GP + head] = top;
        }
        __syncthreads();
        // ---- weights relative to this CTA's maxima, and their sums ----
        float m[GP], l[GP];
#pragma unroll
        for (int g = 0; g < GP; ++g) {
            m[g] = of_warps[g];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) m[g] = fmaxf(m[g], of_warps[w * GP + g]);
            l[g] = 0.0f;
        }
        for (int i = tid; i < (unit1 - unit0) * kUnit; i += kThreads) {
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                const float e = ptx::ex2_approx(scores[i * GP + g] - m[g]);  // (m is finite: a key that is not seen gets zero)
                scores[i * GP + g] = e;
                l[g] += e;
            }
        }
#pragma unroll
        for (int g = 0; g < GP; ++g)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) l[g] += __shfl_xor_sync(0xffffffffu, l[g], o);
        if (lane == 0)
#pragma unroll
            for (int g = 0; g < GP; ++g) of_warps[(kWarps + warp) * GP + g] = l[g];
        __syncthreads();
        if (S > 1 && t == t0) ptx::cluster_wait_acquire();
        if (tid < GP) {  // to all CTAs
            float mine = of_warps[tid], sum = 0.0f;
            for (int w = 1; w < kWarps; ++w) mine = fmaxf(mine, of_warps[w * GP + tid]);
            for (int w = 0; w < kWarps; ++w) sum += of_warps[(kWarps + w) * GP + tid];
            for (int c = 0; c < S; ++c) {
                if (S > 1)
                    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(ptx::map_to_cta(ptx::smem_u32(&stats[rank * GP + tid]), static_cast<uint32_t>(c))),
                                 "f"(mine), "f"(sum)
                                 : "memory");
                else
                    stats[tid] = make_float2(mine, sum);
            }
        }
        // ---- values ----
        if constexpr (kTensor) {
            // Rows 0 ... 7 of the first operand are the heads' weights rounded to bfloat16, rows 8 ... 15 what the rounding left over, rounded: the weights count
            // with 16 bits, at no cost, as there are at most 8 heads.  Column n of product j is feature 8n + j, so that a lane's vectors are its columns.
            // 64 features at a time (the sums of 128 and their vectors do not fit the registers).
#pragma unroll 1
            for (int y = 0; y < kHalves; ++y) {
                float o[8][4] = {};
                auto add = [&](int i, uint4 (&v)[4]) {
                    uint32_t w[2], left[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const float* p = scores + (unit_begin(i) + c + 8 * x) * GP + r;
                        const float w0 = r < GP ? p[0] : 0.0f, w1 = r < GP ? p[4 * GP] : 0.0f;
                        w[x] = ptx::pack_bf16x2(w0, w1);
                        left[x] = ptx::pack_bf16x2(w0 - __uint_as_float(w[x] << 16), w1 - __uint_as_float(w[x] & 0xffff0000u));
                    }
                    const uint32_t word[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w}, {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t which = j & 1 ? 0x7632 : 0x5410;
                        multiply(o[j], w[0], left[0], w[1], left[1], __byte_perm(word[0][j >> 1], word[1][j >> 1], which),
                                 __byte_perm(word[2][j >> 1], word[3][j >> 1], which));
                    }
                };
                for (int i = 0; i < my_units; ++i) {  // two of them are on their way, of this half or the next
                    uint4 v[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) v[x] = values[0][x], values[0][x] = values[1][x];
                    fetch_next(i, y, 2, seen, values[1]);
                    add(i, v);
                }
                if (r < GP)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {  // columns 2c and 2c + 1
                        float* dst = part + (warp * GP + r) * D + y * 64 + c * 16 + x * 4;
                        const int j = x % 2 * 4, e = x / 2;
                        *reinterpret_cast<float4*>(dst) = make_float4(o[j][e] + o[j][e + 2], o[j + 1][e] + o[j + 1][e + 2], o[j + 2][e] + o[j + 2][e + 2],
                                                                      o[j + 3][e] + o[j + 3][e + 2]);
                    }
            }
        } else {
            uint64_t o2[GP][4];
#pragma unroll
            for (int g = 0; g < GP; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) o2[g][e] = 0ull;
            for (int i = 0; i < my_turns; ++i) {
                uint4 v[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = next[x];
                if (i + 1 < my_turns) fetch(cache.V, i + 1, seen, kRowLanes, next);
                const float* p = scores + (turn_begin(i) + lane / kRowLanes) * GP;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    uint64_t y[4];
                    unpack_pairs(v[x], y);
#pragma unroll
                    for (int g = 0; g < GP; ++g) {
                        const float w = p[x * (32 / kRowLanes) * GP + g];
#pragma unroll
                        for (int e = 0; e < 4; ++e) o2[g][e] = ptx::fma2(ptx::pack2(w, w), y[e], o2[g][e]);
                    }
                }
            }
            float o[GP][8];
#pragma unroll
            for (int g = 0; g < GP; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e % 2 == 0) ptx::unpack2(o2[g][e / 2], o[g][e], o[g][e + 1]);
                }
#pragma unroll
            for (int g = 0; g < GP; ++g)
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int x = 16; x >= kRowLanes; x >>= 1) o[g][e] += __shfl_xor_sync(0xffffffffu, o[g][e], x);
            if (lane < kRowLanes)
#pragma unroll
                for (int g = 0; g < GP; ++g) {
                    float4* dst = reinterpret_cast<float4*>(part + (warp * GP + g) * D + lane * 8);
                    dst[0] = make_float4(o[g][0], o[g][1], o[g][2], o[g][3]);
                    dst[1] = make_float4(o[g][4], o[g][5], o[g][6], o[g][7]);
                }
        }
        __syncthreads();
        for (int i = tid; i < GP * D; i += kThreads) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) sum += part[w * GP * D + i];
            out[i] = sum;
        }
        cluster_sync();
        // ---- what the CTAs have, joined: O = sum_c 2^(m_c - M) O_c / sum_c 2^(m_c - M) l_c ----
        auto factors = [&](int g, float* of_sum) {  // M, and 1 / the sum
            float M = -3.0e38f, sum = 0.0f;
            for (int c = 0; c < S; ++c) M = fmaxf(M, stats[c * GP + g].x);
            for (int c = 0; c < S; ++c) sum += stats[c * GP + g].y * ptx::ex2_approx(stats[c * GP + g].x - M);
            *of_sum = sum;
            return M;
        };
        for (int i = 2 * (rank * kThreads + tid); i < shape.group * D; i += 2 * S * kThreads) {
            const int g = i / D;
            float sum;
            const float M = factors(g, &sum), inv = sum != 0.0f ? 1.0f / sum : 0.0f;  // (not a number where a score was none)
            float a = 0.0f, b2 = 0.0f;
            for (int c = 0; c < S; ++c) {
                const float f = ptx::ex2_approx(stats[c * GP + g].x - M) * inv;
                float x, y;
                if (S > 1)
                    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];"
                                 : "=f"(x), "=f"(y)
                                 : "r"(ptx::map_to_cta(ptx::smem_u32(&out[i]), static_cast<uint32_t>(c)))
                                 : "memory");
                else
                    x = out[i], y = out[i + 1];
                a = fmaf(x, f, a);
                b2 = fmaf(y, f, b2);
            }
            *reinterpret_cast<uint32_t*>(O + (static_cast<size_t>(t) * shape.heads + h * shape.group) * D + i) = ptx::pack_bf16x2(a, b2);
        }
        if (lse && rank == 0 && tid < shape.group) {
            float sum;
            const float M = factors(tid, &sum);
            lse[static_cast<size_t>(t) * shape.heads + h * shape.group + tid] =
                sum != 0.0f ? 0.69314718055994531f * (M + ptx::lg2_approx(sum)) : __int_as_float(0xff800000);
        }
        if (WEIGH) {
            float f[GP];
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                float sum;
                const float M = factors(g, &sum);
                f[g] = sum != 0.0f ? ptx::ex2_approx(stats[rank * GP + g].x - M) / sum : 0.0f;
            }
            // (only what is a weight: a head of the group, of a key that the token sees)
            for (int i = tid; i < (unit1 - unit0) * kUnit && key0 + i < seen; i += kThreads) {
                float w = 0.0f;
#pragma unroll
                for (int g = 0; g < GP; ++g)
                    if (g < shape.group) w = fmaf(scores[i * GP + g], f[g], w);
                weights[i] += w;
            }
        }
        if (S > 1 || t + 1 < t1) cluster_sync();  // nobody reads a peer's, or this token's, any more
    }
    if (WEIGH && t1 > t0)
        for (int i = tid; i < (unit1 - unit0) * kUnit && key0 + i < length; i += kThreads) mass_out[mass_row + key0 + i] = mass[mass_row + key0 + i] + weights[i];
}

}  // namespace few
}  // namespace attnw
