// Attention of few new tokens over a paged cache: decoding over caches that are short, or where each key is wanted once.
//
// The operation is attn_paged_kernel's (attn_paged.cuh), which spends some 12 us on its way through tensor memory however little there is to do, 8 more
// where blocks are cut and joined, and reads the keys a second time for their weights.  Here a cluster of up to 8 CTAs has one token's (or one
// sequence's) key head: each takes a range of the keys, dots them with the queries of the group on the FMA pipes, keeps the scores in shared
// memory, turns them into 2^(c s - m) with its own maximum m, adds up the values, and the CTAs join their parts through distributed shared
// memory.  What a key weighs is then there to be added to `mass`: one launch in all.
//
// A warp reads 8 or 16 keys at a time (of one page: pages are multiples of 16), four 16-byte vectors a lane, and the next ones while it works on
// them; the queries stay in registers; the dot products are reduced over a key's lanes by halves, heads first, so that 4 heads over 8 lanes
// take 4 shuffles and not 12.
// Bound: the latency of a chain of loads (lengths, table, keys, values) for small calls (one token over 500 keys, 12 heads, d = 64: 5.2 us); for larger
// ones each warp's own instructions, of which a key takes as many as there are heads (8 sequences of up to 4096 keys, 32 heads on 8, d = 128, with
// weights: 35.3 us, where the 65 MB take 9.9 and half of the CTAs have long been done: a cluster is as slow as the longest sequence).  A ring of
// asynchronous copies with three turns on their way helped one head a group (30 -> 25.5 us), and cost four (16 tokens over 1000 keys 19.4 -> 21.7).
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

// Item: without weights (token, key head), with weights (sequence, key head) and its tokens one after the other.
template <int D, int GP, bool WEIGH>
__global__ void __launch_bounds__(kThreads, 1)
attn_few_kernel(const __nv_bfloat16* Q, long long q_token, long long q_head, const __grid_constant__ paged::Cache cache, const __grid_constant__ Shape shape,
                const int* starts, float scale_log2e, __nv_bfloat16* O, float* lse, const float* mass, float* mass_out) {
    using L = Smem<D, GP>;
    constexpr int kKeyLanes = GP <= 4 ? 8 : D / 8, kVecs = D / 8 / kKeyLanes;  // keys: lanes of a key, vectors of a lane
    constexpr int kRowLanes = D / 8;                                            // values: lanes of a key
    constexpr int kKeys = 4 * (32 / kRowLanes);                                  // that a warp takes at a time, four vectors a lane
    constexpr int kTurns = kUnit / kKeys;                                        // of a unit
    constexpr int kHeadLanes = kKeyLanes / GP > 0 ? kKeyLanes / GP : 1;          // lanes that end up with the same sum
    static_assert(kKeys * kKeyLanes * kVecs == 32 * 4 && kKeyLanes >= GP, "four vectors a lane");
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
    // The pages of this warp's first 32 units, one a lane; -1: none that the cache has.
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
    const float c2 = scale_log2e;

    for (int t = t0; t < t1; ++t) {
        const long long seen_by = static_cast<long long>(length) - (static_cast<long long>(end) - t) + 1;
        const int seen = static_cast<int>(min(max(seen_by, 0ll), static_cast<long long>(length)));
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
        uint4 next[4];
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
        // the first values are on their way while the scores are turned into weights
        if (my_turns > 0) fetch(cache.V, 0, seen, kRowLanes, next);
#pragma unroll
        for (int o = 16; o >= kKeyLanes; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane < kKeyLanes && lane % kHeadLanes == 0) of_warps[warp * GP + head] = top;
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
            const float M = factors(g, &sum), inv = sum > 0.0f ? 1.0f / sum : 0.0f;
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
                sum > 0.0f ? 0.69314718055994531f * (M + ptx::lg2_approx(sum)) : __int_as_float(0xff800000);
        }
        if (WEIGH) {
            float f[GP];
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                float sum;
                const float M = factors(g, &sum);
                f[g] = sum > 0.0f && g < shape.group ? ptx::ex2_approx(stats[rank * GP + g].x - M) / sum : 0.0f;
            }
            for (int i = tid; i < (unit1 - unit0) * kUnit; i += kThreads) {
                float w = 0.0f;
#pragma unroll
                for (int g = 0; g < GP; ++g) w = fmaf(scores[i * GP + g], f[g], w);
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
