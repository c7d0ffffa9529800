// Attention of few new tokens over a paged cache: decoding over caches that are short, or where each key is wanted once.
//
// The operation is attn_paged_kernel's (attn_paged.cuh), which spends some 12 us on its way through tensor memory however little there is to do, 5 more on
// joining cut blocks, and reads the keys a second time for their weights.  Here a cluster of up to 8 CTAs has one token's (or one
// sequence's) key head: each takes a range of the keys, dots them with the queries of the group on the FMA pipes, keeps the scores in shared
// memory, turns them into 2^(c s - m) with its own maximum m, adds up the values, and the CTAs join their parts through distributed shared
// memory.  What a key weighs is then there to be added to `mass`: one launch in all.
//
// A warp reads 16 keys at a time (of one page: pages are multiples of 16), D / 8 lanes a key, 16 bytes each; the queries stay in
// registers; the dot products of a load are reduced over the lanes by halves, heads first, so that GP heads take GP + 1 shuffles (GP > 1) and not 4 GP.
// Bound: the latency of a chain of loads (lengths, table, keys, values) for small calls, HBM for large ones.
#pragma once
#include "attnw_fused.cuh"
#include "paged.cuh"

namespace attnw {
namespace few {

constexpr int kThreads = 256;
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

__device__ __forceinline__ void unpack8(uint4 v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
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
__global__ void __launch_bounds__(kThreads)
attn_few_kernel(const __nv_bfloat16* Q, long long q_token, long long q_head, const __grid_constant__ paged::Cache cache, const __grid_constant__ Shape shape,
                const int* starts, float scale_log2e, __nv_bfloat16* O, float* lse, const float* mass, float* mass_out) {
    using L = Smem<D, GP>;
    constexpr int kLanes = D / 8;             // of a key
    constexpr int kRows = 32 / kLanes;         // keys of a load
    constexpr int kLoads = kUnit / kRows;      // of a unit
    constexpr int kHeadLanes = kLanes / GP > 0 ? kLanes / GP : 1;  // lanes that end up with the same sum
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
    int b, t0, t1, end;
    if (WEIGH) {
        b = item / cache.kv_heads;
        const int s0 = starts[b];
        end = starts[b + 1];
        t0 = min(max(s0, 0), shape.tokens);
        t1 = min(max(end, 0), shape.tokens);
    } else {
        paged::sample_starts(&samples, starts, cache.sequences, kThreads);
        __syncthreads();
        t0 = item / cache.kv_heads;
        b = paged::owner_of(&samples, starts, cache.sequences, t0, &end);
        if (b < 0) return;  // (all CTAs of the cluster)
        t1 = t0 + 1;
    }
    const int length = paged::length_of(cache, b);
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
    const int column = lane % kLanes, of_load = lane / kLanes;  // this lane's 8 features, and its key of a load
    // The pages of this warp's first 32 units, one a lane; -1: none that the cache has.
    const int my_first = unit0 + warp + kWarps * lane;
    const int page_mine = my_first < unit1 ? paged::page_of(cache.table, cache, b, my_first * kUnit) : -1;
    // A unit's rows, as 16-byte vectors: zeros where there is no key that the token sees, or no page.
    auto fetch = [&](const __nv_bfloat16* data, int i, int seen, uint4 (&v)[kLoads]) {
        const int unit = unit0 + warp + kWarps * i;
        const int page = i < 32 ? __shfl_sync(0xffffffffu, page_mine, i & 31) : unit < unit1 ? paged::page_of(cache.table, cache, b, unit * kUnit) : -1;
        const __nv_bfloat16* rows = data + (page >= 0 ? paged::row_offset(cache, page, h, unit * kUnit) : 0) + column * 8;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            const int row = n * kRows + of_load;
            v[n] = page >= 0 && unit * kUnit + row < seen ? __ldcs(reinterpret_cast<const uint4*>(rows + static_cast<size_t>(row) * D)) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    const int my_units = (unit1 - unit0 - warp + kWarps - 1) / kWarps;  // of this warp (0 or less: none)
    const float c2 = scale_log2e;

    for (int t = t0; t < t1; ++t) {
        const long long seen_by = static_cast<long long>(length) - (static_cast<long long>(end) - t) + 1;
        const int seen = static_cast<int>(min(max(seen_by, 0ll), static_cast<long long>(length)));
        float q[GP][8];
#pragma unroll
        for (int g = 0; g < GP; ++g) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (g < shape.group) v = *reinterpret_cast<const uint4*>(Q + t * q_token + (h * shape.group + g) * q_head + column * 8);
            unpack8(v, q[g]);
        }
        // ---- scores, and their maximum ----
        const int head = head_of<GP, kLanes>(lane);
        float top = -3.0e38f;
        for (int i = 0; i < my_units; ++i) {
            uint4 v[kLoads];
            fetch(cache.K, i, seen, v);
            const int at = (warp + kWarps * i) * kUnit;  // the unit's first key, from key0 on
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                float k[8], dot[GP];
                unpack8(v[n], k);
#pragma unroll
                for (int g = 0; g < GP; ++g) {
                    uint64_t sum = ptx::mul2(ptx::pack2(q[g][0], q[g][1]), ptx::pack2(k[0], k[1]));
#pragma unroll
                    for (int e = 2; e < 8; e += 2) sum = ptx::fma2(ptx::pack2(q[g][e], q[g][e + 1]), ptx::pack2(k[e], k[e + 1]), sum);
                    float a, b2;
                    ptx::unpack2(sum, a, b2);
                    dot[g] = a + b2;
                }
                const float z = reduce_heads<GP, kLanes>(dot, lane);
                const int key = at + n * kRows + of_load;
                const float s = key0 + key < seen ? z * c2 : __int_as_float(0xff800000);
                top = fmaxf(top, s);
                if (lane % kHeadLanes == 0) scores[key * GP + head] = s;
            }
        }
        // the first values are on their way while the scores are turned into weights
        uint4 first_v[kLoads];
        if (my_units > 0) fetch(cache.V, 0, seen, first_v);
        if (kRows > 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        if (kRows > 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        if (lane < kLanes && lane % kHeadLanes == 0) of_warps[warp * GP + head] = top;
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
        float o[GP][8] = {};
        for (int i = 0; i < my_units; ++i) {
            uint4 v[kLoads];
            if (i == 0) {
#pragma unroll
                for (int n = 0; n < kLoads; ++n) v[n] = first_v[n];
            } else {
                fetch(cache.V, i, seen, v);
            }
            const int at = (warp + kWarps * i) * kUnit;
#pragma unroll
            for (int n = 0; n < kLoads; ++n) {
                float x[8];
                unpack8(v[n], x);
                const float* p = scores + (at + n * kRows + of_load) * GP;
#pragma unroll
                for (int g = 0; g < GP; ++g) {
                    const uint64_t pp = ptx::pack2(p[g], p[g]);
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        ptx::unpack2(ptx::fma2(pp, ptx::pack2(x[e], x[e + 1]), ptx::pack2(o[g][e], o[g][e + 1])), o[g][e], o[g][e + 1]);
                }
            }
        }
#pragma unroll
        for (int g = 0; g < GP; ++g)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (kRows > 1) o[g][e] += __shfl_xor_sync(0xffffffffu, o[g][e], 16);
                if (kRows > 2) o[g][e] += __shfl_xor_sync(0xffffffffu, o[g][e], 8);
            }
        if (lane < kLanes)
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                float4* dst = reinterpret_cast<float4*>(part + (warp * GP + g) * D + column * 8);
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
