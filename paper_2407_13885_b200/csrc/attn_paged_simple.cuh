// Attention of new tokens over a paged cache, one warp a (token, query head): the plain form of the operation.
//
//     O[t, h] = sum_j p_j V_j,   p_j = exp(z_j - lse),   z_j = scale * Q[t, h] . K_j,   j <= at(t),
// where at(t) is the token's own place in its sequence.  Online form: running maximum and sum.  No visible key: O = 0, lse = -inf.
#pragma once
#include <cfloat>

#include "paged.cuh"

namespace attnw {
namespace pa0 {

constexpr int kWarps = 4;

template <int D>
__global__ void __launch_bounds__(kWarps * 32)
attn_kernel(const __nv_bfloat16* Q, long long q_token, long long q_head, paged::Cache cache, const int* starts, __nv_bfloat16* O, float* lse,
            int tokens, int heads, float scale) {
    __shared__ paged::Samples samples;
    __shared__ float q_row[kWarps][D];
    ptx::grid_dependency_wait();
    paged::sample_starts(&samples, starts, cache.sequences, kWarps * 32);
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long id = static_cast<long long>(blockIdx.x) * kWarps + warp;
    const int t = static_cast<int>(id / heads), h = static_cast<int>(id % heads);
    if (t >= tokens) return;
    int end;
    const int b = paged::owner_of(&samples, starts, cache.sequences, t, &end);
    if (b < 0) return;
    const int kv = h / (heads / cache.kv_heads);
    const int at = paged::length_of(cache, b) - (end - t);
    for (int c = lane; c < D; c += 32) q_row[warp][c] = __bfloat162float(Q[t * q_token + h * q_head + c]);
    __syncwarp();
    float m = -INFINITY, l = 0.0f, o[D / 32] = {};
    for (int j0 = 0; j0 <= at; j0 += 32) {
        const int j = j0 + lane;
        const int page = j <= at ? paged::page_of(cache.table, cache, b, j) : -1;
        const size_t row = page >= 0 ? paged::row_offset(cache, page, kv, j) : 0;
        float z = 0.0f;
        if (page >= 0)
            for (int c = 0; c < D; ++c) z = fmaf(q_row[warp][c], __bfloat162float(cache.K[row + c]), z);
        z = j <= at ? z * scale : -INFINITY;
        float top = z;
        for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
        top = fmaxf(top, m);
        const float p = expf(z - top), alpha = expf(m - top);
        l = l * alpha + p;
        m = top;
        for (int i = 0; i < D / 32; ++i) o[i] *= alpha;
        for (int k = 0; k < 32; ++k) {
            const float w = __shfl_sync(0xffffffffu, p, k);
            const long long r = __shfl_sync(0xffffffffu, page >= 0 ? static_cast<long long>(row) : -1ll, k);
            if (r < 0) continue;
            for (int i = 0; i < D / 32; ++i) o[i] = fmaf(w, __bfloat162float(cache.V[r + i * 32 + lane]), o[i]);
        }
    }
    for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
    for (int i = 0; i < D / 32; ++i) O[(static_cast<size_t>(t) * heads + h) * D + i * 32 + lane] = __float2bfloat16(o[i] * inv);
    if (lse && lane == 0) lse[static_cast<size_t>(t) * heads + h] = l > 0.0f ? m + logf(l) : -INFINITY;
}

// mass_out[b, kv, j] = mass[b, kv, j] + the weights that key j received: one thread a key, over the tokens and heads that see it.
template <int D>
__global__ void __launch_bounds__(128)
mass_kernel(const __nv_bfloat16* Q, long long q_token, long long q_head, paged::Cache cache, const int* starts, const float* lse, const float* mass,
            float* mass_out, int tokens, int heads, float scale, int capacity) {
    ptx::grid_dependency_wait();
    const int row = static_cast<int>(blockIdx.y), b = row / cache.kv_heads, kv = row % cache.kv_heads;
    const int j = static_cast<int>(blockIdx.x) * 128 + static_cast<int>(threadIdx.x);
    if (j >= capacity) return;
    const int first = max(starts[b], 0), end = min(starts[b + 1], tokens), length = paged::length_of(cache, b);
    float sum = mass[static_cast<size_t>(row) * capacity + j];
    if (j < length) {
        const int page = paged::page_of(cache.table, cache, b, j);
        float k[D];
        for (int c = 0; c < D; ++c) k[c] = page >= 0 ? __bfloat162float(cache.K[paged::row_offset(cache, page, kv, j) + c]) : 0.0f;
        const int G = heads / cache.kv_heads;
        float added = 0.0f;
        for (int t = first; t < end; ++t) {
            if (length - (starts[b + 1] - t) < j) continue;
            for (int g = 0; g < G; ++g) {
                const __nv_bfloat16* q = Q + t * q_token + (kv * G + g) * q_head;
                float z = 0.0f;
                for (int c = 0; c < D; ++c) z = fmaf(__bfloat162float(q[c]), k[c], z);
                added += expf(z * scale - lse[static_cast<size_t>(t) * heads + kv * G + g]);
            }
        }
        sum += added;
    }
    mass_out[static_cast<size_t>(row) * capacity + j] = sum;
}

}  // namespace pa0
}  // namespace attnw
