// The attention weight that cached keys receive from new tokens.
#pragma once
#include "paged.cuh"

namespace attnw {
namespace pm {

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

}  // namespace pm
}  // namespace attnw
