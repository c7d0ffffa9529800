// Rotary positions, and new tokens written into a paged cache.
//
// A pair of features (a, b) of a token at position n with frequency f turns by the angle n f:
//     a' = A (a cos - b sin),   b' = A (b cos + a sin)
// ("half": feature c with c + r/2; "interleaved": 2c with 2c + 1; features from r on stay).  The transpose of this map, which takes
// gradients back, is the same with -sin.
//
// Bound by HBM: every row is read once and written once, and one angle serves all heads of a token.  So a thread owns two 16-byte vectors
// of a token's row - the two halves of its pairs, or two neighbours of interleaved ones -, computes the cosines and sines of its pairs
// once, in registers, and walks the heads with them.  Angles are products in 64 bits, reduced there to (-1, 1] half turns: a float32 product loses a
// radian's digits at the far positions that a cache reaches (at 2^20 its spacing is 1/16).  About 60 instructions an angle; none are read.
// Measured: 4 x 32 x 4096 rows of 128 float32 82.5 us, 6.5 TB/s of 537 MB (a plain copy's rate); 4 x 4096 new tokens of 32 + 8 + 8 heads into a
// cache 69.5 us, 5.8 TB/s of 403 MB; a call with one token 4.6 and 5.1.
#pragma once
#include <cstdint>

#include "paged.cuh"

namespace attnw {
namespace rope {

constexpr int kThreads = 256;

struct Rows {  // strided [tokens (two dimensions), heads, d], d contiguous; strides in elements
    const void* src;
    void* dst;
    long long src_batch, src_token, src_head;
    long long dst_batch, dst_token, dst_head;
    int heads;
};

struct Turn {
    const int* positions;       // [tokens]; nullptr: nothing turns
    const double* frequencies;  // [rotary / 2]
    int rotary;
    float amplitude, sign;
};

template <typename T>
struct Vec;  // 16 bytes of a row as float32
template <>
struct Vec<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ void unpack(uint4 v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y), x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ void unpack(uint4 v, float (&x)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {  // nearest even, the only rounding
        return make_uint4(ptx::pack_bf16x2(x[0], x[1]), ptx::pack_bf16x2(x[2], x[3]), ptx::pack_bf16x2(x[4], x[5]), ptx::pack_bf16x2(x[6], x[7]));
    }
};

// One thread's part of a row: two vectors, and the cosines and sines of its kN pairs.
template <typename T, bool HALF>
struct Lane {
    static constexpr int kN = Vec<T>::kN;
    int off0, off1;  // features
    bool turns;
    float cos[kN], sin[kN];

    // `part`: 0 ... d / (2 kN) - 1.  rotary is a multiple of 16, so each part lies on one side of it.
    __device__ __forceinline__ void place(int part, int rotary) {
        turns = part < rotary / (2 * kN);
        off0 = HALF && turns ? part * kN : part * 2 * kN;
        off1 = HALF && turns ? off0 + rotary / 2 : off0 + kN;
    }
    __device__ __forceinline__ void angles(const Turn& t, int part, long long token) {
        if (!turns) return;
        const double n = static_cast<double>(t.positions[token]);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            double h = n * (t.frequencies[part * kN + i] * 0.31830988618379067154);  // half turns
            h -= 2.0 * rint(0.5 * h);
            sincospif(static_cast<float>(h), &sin[i], &cos[i]);
            cos[i] *= t.amplitude;
            sin[i] *= t.amplitude * t.sign;
        }
    }
    __device__ __forceinline__ void apply(uint4& v0, uint4& v1) const {
        if (!turns) return;
        float x[kN], y[kN];
        Vec<T>::unpack(v0, x);
        Vec<T>::unpack(v1, y);
        if (HALF) {
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const float a = x[i], b = y[i];
                x[i] = a * cos[i] - b * sin[i];
                y[i] = b * cos[i] + a * sin[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kN / 2; ++i) {
                float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i] = a * cos[i] - b * sin[i];
                x[2 * i + 1] = b * cos[i] + a * sin[i];
                a = y[2 * i], b = y[2 * i + 1];
                y[2 * i] = a * cos[kN / 2 + i] - b * sin[kN / 2 + i];
                y[2 * i + 1] = b * cos[kN / 2 + i] + a * sin[kN / 2 + i];
            }
        }
        v0 = Vec<T>::pack(x);
        v1 = Vec<T>::pack(y);
    }
};

// Rows of one token, `count` heads, kFlight of them on their way at a time.
constexpr int kFlight = 4;

template <typename T, bool HALF>
struct Rows4 {
    uint4 v0[kFlight], v1[kFlight];
    __device__ __forceinline__ void load(const Lane<T, HALF>& lane, const T* src, long long src_head, int h, int count) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (h + i < count) {
                const T* row = src + (h + i) * src_head;
                v0[i] = __ldcs(reinterpret_cast<const uint4*>(row + lane.off0));
                v1[i] = __ldcs(reinterpret_cast<const uint4*>(row + lane.off1));
            }
    }
    template <bool TURN>
    __device__ __forceinline__ void store(const Lane<T, HALF>& lane, T* dst, long long dst_head, int h, int count) {
#pragma unroll
        for (int i = 0; i < kFlight; ++i)
            if (h + i < count) {
                if (TURN) lane.apply(v0[i], v1[i]);
                T* row = dst + (h + i) * dst_head;
                *reinterpret_cast<uint4*>(row + lane.off0) = v0[i];
                *reinterpret_cast<uint4*>(row + lane.off1) = v1[i];
            }
    }
};

// The first rows have been loaded.
template <typename T, bool HALF, bool TURN>
__device__ __forceinline__ void walk(const Lane<T, HALF>& lane, Rows4<T, HALF>& rows, const T* src, long long src_head, T* dst, long long dst_head, int count) {
    for (int h = 0;;) {
        rows.template store<TURN>(lane, dst, dst_head, h, count);
        h += kFlight;
        if (h >= count) break;
        rows.load(lane, src, src_head, h, count);
    }
}

// Grid: x over (token, part), y over groups of `heads_each` heads.
template <typename T, bool HALF>
__global__ void __launch_bounds__(kThreads) rope_kernel(Rows rows, Turn turn, long long tokens, int per_batch, int parts, int heads_each) {
    const long long id = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const long long token = id / parts;
    const int part = static_cast<int>(id % parts);
    ptx::grid_dependency_wait();
    if (token >= tokens) return;
    Lane<T, HALF> lane;
    lane.place(part, turn.rotary);
    const int h0 = static_cast<int>(blockIdx.y) * heads_each, count = min(heads_each, rows.heads - h0);
    const long long b = token / per_batch, n = token % per_batch;
    const T* src = static_cast<const T*>(rows.src) + b * rows.src_batch + n * rows.src_token + h0 * rows.src_head;
    Rows4<T, HALF> held;
    held.load(lane, src, rows.src_head, 0, count);
    lane.angles(turn, part, token);
    walk<T, HALF, true>(lane, held, src, rows.src_head, static_cast<T*>(rows.dst) + b * rows.dst_batch + n * rows.dst_token + h0 * rows.dst_head, rows.dst_head,
                        count);
}

// Grid: x over (token, part); y over groups of heads, those of the queries first, then those of the keys, then the values'.
template <bool HALF>
__global__ void __launch_bounds__(kThreads)
append_kernel(Rows q, Rows k, Rows v, paged::Cache cache, const int* starts, Turn turn, int tokens, int parts, int heads_each, int q_groups, int kv_groups) {
    using T = __nv_bfloat16;
    __shared__ paged::Samples samples;
    ptx::grid_dependency_wait();
    const long long id = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    const long long token = id / parts;
    const int part = static_cast<int>(id % parts);
    int group = static_cast<int>(blockIdx.y);
    const int kind = group < q_groups ? 0 : group < q_groups + kv_groups ? 1 : 2;
    group -= kind == 0 ? 0 : kind == 1 ? q_groups : q_groups + kv_groups;
    const Rows& rows = kind == 0 ? q : kind == 1 ? k : v;
    const int h0 = group * heads_each, count = min(heads_each, rows.heads - h0);
    const T* src = static_cast<const T*>(rows.src) + token * rows.src_token + h0 * rows.src_head;
    Lane<T, HALF> lane;
    lane.place(part, turn.rotary);
    // (the rows are on their way while the token's sequence and place are looked up)
    Rows4<T, HALF> held;
    if (token < tokens) held.load(lane, src, rows.src_head, 0, count);
    paged::sample_starts(&samples, starts, cache.sequences, kThreads);
    __syncthreads();
    if (token >= tokens) return;
    int end;
    const int b = paged::owner_of(&samples, starts, cache.sequences, static_cast<int>(token), &end);
    if (b < 0) return;
    T* dst;
    long long dst_head;
    if (kind == 0) {
        dst = static_cast<T*>(rows.dst) + token * rows.dst_token + h0 * rows.dst_head;
        dst_head = rows.dst_head;
    } else {
        const int at = paged::length_of(cache, b) - (end - static_cast<int>(token));  // (of an owned token: end - token >= 1)
        if (at < 0) return;
        const int page = paged::page_of(cache.table, cache, b, at);
        if (page < 0) return;
        dst = (kind == 1 ? cache.K : cache.V) + paged::row_offset(cache, page, h0, at);
        dst_head = static_cast<long long>(cache.d) << cache.page_shift;
    }
    if (kind != 2 && turn.positions) {
        lane.angles(turn, part, token);
        walk<T, HALF, true>(lane, held, src, rows.src_head, dst, dst_head, count);
    } else {
        walk<T, HALF, false>(lane, held, src, rows.src_head, dst, dst_head, count);
    }
}

}  // namespace rope
}  // namespace attnw
