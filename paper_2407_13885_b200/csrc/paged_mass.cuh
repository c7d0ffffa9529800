// The attention weight that cached keys receive from new tokens:
//     mass_out[b, g, j] = mass[b, g, j] + sum over the tokens t and heads h of key head g that see key j of exp(scale Q[t, h] . K_j - lse[t, h]).
//
// The logarithms of the sums are attn_paged_kernel's, so each weight is final when it is computed; the scores are computed once more.  The KEYS are
// the rows here (S^T = K Q^T): a thread owns a key and adds up the columns, (token, head) rows of attn_paged's query tiles, in registers; no weight leaves
// them.  A CTA takes pairs of key tiles of one (sequence, key head), unit u of its Softmax warps the pair's tile u, and every query tile that sees
// some of their keys; where a sequence has one query tile (decoding) that one stays and the keys stream past it.
//
// Bound: one exponential an element, 1024 cycles of the special function units a tile of 128 x 128 against 512 of the tensor pipe; for single tokens the
// keys' way from HBM.  Measured: 1024 new tokens of each of two sequences over 5000 keys, 32 heads on 8, d = 128: 166 us, the special function units at
// 60 % while a CTA works; segments are whole key tiles, here five, where 4.3 would be one for each SM.
#pragma once
#include <cstddef>
#include <type_traits>

#include "attn_paged.cuh"

namespace attnw {
namespace pm {

constexpr int kThreads = 576;
constexpr int kSmWarps = 16;  // unit (2) x half of the columns (2) x TMEM lane quarter (4)
constexpr int kProducer = 16;
constexpr int kMma = 17;
constexpr int kSegments = 148;  // about as many segments are wanted in all, of the same cost: one an SM of a B200

enum : uint32_t {  // wait sites
    kSiteKEmpty = 80,
    kSiteQEmpty = 81,
    kSiteMmaK = 82,
    kSiteMmaQ = 83,
    kSiteMmaSFree = 84,
    kSiteSFull = 85,
    kSiteQFull = 86,
};

template <int D>
struct Smem {
    static constexpr int kAtoms = D / 64;
    static constexpr int kAtomBytes = kTile * 128;
    static constexpr int kTileBytes = kAtoms * kAtomBytes;
    // Six places for tiles.  One query tile: two pairs of key tiles, and it.  More: one pair, and four query tiles on their way (with two a tile of
    // 2 x 128 x 128 waited 0.9 us for the next one).
    static constexpr int kPlaces = 6;
    static __device__ __forceinline__ int pairs(bool resident) { return resident ? 2 : 1; }
    static __device__ __forceinline__ int q_stages(bool resident) { return resident ? 1 : 4; }
    static __device__ __forceinline__ int q_offset(bool resident, int stage) { return ((resident ? 4 : 2) + stage) * kTileBytes; }
    static constexpr int kLseOff = kPlaces * kTileBytes;            // float [stage][128]
    static constexpr int kSumOff = kLseOff + 4 * kTile * 4;  // float [pair parity][unit][half][128]
    static constexpr int kBarOff = kSumOff + 2 * 2 * 2 * kTile * 4;
    static constexpr int kBytes = kBarOff + 512;
    static constexpr int kDynamicBytes = kBytes + 1024;
};
static_assert(Smem<128>::kDynamicBytes <= 227 * 1024, "shared memory budget");

struct Segment {
    int b, h;          // sequence (-1: nothing), key head
    int token0, tokens;
    int seen0, length;
    int tile0, tile1;  // key tiles
    int q_tile;        // of the sequence's first query tile, among those of all
};

struct Barriers {
    uint64_t k_full[2], k_empty[2];      // per pair in flight
    uint64_t q_full[4], q_empty[4];
    uint64_t s_full[2][2], s_free[2][2];  // [unit][buffer]
    uint32_t tmem_base;
    uint32_t abort_flag;
    Segment segment;
};
static_assert(sizeof(Barriers) <= 512, "barrier block must fit its slot");

// By one warp.  A segment is a number of key tiles; a key tile's cost is that of its score tiles, and about one more for itself.
__device__ __noinline__ void schedule(const paged::Cache& c, const pa::Shape& s, const int* starts, int index, Segment* out) {
    const int lane = static_cast<int>(threadIdx.x & 31);
    auto cost_of = [&](const pa::Share& r) { return static_cast<long long>((r.n + s.tile_tokens - 1) / s.tile_tokens) + 1; };  // of a key tile
    long long total = 0;
    for (int b = lane; b < c.sequences; b += 32) {
        const pa::Share r = pa::share_of(c, s, starts, b);
        if (r.n > 0) total += cost_of(r) * ((r.length + kTile - 1) / kTile) * c.kv_heads;
    }
    total = pa::warp_sum(total);
    const long long most = max(1ll, (total + total / 16 + kSegments - 1) / kSegments);  // (a little more: what does not fit one round of CTAs takes another)
    long long first = 0, q_first = 0;
    if (lane == 0) out->b = -1;
    __syncwarp();
    for (int b0 = 0; b0 < c.sequences; b0 += 32) {
        const int b = b0 + lane;
        pa::Share r{};
        if (b < c.sequences) r = pa::share_of(c, s, starts, b);
        const int tiles = r.n > 0 ? (r.length + kTile - 1) / kTile : 0;
        // As many as come nearest to that cost; of single tokens, whose keys only pass by, an even number of key tiles each.  (The same for more tokens:
        // 2 x 1024 over 4000 keys 346 us and not 325, 1 x 512 over 1000 85 and not 74.5, 2048 over none 191 and not 160.  Boundaries by what the tiles behind
        // the diagonal cost less: 311, 84, 160.)
        const long long wanted = max(1ll, (tiles * cost_of(r) + most / 2) / most), unit = r.n > s.tile_tokens ? 1 : 2;
        const long long each = (tiles + unit * wanted - 1) / (unit * wanted) * unit;
        const long long segments = tiles > 0 ? (tiles + each - 1) / each : 0;
        const long long end = first + pa::warp_scan(segments * c.kv_heads, lane), begin = end - segments * c.kv_heads;
        const long long q_tiles = (r.n + s.tile_tokens - 1) / s.tile_tokens, q_end = q_first + pa::warp_scan(q_tiles, lane);
        if (index >= begin && index < end) {
            const long long at = index - begin, seg = at / c.kv_heads;
            out->h = static_cast<int>(at % c.kv_heads);
            out->token0 = min(max(starts[b], 0), s.tokens);
            out->tokens = r.n;
            out->seen0 = r.seen0;
            out->length = r.length;
            out->tile0 = static_cast<int>(seg * each);
            out->tile1 = static_cast<int>(min(static_cast<long long>(tiles), (seg + 1) * each));
            out->q_tile = static_cast<int>(q_end - q_tiles);
            out->b = b;
        }
        first = __shfl_sync(0xffffffffu, end, 31);
        q_first = __shfl_sync(0xffffffffu, q_end, 31);
    }
    __syncwarp();
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
mass_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ paged::Cache cache,
            const __grid_constant__ pa::Shape shape, const int* starts, const float* lse2, float scale_log2e, const float* mass, float* mass_out) {
    using L = Smem<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Barriers* bars = reinterpret_cast<Barriers*>(smem + L::kBarOff);
    const uint32_t bar = ptx::smem_u32(bars);
    auto bar_of = [bar](size_t field, int n) { return bar + static_cast<uint32_t>(field) + 8u * static_cast<uint32_t>(n); };
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    if (shape.least > 1 && pa::nothing_to_do(cache, shape, starts)) return;

    // ---- set-up ------------------------------------------------------------------------------
    if (warp == kProducer && lane == 0) {
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(&bars->k_full[s], 1);
            ptx::mbar_init(&bars->k_empty[s], 1);
        }
        for (int s = 0; s < 4; ++s) {
            ptx::mbar_init(&bars->q_full[s], 1);
            ptx::mbar_init(&bars->q_empty[s], 1 + kSmWarps);
        }
        for (int u = 0; u < 2; ++u)
            for (int i = 0; i < 2; ++i) {
                ptx::mbar_init(&bars->s_full[u][i], 1);
                ptx::mbar_init(&bars->s_free[u][i], 8);
            }
        bars->abort_flag = 0;
        ptx::mbar_fence_init();
        ptx::prefetch_tensormap(&tm_q);
        ptx::prefetch_tensormap(&tm_k);
    }
    if (warp == kMma) {
        ptx::tmem_alloc(&bars->tmem_base, kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::grid_dependency_wait();
    if (warp == 0) schedule(cache, shape, starts, static_cast<int>(blockIdx.x), &bars->segment);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
    const Segment seg = bars->segment;
    const int capacity = cache.table_width << cache.page_shift;
    const bool copies = mass != mass_out;
    // The query tiles: `t_first` of a pair is the first that sees its first key.
    const int q_tiles = (seg.tokens + shape.tile_tokens - 1) / shape.tile_tokens;
    const int pairs = seg.b < 0 ? 0 : (seg.tile1 - seg.tile0 + 1) / 2;
    const bool resident = q_tiles == 1;
    const int k_stages = L::pairs(resident), q_stages = L::q_stages(resident);
    auto t_first = [&](int kt) { return max(kt * kTile - seg.seen0 + 1, 0) / shape.tile_tokens; };  // q_tiles or more: nobody sees it
    struct Entry {  // of a ring
        int stage = 0;
        uint32_t phase = 0;
        __device__ __forceinline__ void next(int stages) {
            if (++stage == stages) {
                stage = 0;
                phase ^= 1u;
            }
        }
    };
    int k_loads = 0, q_loads = 0;

    if (warp == kProducer) {
        const uint64_t keep = ptx::policy_evict_last();
        const int page_shift = min(cache.page_shift, 7), parts = kTile >> page_shift;
        const int part = lane / L::kAtoms, atom = lane % L::kAtoms;
        const bool fetches = part < parts;
        const int* table = cache.table + static_cast<size_t>(max(seg.b, 0)) * cache.table_width;
        auto place = [&](int kt) {  // (see attn_paged_kernel)
            const int at = kt * kTile + (part << page_shift);
            int p = -1;
            if (fetches && at < seg.length) p = table[at >> cache.page_shift];
            return static_cast<unsigned>(p) < static_cast<unsigned>(cache.pages) ? p * cache.kv_heads + seg.h : cache.pages * cache.kv_heads;
        };
        const int q_bytes = shape.tile_tokens * shape.group * 128 * L::kAtoms;
        Entry ek, eq;
        bool ok = true;
        auto load_q = [&](int t) {
            ok = ok && warp_wait(bar_of(offsetof(Barriers, q_empty), eq.stage), eq.phase ^ 1u, abort_flag, kSiteQEmpty);
            if (!ok) return;
            if (lane == 0) {
                const uint32_t full = bar_of(offsetof(Barriers, q_full), eq.stage);
                ptx::mbar_expect_tx(full, static_cast<uint32_t>(q_bytes + kTile * 4));
                for (int a = 0; a < L::kAtoms; ++a)
                    ptx::tma_load_4d(smem + L::q_offset(resident, eq.stage) + a * L::kAtomBytes, &tm_q, &bars->q_full[eq.stage], a * 64, 0, seg.h,
                                     seg.token0 + t * shape.tile_tokens);
                ptx::bulk_load_1d(ptx::smem_u32(smem + L::kLseOff + eq.stage * kTile * 4),
                                  lse2 + (static_cast<size_t>(min(seg.q_tile + t, shape.q_tiles - 1)) * cache.kv_heads + seg.h) * kTile, kTile * 4,
                                  &bars->q_full[eq.stage]);
            }
            __syncwarp();
            eq.next(q_stages);
            ++q_loads;
        };
        for (int p = 0; ok && p < pairs; ++p) {
            const int kt = seg.tile0 + 2 * p, t0 = t_first(kt);
            if (t0 >= q_tiles) continue;
            const bool both = kt + 1 < seg.tile1;
            const int where[2] = {place(kt), both ? place(kt + 1) : 0};
            if (p == 0 && resident) load_q(0);
            ok = ok && warp_wait(bar_of(offsetof(Barriers, k_empty), ek.stage), ek.phase ^ 1u, abort_flag, kSiteKEmpty);
            if (!ok) break;
            const uint32_t full = bar_of(offsetof(Barriers, k_full), ek.stage);
            if (lane == 0) ptx::mbar_expect_tx(full, static_cast<uint32_t>((both ? 2 : 1) * L::kTileBytes));
            __syncwarp();
            if (fetches)
                for (int u = 0; u < (both ? 2 : 1); ++u)
                    ptx::tma_load_3d(smem + (2 * ek.stage + u) * L::kTileBytes + atom * L::kAtomBytes + (part << page_shift) * 128, &tm_k, full, atom * 64,
                                     ((kt + u) * kTile) & ((1 << cache.page_shift) - 1) & ~(kTile - 1), where[u], keep);
            __syncwarp();
            ek.next(k_stages);
            ++k_loads;
            if (!resident)
                for (int t = t0; ok && t < q_tiles; ++t) load_q(t);
        }
    } else if (warp == kMma) {
        const uint32_t base = ptx::smem_u32(smem);
        const uint32_t prior_failure = *reinterpret_cast<volatile unsigned int*>(&g_attnw_status);
        bool ok = !__any_sync(0xffffffffu, prior_failure != 0u);
        if (!ok) *abort_flag = 1;
        Entry ek, eq;
        int uses[2] = {0, 0};  // score tiles of each unit so far
        for (int p = 0; ok && p < pairs; ++p) {
            const int kt = seg.tile0 + 2 * p, t0 = t_first(kt);
            if (t0 >= q_tiles) continue;
            const int units = kt + 1 < seg.tile1 ? 2 : 1;
            ok = warp_wait(bar_of(offsetof(Barriers, k_full), ek.stage), ek.phase, abort_flag, kSiteMmaK);
            for (int t = t0; ok && t < q_tiles; ++t) {
                ok = warp_wait(bar_of(offsetof(Barriers, q_full), eq.stage), eq.phase, abort_flag, kSiteMmaQ);
                // columns beyond the tile's rows are not computed
                const int columns = min(shape.tile_tokens, seg.tokens - t * shape.tile_tokens) * shape.group;
                const uint32_t idesc = ptx::umma_idesc_bf16_f32(kTile, (columns + 15) & ~15);
                for (int u = 0; ok && u < units; ++u) {
                    const int buffer = uses[u] & 1;
                    ok = warp_wait(bar_of(offsetof(Barriers, s_free), u * 2 + buffer), (static_cast<uint32_t>(uses[u] >> 1) & 1u) ^ 1u, abort_flag, kSiteMmaSFree);
                    if (!ok) break;
                    ++uses[u];
                    ptx::tc_fence_after_sync();
                    const uint64_t a_desc = ptx::umma_desc_kmajor_sw128(base + static_cast<uint32_t>((2 * ek.stage + u) * L::kTileBytes));
                    const uint64_t b_desc = ptx::umma_desc_kmajor_sw128(base + static_cast<uint32_t>(L::q_offset(resident, eq.stage)));
                    if (ptx::elect_one()) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k) {
                            const uint64_t off = static_cast<uint64_t>(((k >> 2) * L::kAtomBytes + (k & 3) * 32) >> 4);
                            ptx::umma_f16_ss(tmem_base + static_cast<uint32_t>((u * 2 + buffer) * kTile), a_desc + off, b_desc + off, idesc, k > 0 ? 1u : 0u);
                        }
                        ptx::umma_commit(&bars->s_full[u][buffer]);
                    }
                    __syncwarp();
                }
                if (!ok) break;
                if (!resident) {
                    if (ptx::elect_one()) ptx::umma_commit(&bars->q_empty[eq.stage]);
                    __syncwarp();
                    eq.next(q_stages);
                }
            }
            if (!ok) break;
            if (ptx::elect_one()) ptx::umma_commit(&bars->k_empty[ek.stage]);
            __syncwarp();
            ek.next(k_stages);
        }
    } else {
        // ================= Softmax warps: two threads per key, 64 columns of a tile each =================
        const int u = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3;
        const int row = quarter * 32 + lane;
        const uint32_t t_own = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + static_cast<uint32_t>(u * 2 * kTile + half * kHalf);
        const uint64_t c2c2 = ptx::pack2(scale_log2e, scale_log2e);
        float* sums = reinterpret_cast<float*>(smem + L::kSumOff);
        Entry eq;
        int uses = 0;
        bool ok = true;
        // What no pair covers is copied: sequences without new tokens, and the places behind a length.
        if (copies && u == 1) {
            const bool failed = *reinterpret_cast<volatile unsigned int*>(&g_attnw_status) != 0u;
            const int rows = cache.sequences * cache.kv_heads;
            for (int r = static_cast<int>(blockIdx.x); r < rows && !failed; r += static_cast<int>(gridDim.x)) {
                const pa::Share s = pa::share_of(cache, shape, starts, r / cache.kv_heads);
                if (s.n == 0 && shape.least > 1) continue;  // (attn_few_kernel's)
                for (int j = (s.n > 0 ? s.length : 0) + (warp - 8) * 32 + lane; j < capacity; j += 256)
                    mass_out[static_cast<size_t>(r) * capacity + j] = mass[static_cast<size_t>(r) * capacity + j];
            }
        }
        for (int p = 0; p < pairs; ++p) {
            const int kt = seg.tile0 + 2 * p, t0 = t_first(kt);
            const bool active = u == 0 || kt + 1 < seg.tile1;
            const int key = (kt + u) * kTile + row;
            uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
            for (int t = t0; ok && t < q_tiles; ++t) {
                ok = warp_wait(bar_of(offsetof(Barriers, q_full), eq.stage), eq.phase, abort_flag, kSiteQFull);
                if (ok && active) {
                    const int buffer = uses & 1;
                    ok = warp_wait(bar_of(offsetof(Barriers, s_full), u * 2 + buffer), static_cast<uint32_t>(uses >> 1) & 1u, abort_flag, kSiteSFull);
                    ++uses;
                    if (ok) {
                        ptx::tc_fence_after_sync();
                        const int first = t * shape.tile_tokens;  // the tile's first token
                        const int columns = min(shape.tile_tokens, seg.tokens - first) * shape.group;
                        // this thread's columns: tokens that see the key begin at `from`, and the tile ends at `to`
                        const int from = max(key - seg.seen0 + 1 - first, 0) * shape.group - half * kHalf, to = columns - half * kHalf;
                        const bool masked = columns < kTile || (kt + u) * kTile + kTile - 1 - seg.seen0 + 1 > first;
                        const float4* nlse = reinterpret_cast<const float4*>(smem + L::kLseOff + eq.stage * kTile * 4) + half * (kHalf / 4);
                        if (to > 0) {  // (the columns of few rows lie in the first half)
                            // all scores to registers: the buffer goes back, and the exponentials have nothing to wait for
                            uint32_t s0[kChunk], s1[kChunk];
                            ptx::tmem_ld_32x32b_x32(t_own + static_cast<uint32_t>(buffer * kTile), s0);
                            ptx::tmem_ld_32x32b_x32(t_own + static_cast<uint32_t>(buffer * kTile + kChunk), s1);
                            ptx::tmem_wait_ld();
                            ptx::tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(&bars->s_free[u][buffer]);
                            auto add_up = [&](const uint32_t(&s)[kChunk], int c, auto some) {
#pragma unroll
                                for (int i = 0; i < kChunk; i += 4) {
                                    const float4 n = nlse[(c + i) / 4];
                                    float x[4];
                                    ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), c2c2, ptx::pack2(n.x, n.y)), x[0], x[1]);
                                    ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])), c2c2, ptx::pack2(n.z, n.w)), x[2], x[3]);
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        x[e] = ptx::ex2_approx(x[e]);
                                        if constexpr (decltype(some)::value) x[e] = c + i + e >= from && c + i + e < to ? x[e] : 0.0f;
                                    }
                                    acc[(i >> 1) & 3] = ptx::add2(acc[(i >> 1) & 3], ptx::pack2(x[0], x[1]));
                                    acc[((i >> 1) + 1) & 3] = ptx::add2(acc[((i >> 1) + 1) & 3], ptx::pack2(x[2], x[3]));
                                }
                            };
                            if (masked) {
                                add_up(s0, 0, std::true_type{});
                                if (to > kChunk) add_up(s1, kChunk, std::true_type{});
                            } else {
                                add_up(s0, 0, std::false_type{});
                                add_up(s1, kChunk, std::false_type{});
                            }
                        } else {
                            __syncwarp();
                            if (lane == 0) ptx::mbar_arrive(&bars->s_free[u][buffer]);
                        }
                    }
                }
                if (!resident) {
                    __syncwarp();
                    if (ok && lane == 0) ptx::mbar_arrive(&bars->q_empty[eq.stage]);
                    eq.next(q_stages);
                }
            }
            // the halves of a key's columns meet in shared memory (even and odd pairs in places of their own: nobody is two pairs ahead)
            float a[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) ptx::unpack2(acc[i], a[2 * i], a[2 * i + 1]);
            const float sum = ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
            float* mine = sums + ((p & 1) * 2 + u) * 2 * kTile;
            mine[half * kTile + row] = sum;
            ptx::named_sync(static_cast<uint32_t>(1 + u), 256);
            if (half == 0 && active && ok && key < seg.length) {
                const size_t at = (static_cast<size_t>(seg.b) * cache.kv_heads + seg.h) * capacity + key;
                mass_out[at] = mass[at] + (sum + mine[kTile + row]);
            }
        }
    }

    // ---- teardown: every role falls through to here, also after a wait gave up ----
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        // Unwinding: let the copies already in flight land before shared memory is released.
        if (warp == kProducer && lane == 0) {
            const long long t0 = clock64();
            auto land = [&](uint64_t* full, int stages, int loads) {
                for (int it = loads > stages ? loads - stages : 0; it < loads; ++it)
                    while (!ptx::mbar_try_wait(&full[it % stages], static_cast<uint32_t>(it / stages) & 1u) && clock64() - t0 < kWaitLimitCycles / 8) {
                    }
            };
            land(bars->k_full, k_stages, k_loads);
            land(bars->q_full, q_stages, q_loads);
        }
    }
    if (warp == kMma) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

}  // namespace pm
}  // namespace attnw
