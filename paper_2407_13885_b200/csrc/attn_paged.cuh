// Attention of new tokens over a paged cache on the tensor cores: one pass over the keys with a running maximum and sum (as in
// attn_onepass.cuh, whose Softmax this is).
//
//     O[t, h] = sum_j p_j V_j,   p_j = exp(z_j - lse),   z_j = scale * Q[t, h] . K_j,   j <= at(t),
// where at(t) is the token's own place in its sequence.  No visible key: O = 0, lse = -inf.
//
// The G query heads of a key head read the same keys, so the rows of a query tile are (token, head of the group): floor(128 / G) tokens
// and their G heads, by one four-dimensional TMA box, whatever G is and wherever tokens and heads lie.  A block is up to two query tiles of
// one (sequence, key head).  Its CTA has two units that share the tensor pipe:
//   whole   two query tiles: unit q has tile q, every key tile serves both;
//   split   one query tile (decoding, and what a chunk leaves over): unit 0 has the even key tiles, unit 1 the odd ones, merged at the end.
// A key tile is 128 keys of one or more pages, one TMA box (per 64 features) a page.  The keys of a block may be cut into segments, each a CTA's:
// its unnormalised O, offset and sum go to a workspace and combine_kernel joins them.
//
// What the host knows is the number of tokens, of sequences, and the width of the table; the lengths are on the device.  So each CTA works out for itself
// what it does (schedule): the cost of all blocks, the segment length that gives kSegments of them, and which segment has its index.
#pragma once
#include <cstddef>

#include "attn_onepass.cuh"
#include "paged.cuh"

namespace attnw {
namespace pa {

using av1::kLazy;
using av1::kPassAt;

constexpr int kThreads = 608;
constexpr int kSmWarps = 16;  // Softmax warps: unit (2) x column half (2) x TMEM lane quarter (4)
constexpr int kProducer = 16;
constexpr int kMma = 17;         // the scores' issuer
constexpr int kMmaProduct = 18;  // the products'
constexpr int kSegments = 592;   // about as many segments are wanted in all: four an SM of a B200
constexpr int kLeastCost = 4;    // of a segment: key tiles of one query tile

enum : uint32_t {  // wait sites of this kernel (low byte of the status word)
    kSiteProducerEmpty = 112,
    kSiteMmaQ = 113,
    kSiteMmaKFull = 114,
    kSiteMmaSFree = 115,
    kSiteMmaPFull = 116,
    kSiteSFull = 117,
    kSitePFree = 118,
    kSiteOFull = 119,
    kSiteLFull = 120,
};

constexpr int kUnitStats = 4 * kTile;

template <int D>
struct Smem {
    static constexpr int kAtoms = D / 64;
    static constexpr int kAtomBytes = kTile * 128;          // 128 rows x 128 bytes
    static constexpr int kTileBytes = kAtoms * kAtomBytes;  // a Q, K or V tile
    // K and V tiles.  Split: one more, in the second query tile's place.  Each kind has a ring of its own, because it has an issuer of its own: an issuer
    // waits for its tiles by the parity of a stage's uses, and would take the use before the last for the last where the one between is the other's.
    static constexpr int kStages = (D == 128) ? 4 : 6;
    static constexpr int kKStages = kStages / 2;
    static __device__ __forceinline__ int v_stages(bool whole) { return whole ? kStages / 2 : kStages / 2 + 1; }
    // Tensor memory as in attn_onepass.cuh: d = 64 has room for scores, O and P of both units, d = 128 for one buffer of scores that they use in turn.
    static constexpr bool kSharedS = D == 128;
    static __host__ __device__ constexpr uint32_t s_col(int q) { return kSharedS ? 0u : static_cast<uint32_t>(q * 256); }
    static __host__ __device__ constexpr uint32_t p_col(int q) { return kSharedS ? 128u + static_cast<uint32_t>(q * 64) : static_cast<uint32_t>(q * 256 + 192); }
    static __host__ __device__ constexpr uint32_t o_col(int q) { return kSharedS ? 256u + static_cast<uint32_t>(q * 128) : static_cast<uint32_t>(q * 256 + 128); }
    static constexpr int kQOff = 0;
    static constexpr int kKOff = kQOff + 2 * kTileBytes;
    static constexpr int kStatOff = kKOff + kStages * kTileBytes;  // per unit: maxima, float [2 steps][2 halves][128 rows]; at the end sums and offset
    static constexpr int kBarOff = kStatOff + 2 * kUnitStats * 4;
    static constexpr int kBytes = kBarOff + 512;
    static constexpr int kDynamicBytes = kBytes + 1024;
};
static_assert(Smem<128>::kDynamicBytes <= 227 * 1024, "shared memory budget");

// What one CTA does.
struct Segment {
    int b;             // sequence, -1: nothing
    int h;             // key head
    int token0;        // the block's first token and how many it has
    int tokens;
    int seen0;         // keys that the first token sees, not cut off below zero
    int length;        // keys of the sequence
    int tile0, tile1;  // key tiles
    int segments;      // that the block is cut into
    int whole;
    int q_tile;        // the block's first query tile, among those of all sequences
    long long part;    // segments > 1: the workspace's row of the segment's first row
};

struct Barriers {
    uint64_t q_full;
    uint64_t k_full[3], k_empty[3], v_full[4], v_empty[4];
    uint64_t s_full[2], s_free[2];  // per unit: scores written / read into registers (8 warps)
    uint64_t p_full[2], p_free[2];  // per unit: P written (8 warps) / read by its MMAs
    uint64_t o_full[2];             // per unit: every product complete
    uint64_t l_full[2], l_both;     // the row statistics are in shared memory: whole, per unit (8 warps); split (16)
    uint32_t tmem_base;
    uint32_t abort_flag;
    Segment segment;
};
static_assert(sizeof(Barriers) <= 512, "barrier block must fit its slot");

struct Shape {
    int tokens, heads, group;  // query heads of a key head
    int tile_tokens;           // tokens of a query tile: floor(128 / group)
    int part_rows;             // rows that the workspace has
    int q_tiles;               // query tiles a key head, at most (of all sequences)
};

// A sequence's part in the schedule.
struct Share {
    int n, seen0, length, blocks, rows;  // new tokens, (see Segment), blocks a key head, rows of a block
    long long cost;                      // of a block
};

__device__ __forceinline__ Share share_of(const paged::Cache& c, const Shape& s, const int* starts, int b) {
    Share r;
    const int s0 = starts[b], s1 = starts[b + 1];
    const int t0 = min(max(s0, 0), s.tokens), t1 = min(max(s1, 0), s.tokens);
    r.n = max(t1 - t0, 0);
    r.length = paged::length_of(c, b);
    const long long seen = static_cast<long long>(r.length) - (static_cast<long long>(s1) - t0) + 1;
    r.seen0 = static_cast<int>(max(seen, -(1ll << 30)));
    r.blocks = (r.n + 2 * s.tile_tokens - 1) / (2 * s.tile_tokens);
    r.rows = min(r.n, 2 * s.tile_tokens) * s.group;
    r.cost = static_cast<long long>((r.length + kTile - 1) / kTile) * (r.n > s.tile_tokens ? 2 : 1);
    return r;
}

__device__ __forceinline__ long long warp_sum(long long x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ long long warp_scan(long long x, int lane) {  // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// What combine_kernel has to know of a sequence: the segments of its blocks (1: nothing to join), the workspace's row that they begin at, and the
// first of its query tiles.
struct Plan {
    int segments, rows;
    long long part, q_tile;
};

// Where the sums of a query tile's rows lie for mass_kernel: minus their logarithms to base 2, float [query tile][key head][128].
__device__ __forceinline__ size_t lse2_row(const paged::Cache& c, long long q_tile, int h) { return (static_cast<size_t>(q_tile) * c.kv_heads + h) * kTile; }

// By one warp.  Finds segment `index`; index 0 also writes the plan.
__device__ __noinline__ void schedule(const paged::Cache& c, const Shape& s, const int* starts, int index, Segment* out, Plan* plan) {
    const int lane = static_cast<int>(threadIdx.x & 31);
    long long total = 0;
    for (int b0 = 0; b0 < c.sequences; b0 += 32) {
        if (b0 + lane < c.sequences) {
            const Share r = share_of(c, s, starts, b0 + lane);
            total += r.cost * r.blocks * c.kv_heads;
        }
    }
    total = warp_sum(total);
    // The cost of a segment; one of two query tiles twice that.  So there are at most kSegments more segments than blocks, and those that come
    // from cutting a block up are at most 2 kSegments, of 128 rows at most (or half as many, of 256).
    const long long most = max(static_cast<long long>(kLeastCost), (total + kSegments - 1) / kSegments);
    long long first = 0, part = 0, q_first = 0;  // segments, workspace rows and query tiles of the sequences in front
    if (lane == 0) out->b = -1;
    __syncwarp();
    for (int b0 = 0; b0 < c.sequences; b0 += 32) {
        const int b = b0 + lane;
        Share r{};
        if (b < c.sequences) r = share_of(c, s, starts, b);
        const long long own_most = r.n > s.tile_tokens ? 2 * most : most;
        int cut = static_cast<int>(max(1ll, (r.cost + own_most - 1) / own_most));
        const long long blocks = static_cast<long long>(r.blocks) * c.kv_heads;
        const long long rows = cut > 1 ? blocks * cut * r.rows : 0;
        const long long part_end = part + warp_scan(rows, lane);
        if (part_end > s.part_rows) cut = 1;  // (the host's bound holds for tokens that belong to one sequence each)
        const long long end = first + warp_scan(blocks * cut, lane), begin = end - blocks * cut;
        const long long q_tiles = (r.n + s.tile_tokens - 1) / s.tile_tokens, q_end = q_first + warp_scan(q_tiles, lane);
        if (index == 0 && plan && b < c.sequences) plan[b] = {cut, r.rows, part_end - rows, q_end - q_tiles};
        if (index >= begin && index < end) {
            int at = static_cast<int>(index - begin);
            const int seg = at % cut;
            at /= cut;
            const int h = at % c.kv_heads, block = r.blocks - 1 - at / c.kv_heads;  // the longest first
            const int i0 = block * 2 * s.tile_tokens;
            out->h = h;
            out->token0 = min(max(starts[b], 0), s.tokens) + i0;
            out->tokens = min(r.n - i0, 2 * s.tile_tokens);
            out->seen0 = r.seen0 + i0;
            out->length = r.length;
            const int seen = min(max(out->seen0 + out->tokens - 1, 0), r.length), tiles = (seen + kTile - 1) / kTile;
            out->tile0 = static_cast<int>(static_cast<long long>(tiles) * seg / cut);
            out->tile1 = static_cast<int>(static_cast<long long>(tiles) * (seg + 1) / cut);
            out->segments = cut;
            out->whole = out->tokens > s.tile_tokens;
            out->q_tile = static_cast<int>(q_end - q_tiles) + 2 * block;
            out->part = part_end - rows + ((static_cast<long long>(block) * c.kv_heads + h) * cut + seg) * r.rows;
            out->b = b;
        }
        first = __shfl_sync(0xffffffffu, end, 31);
        part = __shfl_sync(0xffffffffu, part_end, 31);
        q_first = __shfl_sync(0xffffffffu, q_end, 31);
    }
    __syncwarp();
}

// The logarithm of a row's sum l 2^top: to the caller, and for mass_kernel.
__device__ __forceinline__ void store_lse(const paged::Cache& c, const Shape& s, float* lse, float* lse2, size_t out_row, long long q_tile, int h, int row, float top,
                                          float l) {
    const float log2_sum = l > 0.0f ? top + ptx::lg2_approx(l) : __int_as_float(0xff800000);
    if (lse) lse[out_row] = 0.69314718055994531f * log2_sum;
    if (lse2 && q_tile < s.q_tiles) lse2[lse2_row(c, q_tile, h) + row] = -log2_sum;  // (the host's bound holds for tokens of one sequence each)
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
attn_paged_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ paged::Cache cache, const __grid_constant__ Shape shape, const int* starts, float scale_log2e,
                  __nv_bfloat16* O, float* lse, float* lse2, float* part_o, float2* part_stats, Plan* plan) {
    using L = Smem<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Barriers* bars = reinterpret_cast<Barriers*>(smem + L::kBarOff);
    const uint32_t bar = ptx::smem_u32(bars);
    auto bar_of = [bar](size_t field, int n) { return bar + static_cast<uint32_t>(field) + 8u * static_cast<uint32_t>(n); };
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    // ---- set-up ------------------------------------------------------------------------------
    if (warp == kProducer && lane == 0) {
        ptx::mbar_init(&bars->q_full, 1);
        for (int s = 0; s < 3; ++s) {
            ptx::mbar_init(&bars->k_full[s], 1);
            ptx::mbar_init(&bars->k_empty[s], 1);
        }
        for (int s = 0; s < 4; ++s) {
            ptx::mbar_init(&bars->v_full[s], 1);
            ptx::mbar_init(&bars->v_empty[s], 1);
        }
        for (int q = 0; q < 2; ++q) {
            ptx::mbar_init(&bars->s_full[q], 1);
            ptx::mbar_init(&bars->s_free[q], 8);
            ptx::mbar_init(&bars->p_full[q], 8);
            ptx::mbar_init(&bars->p_free[q], 1);
            ptx::mbar_init(&bars->o_full[q], 1);
            ptx::mbar_init(&bars->l_full[q], 8);
        }
        ptx::mbar_init(&bars->l_both, 16);
        bars->abort_flag = 0;
        ptx::mbar_fence_init();
        ptx::prefetch_tensormap(&tm_q);
        ptx::prefetch_tensormap(&tm_k);
        ptx::prefetch_tensormap(&tm_v);
    }
    if (warp == kMma) {
        ptx::tmem_alloc(&bars->tmem_base, kTmemCols);
        ptx::tmem_relinquish();
    }
    ptx::grid_dependency_wait();
    if (warp == 0) schedule(cache, shape, starts, static_cast<int>(blockIdx.x), &bars->segment, plan);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
    const Segment& seg = bars->segment;
    const bool whole = seg.whole != 0;
    const int tiles = seg.b < 0 ? 0 : seg.tile1 - seg.tile0;
    // The key tiles of a unit: all of them, or every other one.
    const int steps[2] = {whole ? tiles : (tiles + 1) / 2, whole ? tiles : tiles / 2};
    const int tile0 = seg.tile0;
    const int v_stages = L::v_stages(whole);
    auto k_offset = [](int s) { return L::kKOff + s * L::kTileBytes; };
    auto v_offset = [](int s) { return s < L::kStages - L::kKStages ? L::kKOff + (L::kKStages + s) * L::kTileBytes : L::kQOff + L::kTileBytes; };
    auto key_tile = [&](int j, int q) { return tile0 + (whole ? j : 2 * j + q); };
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
    int k_loads = 0, v_loads = 0;  // producer: tiles asked for

    if (tiles == 0) {
        // nothing to compute: a segment index behind the last, or a block that sees no key
    } else if (warp == kProducer) {
        // ================= TMA producer: Q once, then the K and V tiles in the order the MMA issuers read them =========
        // A key tile is up to 8 pages; lane i fetches the part of its page and atom.  Places behind the sequence's length, and pages
        // outside the cache, are fetched from behind the cache: the tensor map fills in zeros.
        const uint64_t policy = seg.tokens < shape.tile_tokens ? ptx::policy_evict_first() : ptx::policy_evict_last();
        const int q_rows = shape.tile_tokens * shape.group;
        if (lane == 0) {
            ptx::mbar_expect_tx(&bars->q_full, static_cast<uint32_t>((whole ? 2 : 1) * L::kAtoms * q_rows * 128));
            for (int q = 0; q < (whole ? 2 : 1); ++q)
                for (int a = 0; a < L::kAtoms; ++a)
                    ptx::tma_load_4d(smem + L::kQOff + q * L::kTileBytes + a * L::kAtomBytes, &tm_q, &bars->q_full, a * 64, 0, seg.h,
                                     seg.token0 + q * shape.tile_tokens);
        }
        __syncwarp();
        const int page_shift = min(cache.page_shift, 7), parts = kTile >> page_shift;  // boxes of a tile, and keys (log2) of a box
        const int part = lane / L::kAtoms, atom = lane % L::kAtoms;
        const bool fetches = part < parts;
        const int* table = cache.table + static_cast<size_t>(seg.b) * cache.table_width;
        auto place = [&](int kt) {  // the page's place among those of all heads
            const int at = kt * kTile + (part << page_shift);
            int p = -1;
            if (fetches && at < seg.length) p = table[at >> cache.page_shift];
            return static_cast<unsigned>(p) < static_cast<unsigned>(cache.pages) ? p * cache.kv_heads + seg.h : cache.pages * cache.kv_heads;
        };
        Entry ek, ev;
        bool ok = true;
        auto load = [&](const CUtensorMap* map, uint32_t full, uint32_t empty, uint32_t phase, uint8_t* dst, int kt, int where) {
            if (!ok) return;
            ok = warp_wait(empty, phase ^ 1u, abort_flag, kSiteProducerEmpty);
            if (!ok) return;
            if (lane == 0) ptx::mbar_expect_tx(full, static_cast<uint32_t>(L::kTileBytes));
            __syncwarp();
            if (fetches)
                ptx::tma_load_3d(dst + atom * L::kAtomBytes + (part << page_shift) * 128, map, full, atom * 64,
                                 (kt * kTile) & ((1 << cache.page_shift) - 1) & ~(kTile - 1), where, policy);
            __syncwarp();
        };
        auto load_k = [&](int kt, int where) {
            load(&tm_k, bar_of(offsetof(Barriers, k_full), ek.stage), bar_of(offsetof(Barriers, k_empty), ek.stage), ek.phase, smem + k_offset(ek.stage), kt, where);
            ek.next(L::kKStages);
            k_loads += ok ? 1 : 0;
        };
        auto load_v = [&](int kt, int where) {
            load(&tm_v, bar_of(offsetof(Barriers, v_full), ev.stage), bar_of(offsetof(Barriers, v_empty), ev.stage), ev.phase, smem + v_offset(ev.stage), kt, where);
            ev.next(v_stages);
            v_loads += ok ? 1 : 0;
        };
        const int lists = whole ? 1 : 2;  // units that have key tiles of their own
        int where_k[2] = {place(key_tile(0, 0)), lists > 1 && steps[1] > 0 ? place(key_tile(0, 1)) : 0}, where_v[2] = {0, 0};
        for (int j = -1; ok && j < steps[0]; ++j) {
            for (int q = 0; q < lists; ++q) {
                const int next = where_k[q];
                if (j + 2 < steps[q]) where_k[q] = place(key_tile(j + 2, q));  // a step ahead of its use
                if (j + 1 < steps[q]) load_k(key_tile(j + 1, q), next);
                if (j >= 0 && j < steps[q]) load_v(key_tile(j, q), where_v[q]);
                where_v[q] = next;
            }
        }
    } else if (warp == kMma || warp == kMmaProduct) {
        // ================= MMA issuers (warp-uniform loops, one elected lane issues): of scores, of products =================
        constexpr uint32_t idesc_s = ptx::umma_idesc_bf16_f32(kTile, kTile);
        constexpr uint32_t idesc_o = ptx::umma_idesc_bf16_f32(kTile, D) | (1u << 16);  // B operand MN-major
        const uint32_t base = ptx::smem_u32(smem);
        // Did an earlier launch give up?  Then this one computes and writes nothing.
        const uint32_t prior_failure = *reinterpret_cast<volatile unsigned int*>(&g_attnw_status);
        bool ok = warp_wait(bar_of(offsetof(Barriers, q_full), 0), 0, abort_flag, kSiteMmaQ);
        if (__any_sync(0xffffffffu, prior_failure != 0u)) {
            *abort_flag = 1;
            ok = false;
        }
        Entry e;  // of the issuer's own ring
        auto arrived = [&](size_t full) { ok = ok && warp_wait(bar_of(full, e.stage), e.phase, abort_flag, kSiteMmaKFull); };
        auto release = [&](uint64_t* empty, int stages) {  // the tile may be replaced once the MMAs issued so far are complete
            if (ptx::elect_one()) ptx::umma_commit(empty + e.stage);
            __syncwarp();
            e.next(stages);
        };
        int last_q = 0, last_j = -1;  // kSharedS: whose scores the buffer holds
        auto scores = [&](int q, int j) {  // S of step j
            const int before_q = L::kSharedS ? last_q : q, before_j = L::kSharedS ? last_j : j - 1;
            ok = ok && warp_wait(bar_of(offsetof(Barriers, s_free), before_q), static_cast<uint32_t>(before_j) & 1u, abort_flag, kSiteMmaSFree);
            if (!ok) return;
            last_q = q;
            last_j = j;
            ptx::tc_fence_after_sync();
            const uint32_t d_tmem = tmem_base + L::s_col(q);
            const uint64_t a_desc = ptx::umma_desc_kmajor_sw128(base + L::kQOff + (whole ? static_cast<uint32_t>(q * L::kTileBytes) : 0u));
            const uint64_t b_desc = ptx::umma_desc_kmajor_sw128(base + static_cast<uint32_t>(k_offset(e.stage)));
            if (ptx::elect_one()) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint64_t off = static_cast<uint64_t>(((k >> 2) * L::kAtomBytes + (k & 3) * 32) >> 4);
                    ptx::umma_f16_ss(d_tmem, a_desc + off, b_desc + off, idesc_s, k > 0 ? 1u : 0u);
                }
                ptx::umma_commit(&bars->s_full[q]);
            }
            __syncwarp();
        };
        auto product = [&](int q, int j) {  // O += P V of step j
            ok = ok && warp_wait(bar_of(offsetof(Barriers, p_full), q), static_cast<uint32_t>(j) & 1u, abort_flag, kSiteMmaPFull);
            if (!ok) return;
            ptx::tc_fence_after_sync();
            const uint32_t o_tmem = tmem_base + L::o_col(q), p_tmem = tmem_base + L::p_col(q);
            const uint64_t b_desc = av::umma_desc_mnmajor_sw128(base + static_cast<uint32_t>(v_offset(e.stage)), L::kAtomBytes);
            if (ptx::elect_one()) {
#pragma unroll
                for (int kk = 0; kk < kTile / 16; ++kk)  // 16 keys per instruction
                    ptx::umma_f16_ts(o_tmem, p_tmem + static_cast<uint32_t>(kk * 8), b_desc + static_cast<uint64_t>(kk * 16 * 128 >> 4), idesc_o,
                                     (j > 0 || kk > 0) ? 1u : 0u);
                ptx::umma_commit(&bars->p_free[q]);
                if (j + 1 == steps[q]) ptx::umma_commit(&bars->o_full[q]);
            }
            __syncwarp();
        };
        // The values behind the sequence's length may be anything, NaN too, and a weight of zero does not silence that: such rows become zeros.
        auto clear_unused = [&](int kt) {
            const int used = seg.length - kt * kTile;
            if (!ok || used >= kTile) return;
            uint8_t* rows = smem + v_offset(e.stage);
            for (int i = max(used, 0) * 8 + lane; i < kTile * 8; i += 32)
                for (int a = 0; a < L::kAtoms; ++a) *reinterpret_cast<uint4*>(rows + a * L::kAtomBytes + i * 16) = make_uint4(0u, 0u, 0u, 0u);
            ptx::fence_proxy_async_smem();
            __syncwarp();
        };
        if (warp == kMma) {
            for (int j = 0; ok && j < steps[0]; ++j) {
                for (int q = 0; ok && q < (whole ? 1 : 2); ++q) {
                    if (j >= steps[q]) continue;
                    arrived(offsetof(Barriers, k_full));
                    scores(q, j);
                    if (whole) scores(1, j);
                    release(bars->k_empty, L::kKStages);
                }
            }
        } else {
            for (int j = 0; ok && j < steps[0]; ++j) {
                for (int q = 0; ok && q < (whole ? 1 : 2); ++q) {
                    if (j >= steps[q]) continue;
                    arrived(offsetof(Barriers, v_full));
                    clear_unused(key_tile(j, q));
                    product(q, j);
                    if (whole) product(1, j);
                    release(bars->v_empty, v_stages);
                }
            }
        }
    }
    if (warp < kSmWarps && seg.b >= 0) {
        // ================= Softmax warps: two threads per query row, 64 key columns of a tile each =================
        const int q = warp >> 3;
        const int half = (warp >> 2) & 1;
        const int quarter = warp & 3;
        const uint32_t t_quarter = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        const uint32_t t_own = t_quarter + L::s_col(q) + static_cast<uint32_t>(half * kHalf);
        const uint32_t o_own = t_quarter + L::o_col(q) + static_cast<uint32_t>(half * (D / 2));  // this thread's D/2 columns of O
        const float c2 = scale_log2e;
        const uint64_t c2c2 = ptx::pack2(c2, c2);
        const int row = quarter * 32 + lane;
        float* const stats = reinterpret_cast<float*>(smem + L::kStatOff) + q * kUnitStats;
        const uint32_t max_own = ptx::smem_u32(stats + half * kTile + row), max_other = ptx::smem_u32(stats + (half ^ 1) * kTile + row);
        const uint32_t lane0 = lane == 0;
        const uint32_t p_own = t_quarter + L::p_col(q) + static_cast<uint32_t>(half * 32);  // its 64 keys of P
        // The row's token (of the block), and the keys that it sees: a token more for each row of G.  A row that is none's gets what its place would.
        const int tile_first = whole ? q * shape.tile_tokens : 0;  // the first token of this unit's query tile
        const int token = tile_first + row / shape.group;
        const int seen = min(max(seg.seen0 + token, 0), seg.length);
        const int seen_least = min(max(seg.seen0 + tile_first, 0), seg.length);  // of the tile's rows
        float smax = -3.0e38f;  // running maximum of the raw scores of this row (all columns)
        float mb = -3.0e38f;    // the offset the weights, l and O's row are relative to (follows smax * c2 lazily)
        float l = 0.0f;         // sum of this thread's weights
        bool ok = true;
        const int my_steps = q == 0 ? steps[0] : steps[1], other_steps = q == 0 ? steps[1] : steps[0];
        // The units take turns at the exponentials (see attn_onepass.cuh); the barrier of a turn is the one that the two threads of a row exchange
        // their maxima by.  Every warp takes part in all of them, also after a wait has given up.
        const uint32_t turn_own = static_cast<uint32_t>(1 + q * 4 + quarter), turn_other = static_cast<uint32_t>(1 + (q ^ 1) * 4 + quarter);
        const int behind = q == 0 ? 1 : 0;
        auto take_turn = [&](int j) { ptx::named_sync(turn_own, j >= behind && j - behind < other_steps ? 128u : 64u); };
        auto pass_turn = [&](int j) {
            if (j + 1 - behind < other_steps) ptx::named_arrive(turn_other, 128u);
        };
        for (int j = 0; j < my_steps; ++j) {
            if (ok) ok = warp_wait(bar_of(offsetof(Barriers, s_full), q), static_cast<uint32_t>(j) & 1u, abort_flag, kSiteSFull);
            if (!ok) {
                take_turn(j);
                pass_turn(j);
                continue;
            }
            ptx::tc_fence_after_sync();
            const int tile_begin = key_tile(j, q) * kTile;
            const bool masked = seen_least - tile_begin < kTile;  // for some row of the tile
            const int valid = seen - tile_begin - half * kHalf;   // of this thread's columns
            float s[kHalf];
            {
                uint32_t r0[kChunk], r1[kChunk];
                ptx::tmem_ld_32x32b_x32(t_own, r0);
                ptx::tmem_ld_32x32b_x32(t_own + kChunk, r1);
                ptx::tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < kChunk; ++i) {
                    s[i] = __uint_as_float(r0[i]);
                    s[kChunk + i] = __uint_as_float(r1[i]);
                }
            }
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&bars->s_free[q]);
            if (masked) {
#pragma unroll
                for (int i = 0; i < kHalf; ++i)
                    if (i >= valid) s[i] = -3.0e38f;
            }
            // ---- row maximum, lazy offset ----
            float m0 = s[0], m1 = s[1], m2 = s[2], m3 = s[3];
#pragma unroll
            for (int i = 4; i < kHalf; i += 8) {
                m0 = ptx::max3(m0, s[i + 0], s[i + 1]);
                m1 = ptx::max3(m1, s[i + 2], s[i + 3]);
                if (i + 4 < kHalf) {
                    m2 = ptx::max3(m2, s[i + 4], s[i + 5]);
                    m3 = ptx::max3(m3, s[i + 6], s[i + 7]);
                }
            }
            m0 = ptx::max3(fmaxf(m0, m1), m2, m3);
            const uint32_t slot = static_cast<uint32_t>(j & 1) * (2 * kTile * 4);
            ptx::st_shared_f32(max_own + slot, m0);
            ok = static_cast<bool>(
                __all_sync(0xffffffffu, av1::wait_in_place(&bars->p_free[q], (static_cast<uint32_t>(j) & 1u) ^ 1u, abort_flag, kSitePFree)));
            take_turn(j);
            if (!ok) {
                pass_turn(j);
                continue;
            }
            smax = ptx::max3(smax, m0, ptx::ld_shared_f32(max_other + slot));
            const float mb_cand = fmaxf(smax * c2, -3.0e38f);
            const bool move = j == 0 || mb_cand - mb > kLazy;
            ptx::tc_fence_after_sync();
            uint32_t w[16];  // 32 keys of P on their way to tensor memory
            if (j == 0) {
                mb = mb_cand;
            } else if (__any_sync(0xffffffffu, move)) {
                const float alpha = move ? ptx::ex2_approx(mb - mb_cand) : 1.0f;
                if (move) mb = mb_cand;
                l *= alpha;
                ptx::tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < D / 2; c += 8) {  // 8 columns at a time: the row of scores stays in registers
                    uint32_t r[8];
                    ptx::tmem_ld_32x32b_x8(o_own + static_cast<uint32_t>(c), r);
                    ptx::tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
                    ptx::tmem_st_32x32b_x8(o_own + static_cast<uint32_t>(c), r);
                }
                ptx::tmem_wait_st();
            }
            // ---- weights: p = 2^(c2 s - mb) (below 2^8), row sum, bf16, into tensor memory ----
            const uint64_t nmb2 = ptx::pack2(-mb, -mb);
            uint64_t acc[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
            for (int g = 0; g < kHalf / 8; ++g) {
                float p[8];
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    float x0, x1;
                    ptx::unpack2(ptx::fma2(ptx::pack2(s[g * 8 + i], s[g * 8 + i + 1]), c2c2, nmb2), x0, x1);
                    p[i] = ptx::ex2_approx(x0);
                    p[i + 1] = ptx::ex2_approx(x1);
                    if (masked) {  // weight zero
                        p[i] = (g * 8 + i < valid) ? p[i] : 0.0f;
                        p[i + 1] = (g * 8 + i + 1 < valid) ? p[i + 1] : 0.0f;
                    }
                    acc[(i >> 1) & 3] = ptx::add2(acc[(i >> 1) & 3], ptx::pack2(p[i], p[i + 1]));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) w[(g & 3) * 4 + i] = ptx::pack_bf16x2(p[2 * i], p[2 * i + 1]);
                if (g == kPassAt) pass_turn(j);
                if ((g & 3) == 3) ptx::tmem_st_32x32b_x16(p_own + static_cast<uint32_t>((g >> 2) * 16), w);
            }
            float a0, a1, a2, a3;
            ptx::unpack2(ptx::add2(acc[0], acc[1]), a0, a1);
            ptx::unpack2(ptx::add2(acc[2], acc[3]), a2, a3);
            l += (a0 + a1) + (a2 + a3);
            ptx::tmem_wait_st();
            ptx::tc_fence_before_sync();  // orders P in tensor memory and the rescale of O before the MMAs that use them
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&bars->p_full[q]);
        }

        // ---- epilogue ----
        // The rows' statistics meet in shared memory: whole, those of the two threads of a row; split, of its four, who take D / 4 columns each of
        // 2^(mb_0 - mb) O_0 + 2^(mb_1 - mb) O_1.
        if (tiles > 0) {
            if (ok && my_steps > 0) ok = warp_wait(bar_of(offsetof(Barriers, o_full), q), 0, abort_flag, kSiteOFull);
            if (ok && !whole && other_steps > 0) ok = warp_wait(bar_of(offsetof(Barriers, o_full), q ^ 1), 0, abort_flag, kSiteOFull);
            if (ok) {
                stats[half * kTile + row] = l;  // (the maxima have all been read: the last product has them behind it)
                if (half == 0) stats[2 * kTile + row] = mb;
                __syncwarp();
                const uint32_t l_bar = whole ? bar_of(offsetof(Barriers, l_full), q) : bar_of(offsetof(Barriers, l_both), 0);
                ptx::mbar_arrive_if(l_bar, lane0);
                ok = warp_wait(l_bar, 0, abort_flag, kSiteLFull);
            }
        } else {
            ok = *reinterpret_cast<volatile unsigned int*>(&g_attnw_status) == 0u;
        }
        if (ok) {
            float l_row = 0.0f, top = -3.0e38f, f_own = 0.0f, f_other = 0.0f;
            if (tiles > 0) {
                const float* peer = reinterpret_cast<const float*>(smem + L::kStatOff) + (q ^ 1) * kUnitStats;
                const float l_own = l + stats[(half ^ 1) * kTile + row];
                l_row = l_own;
                top = mb;
                f_own = 1.0f;
                if (!whole) {
                    const float l_other = peer[row] + peer[kTile + row], mb_other = peer[2 * kTile + row];
                    // (a unit that has seen nothing of the row has a sum of zero, and its offset no say)
                    top = l_own > 0.0f ? (l_other > 0.0f ? fmaxf(mb, mb_other) : mb) : mb_other;
                    f_own = l_own > 0.0f ? ptx::ex2_approx(mb - top) : 0.0f;
                    f_other = l_other > 0.0f ? ptx::ex2_approx(mb_other - top) : 0.0f;
                    l_row = l_own * f_own + l_other * f_other;
                }
            }
            const bool joined = seg.segments > 1;  // by combine_kernel
            if (!joined) {
                const float inv = l_row > 0.0f ? 1.0f / l_row : 0.0f;
                f_own *= inv;
                f_other *= inv;
            }
            ptx::tc_fence_after_sync();
            const int in_tile = row / shape.group, g = row - in_tile * shape.group;
            const bool stored = in_tile < shape.tile_tokens && token < seg.tokens && (whole || tiles > 0 || q == 0);
            const int cols = whole || tiles == 0 ? D / 2 : D / 4;
            const int col0 = whole || tiles == 0 ? half * (D / 2) : (q * 2 + half) * (D / 4);
            const size_t out_row = static_cast<size_t>(seg.token0 + token) * shape.heads + seg.h * shape.group + g;
            const size_t part_row = static_cast<size_t>(seg.part) + token * shape.group + g;
            if (stored && half == 0 && (whole || q == 0)) {
                if (joined)
                    part_stats[part_row] = make_float2(top, l_row);
                else
                    store_lse(cache, shape, lse, lse2, out_row, seg.q_tile + (whole ? q : 0), seg.h, row, top, l_row);
            }
            __syncwarp();
            const uint32_t o_unit = t_quarter + L::o_col(q), o_peer = t_quarter + L::o_col(q ^ 1);
            const bool has_own = tiles > 0 && my_steps > 0, has_other = tiles > 0 && !whole && other_steps > 0;
#pragma unroll 1
            for (int c = col0; c < col0 + cols; c += 16) {
                float v[16];
                uint32_t o[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = 0.0f;
                if (has_own) {
                    ptx::tmem_ld_32x32b_x16(o_unit + static_cast<uint32_t>(c), o);
                    ptx::tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(o[i]) * f_own;
                }
                if (has_other) {
                    ptx::tmem_ld_32x32b_x16(o_peer + static_cast<uint32_t>(c), o);
                    ptx::tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = fmaf(__uint_as_float(o[i]), f_other, v[i]);
                }
                // (no branch around the rest of the loop: the loads of the next columns are the whole warp's)
                if (stored && joined) {
                    float4* dst = reinterpret_cast<float4*>(part_o + part_row * D + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) dst[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                } else if (stored) {
                    uint4* dst = reinterpret_cast<uint4*>(O + out_row * D + c);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        dst[i] = make_uint4(ptx::pack_bf16x2(v[8 * i], v[8 * i + 1]), ptx::pack_bf16x2(v[8 * i + 2], v[8 * i + 3]),
                                            ptx::pack_bf16x2(v[8 * i + 4], v[8 * i + 5]), ptx::pack_bf16x2(v[8 * i + 6], v[8 * i + 7]));
                }
                __syncwarp();
            }
        }
    }

    // ---- teardown: every role falls through to here, also after a wait gave up ----
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        // Unwinding: let the copies already in flight land before shared memory is released.
        if (warp == kProducer && lane == 0 && tiles > 0) {
            const long long t0 = clock64();
            auto land = [&](uint64_t* full, int stages, int loads) {
                for (int it = loads > stages ? loads - stages : 0; it < loads; ++it)
                    while (!ptx::mbar_try_wait(&full[it % stages], static_cast<uint32_t>(it / stages) & 1u) && clock64() - t0 < kWaitLimitCycles / 8) {
                    }
            };
            land(bars->k_full, L::kKStages, k_loads);
            land(bars->v_full, v_stages, v_loads);
            while (!ptx::mbar_try_wait(&bars->q_full, 0) && clock64() - t0 < kWaitLimitCycles / 8) {
            }
        }
    }
    if (warp == kMma) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

// Joins the segments of the rows that were cut: O = sum_s 2^(mb_s - top) O_s / sum_s 2^(mb_s - top) l_s, in the segments' order.  One warp a row.
constexpr int kJoinWarps = 8;

template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32)
combine_kernel(const __grid_constant__ paged::Cache cache, const __grid_constant__ Shape shape, const int* starts, const float* part_o, const float2* part_stats,
               const Plan* plan, __nv_bfloat16* O, float* lse, float* lse2) {
    __shared__ paged::Samples samples;
    ptx::grid_dependency_wait();
    if (*reinterpret_cast<volatile unsigned int*>(&g_attnw_status) != 0u) return;
    paged::sample_starts(&samples, starts, cache.sequences, kJoinWarps * 32);
    __syncthreads();
    const int lane = static_cast<int>(threadIdx.x & 31), warp = static_cast<int>(threadIdx.x >> 5);
    const long long rows = static_cast<long long>(shape.tokens) * shape.heads;
    constexpr int kCols = D / 32;
    for (long long id = static_cast<long long>(blockIdx.x) * kJoinWarps + warp; id < rows; id += static_cast<long long>(gridDim.x) * kJoinWarps) {
        const int t = static_cast<int>(id / shape.heads), head = static_cast<int>(id % shape.heads);
        int end;
        const int b = paged::owner_of(&samples, starts, cache.sequences, t, &end);
        if (b < 0) continue;
        const Plan p = plan[b];
        if (p.segments <= 1) continue;
        const int i = t - max(starts[b], 0), block = i / (2 * shape.tile_tokens), in_block = i - block * 2 * shape.tile_tokens;
        const int h = head / shape.group, g = head - h * shape.group;
        const long long first = p.part + (static_cast<long long>(block) * cache.kv_heads + h) * p.segments * p.rows + in_block * shape.group + g;
        float top = -3.0e38f, l = 0.0f, v[kCols] = {};
        for (int s = 0; s < p.segments; ++s) {
            const long long at = first + static_cast<long long>(s) * p.rows;
            const float2 st = part_stats[at];
            if (!(st.y > 0.0f)) continue;
            const float next = l > 0.0f ? fmaxf(top, st.x) : st.x;
            const float f_before = l > 0.0f ? ptx::ex2_approx(top - next) : 0.0f, f = ptx::ex2_approx(st.x - next);
            top = next;
            l = l * f_before + st.y * f;
            const float* src = part_o + at * D + lane * kCols;
#pragma unroll
            for (int c = 0; c < kCols; ++c) v[c] = fmaf(src[c], f, v[c] * f_before);
        }
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        __nv_bfloat16* dst = O + static_cast<size_t>(id) * D + lane * kCols;
#pragma unroll
        for (int c = 0; c < kCols; c += 2) *reinterpret_cast<uint32_t*>(dst + c) = ptx::pack_bf16x2(v[c] * inv, v[c + 1] * inv);
        if (lane == 0)
            store_lse(cache, shape, lse, lse2, static_cast<size_t>(id), p.q_tile + i / shape.tile_tokens, h, i % shape.tile_tokens * shape.group + g, top, l);
    }
}

}  // namespace pa
}  // namespace attnw
