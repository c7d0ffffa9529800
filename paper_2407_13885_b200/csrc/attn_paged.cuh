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
// A key tile is 128 keys of one or more pages, one TMA box (per 64 features) a page.
//
// What the host knows is the number of tokens, of sequences, and the width of the table; the lengths are on the device.  So there is one CTA an SM,
// and each works out for itself what it does: all blocks lie in a row, each as long as it costs, and the CTA has a stretch of it (Walk).  It may
// begin and end inside a block: then its unnormalised O, offset and sum go to a workspace, and combine_kernel joins them.  A CTA
// goes through its blocks without a stop: while its Softmax warps finish one, the tiles of the next arrive.
//
// Bound: HBM for single tokens over long caches (24 over up to 32768 keys, 32 heads on 8, d = 128, 1.8 GB: 284 us, 6.5 TB/s, as fast as a plain copy; 332 in
// a loop at the power cap).  For chunks tensor pipe and special function units, 1024 cycles each a tile of 128 x 128 at d = 128: 4 x 2048 tokens over some
// 6000 keys each 705 us, 1.03 PFLOP/s (817 in a loop, 0.89); both at 55 % in one such sequence, 50 % in 2 x 1024 over 4000, the rest are hand-overs between
// the roles and tiles cut by the diagonal.
#pragma once
#include <cstddef>

#include "attn_onepass.cuh"
#include "paged.cuh"

namespace attnw {
namespace pa {

using av1::kLazy;
using av1::kPassAt;

constexpr int kThreads = 640;
constexpr int kSmWarps = 16;  // Softmax warps: unit (2) x column half (2) x TMEM lane quarter (4)
constexpr int kProducer = 16;
constexpr int kMma = 17;         // the scores' issuer
constexpr int kMmaProduct = 18;  // the products'
constexpr int kScheduler = 19;
constexpr int kRoles = 19;       // warps that work on segments
// Costs are in keys of one query tile (two query tiles: twice that).
constexpr int kBlockCost = 2 * kTile;                // of a block besides: its set-up and its result
constexpr int kLeastCost = kBlockCost + 4 * kTile;   // of a CTA's stretch
constexpr int kLeastEven = 4 * kTile, kFewBlocks = 18;  // where blocks begin with a stretch (Walk::find)
constexpr int kLeastCut = 8;                         // key tiles of a block that may be cut
constexpr int kSlots = 4;                            // segments on their way from the scheduler to the others

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
    kSiteOFree = 121,
    kSiteQFree = 122,
    kSiteSegment = 123,
    kSiteSegmentFree = 124,
};

constexpr int kUnitStats = 4 * kTile;

template <int D>
struct Smem {
    static constexpr int kAtoms = D / 64;
    static constexpr int kAtomBytes = kTile * 128;          // 128 rows x 128 bytes
    static constexpr int kTileBytes = kAtoms * kAtomBytes;  // a Q, K or V tile
    // K and V tiles.  Each kind has a ring of its own, because it has an issuer of its own: an issuer waits for its tiles by the parity of a
    // stage's uses, and would take the use before the last for the last where the one between is the other's.
    static constexpr int kStages = (D == 128) ? 2 : 3;
    // Tensor memory as in attn_onepass.cuh: d = 64 has room for scores, O and P of both units, d = 128 for one buffer of scores that they use in turn.
    static constexpr bool kSharedS = D == 128;
    static __host__ __device__ constexpr uint32_t s_col(int q) { return kSharedS ? 0u : static_cast<uint32_t>(q * 256); }
    static __host__ __device__ constexpr uint32_t p_col(int q) { return kSharedS ? 128u + static_cast<uint32_t>(q * 64) : static_cast<uint32_t>(q * 256 + 192); }
    static __host__ __device__ constexpr uint32_t o_col(int q) { return kSharedS ? 256u + static_cast<uint32_t>(q * 128) : static_cast<uint32_t>(q * 256 + 128); }
    static constexpr int kQOff = 0;
    static constexpr int kKOff = kQOff + 2 * kTileBytes;  // (two query tiles: of one block, or of two split ones)
    static constexpr int kVOff = kKOff + kStages * kTileBytes;
    static constexpr int kStatOff = kVOff + kStages * kTileBytes;  // per unit: maxima, float [2 steps][2 halves][128 rows]
    static constexpr int kSumOff = kStatOff + 2 * 4 * kTile * 4;    // per unit: sums of both halves, offset, float [3][128]
    static constexpr int kLostOff = kSumOff + 2 * 3 * kTile * 4;    // per segment on its way, int [D]: (Barriers::lost)
    static constexpr int kBarOff = kLostOff + kSlots * D * 4;
    static constexpr int kBytes = kBarOff + 768;
    static constexpr int kDynamicBytes = kBytes + 1024;
};
static_assert(Smem<128>::kDynamicBytes <= 227 * 1024, "shared memory budget");

// A block, or a part of its keys, that a CTA works on.
struct Segment {
    int b;             // sequence, -1: there is no more
    int h;             // key head
    int token0;        // the block's first token and how many it has
    int tokens;
    int seen0;         // keys that the first token sees, not cut off below zero
    int length;        // keys of the sequence
    int tile0, tile1;  // key tiles
    int whole;
    int q_tile;        // the block's first query tile, among those of all sequences
    int part;          // the workspace's slot; -1: the segment is all of the block
};

struct Barriers {
    uint64_t q_full[2], q_free[2];  // per query tile's place
    uint64_t k_full[3], k_empty[3], v_full[3], v_empty[3];
    uint64_t s_full[2], s_free[2];  // per unit: scores written / read into registers (8 warps)
    uint64_t p_full[2], p_free[2];  // per unit: P written (8 warps) / read by its MMAs
    uint64_t o_full[2];             // per unit: every product of a segment complete
    uint64_t o_free;                // split: O of both units has been read (16 warps)
    uint64_t l_full[2], l_both;     // the row statistics are in shared memory: whole, per unit (8 warps); split (16)
    uint64_t seg_full[kSlots], seg_free[kSlots];
    uint32_t tmem_base;
    uint32_t abort_flag;
    // Does the segment have values that are not finite and that some of its rows see, but not all?  Then Smem::kLostOff has, for each feature, the first key
    // with such a value; rows that see it lose the feature.
    uint32_t lost[kSlots];
    Segment segment[kSlots];
};
static_assert(sizeof(Barriers) <= 768, "barrier block must fit its slot");

struct Shape {
    int tokens, heads, group;  // query heads of a key head
    int tile_tokens;           // tokens of a query tile: floor(128 / group)
    int part_rows;             // rows of a slot of the workspace; 0: no block can be cut
    int q_tiles;               // query tiles a key head, at most (of all sequences)
    int ctas;                  // of attn_paged_kernel
    int least;                 // sequences with fewer new tokens are attn_few_kernel's; 1: none are
};

// A sequence's blocks.
struct Share {
    int n, token0, seen0, length, blocks;  // new tokens, the first of them, (see Segment), blocks a key head

    __device__ __forceinline__ int tokens_of(const Shape& s, int r) const { return min(n - r * 2 * s.tile_tokens, 2 * s.tile_tokens); }
    __device__ __forceinline__ int seen_of(const Shape& s, int r) const {  // keys that block r's last token sees
        return min(max(seen0 + r * 2 * s.tile_tokens + tokens_of(s, r) - 1, 0), length);
    }
    // Cost of the first r blocks.  All but the last have as many tokens, and each sees that many more keys than the one in front.
    __device__ __forceinline__ long long cost_upto(const Shape& s, int r) const {
        if (r == 0) return 0;
        const long long step = 2 * s.tile_tokens, least = seen0 + step - 1;
        const int even = min(r, blocks - 1);
        const long long skip = least > 0 ? 0 : (step - least) / step, m = even - skip;  // blocks in front that see nothing
        long long cost = static_cast<long long>(r) * kBlockCost + (m > 0 ? 2 * (m * (least + skip * step) + step * (m * (m - 1) / 2)) : 0);
        if (r > even) cost += static_cast<long long>(seen_of(s, r - 1)) * (tokens_of(s, r - 1) > s.tile_tokens ? 2 : 1);
        return cost;
    }
};

__device__ __forceinline__ Share share_of(const paged::Cache& c, const Shape& s, const int* starts, int b) {
    Share r;
    const int s0 = starts[b], s1 = starts[b + 1];
    const int t0 = min(max(s0, 0), s.tokens), t1 = min(max(s1, 0), s.tokens);
    r.n = max(t1 - t0, 0);
    if (r.n < s.least) r.n = 0;
    r.token0 = t0;
    r.length = paged::length_of(c, b);
    const long long seen = static_cast<long long>(r.length) - (static_cast<long long>(s1) - t0) + 1;
    r.seen0 = static_cast<int>(min(max(seen, -(1ll << 30)), 1ll << 30));
    r.blocks = (r.n + 2 * s.tile_tokens - 1) / (2 * s.tile_tokens);
    return r;
}

// Are all sequences attn_few_kernel's (Shape::least)?  By all threads of a block, in front of everything else: then the launch has nothing to do, and what
// it would set up takes longer than to find that out.
__device__ __forceinline__ bool nothing_to_do(const paged::Cache& c, const Shape& s, const int* starts) {
    ptx::grid_dependency_wait();
    bool some = false;
    for (int b = static_cast<int>(threadIdx.x); b < c.sequences; b += static_cast<int>(blockDim.x))
        some = some || static_cast<long long>(starts[b + 1]) - starts[b] >= s.least;  // (no fewer than are within the tokens)
    return __syncthreads_or(some) == 0;
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

// (of numbers that are not negative; a division of 64 bits takes a hundred instructions)
__device__ __forceinline__ long long divided(long long a, long long b) {
    return (a | b) >> 32 == 0 ? static_cast<long long>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)) : a / b;
}

// How many of a block's key tiles lie in front of stretch `index`: its keys begin at `keys`, and it has `all` tiles, each of 2^shift keys' cost.
__device__ __forceinline__ int tiles_in_front(long long index, long long stretch, long long keys, int all, int shift) {
    const long long into = index * stretch - keys;
    if (into <= 0) return 0;
    const long long t = (into + (1ll << shift) - 1) >> shift;
    if (t >= all) return all;
    if (all < kLeastCut) return 2 * t < all ? 0 : all;
    const long long least = max(2ll, stretch >> (5 + shift));  // a shorter part goes to the CTA with the rest
    return t < least ? 0 : t > all - least ? all : static_cast<int>(t);
}

// What combine_kernel has to know of a block that was cut, from the CTA that has its last part.
struct Join {
    int b, h, token0, tokens, q_tile;
    int first, parts;  // the CTA with the first part; those from it to the last one's, 0: there is nothing to join
    int all, shift;    // (tiles_in_front)
    long long keys, stretch;
};

// A warp's way along the row of all blocks: sequence by sequence, key head by key head, block by block.  Lane i has the share of sequence
// b0 + i; everything else is the same in all lanes.
struct Walk {
    int lane, b0 = 0;
    Share mine;
    long long stretch;  // cost of a CTA's
    bool even;          // every block begins with a stretch, and costs whole ones
    // the block at hand
    int b = -1, h = 0, r = 0, q_tile0 = 0;  // b < 0: behind the last
    Share share;
    long long begin = 0;

    __device__ __forceinline__ void load(const paged::Cache& c, const Shape& s, const int* starts) {
        mine = {};
        if (b0 + lane < c.sequences) mine = share_of(c, s, starts, b0 + lane);
    }
    __device__ __forceinline__ void take(int from) {  // the share of lane `from`
        share.n = __shfl_sync(0xffffffffu, mine.n, from);
        share.token0 = __shfl_sync(0xffffffffu, mine.token0, from);
        share.seen0 = __shfl_sync(0xffffffffu, mine.seen0, from);
        share.length = __shfl_sync(0xffffffffu, mine.length, from);
        share.blocks = __shfl_sync(0xffffffffu, mine.blocks, from);
    }
    __device__ __forceinline__ int q_tiles_of(const Shape& s, const Share& x) const { return (x.n + s.tile_tokens - 1) / s.tile_tokens; }

    // The cost of everything, and the block that `index` stretches behind the beginning lies in.
    __device__ __forceinline__ void find(const paged::Cache& c, const Shape& s, const int* starts, long long index) {
        lane = static_cast<int>(threadIdx.x & 31);
        long long total = 0, blocks = 0;
        bool many = false;
        for (b0 = 0; b0 < c.sequences; b0 += 32) {
            load(c, s, starts);
            total += mine.cost_upto(s, mine.blocks) * c.kv_heads;
            blocks += static_cast<long long>(mine.blocks) * c.kv_heads;
            many = many || mine.blocks > 1;
        }
        total = warp_sum(total);
        blocks = warp_sum(blocks);
        stretch = max(static_cast<long long>(kLeastCost), divided(total + s.ctas - 1, s.ctas));
        // Few blocks: a CTA's way from one to the next takes as long as several key tiles, so none has parts of two.  Rounded up to whole stretches
        // they take at most a stretch more each.  (us per call without -> with it, d = 128, single tokens over 4000 keys: 8 blocks 19.3 -> 16.2, 16 20.3 -> 17.5,
        // 24 21.2 -> 20.1, 32 22.9 -> 25.4; over 16000: 4 blocks 32.8 -> 37.0, 8 34.1 -> 32.3, 16 37.5 -> 36.9, 18 39.4 -> 39.6, 24 45.4 -> 45.9, 32 54 -> 56; over
        // 2000, d = 64: 16 19.3 -> 17.3, 40 21.2 -> 20.6, 64 23.1 -> 26.1.  kFewBlocks is where the longest stop to gain.)
        even = !__any_sync(0xffffffffu, many) && blocks <= kFewBlocks && 2 * blocks <= s.ctas;
        if (even) stretch = max(static_cast<long long>(kLeastEven), divided(total + (s.ctas - blocks) - 1, s.ctas - blocks));
        const long long at = index * stretch;
        long long first = 0;
        int q_first = 0;
        for (b0 = 0; b0 < c.sequences; b0 += 32) {
            if (c.sequences > 32) load(c, s, starts);  // (else they are at hand)
            const long long a_head = even ? (mine.blocks > 0 ? rounded(mine.seen_of(s, 0) * weight_of(s, mine, 0)) : 0) : mine.cost_upto(s, mine.blocks);
            const long long cost = a_head * c.kv_heads;
            const long long end = first + warp_scan(cost, lane);
            const int q_tiles = q_tiles_of(s, mine), q_end = q_first + static_cast<int>(warp_scan(q_tiles, lane));
            const uint32_t here = __ballot_sync(0xffffffffu, at >= end - cost && at < end);
            if (here) {
                const int from = __ffs(here) - 1;
                take(from);
                b = b0 + from;
                q_tile0 = __shfl_sync(0xffffffffu, q_end - q_tiles, from);
                const long long seq_begin = __shfl_sync(0xffffffffu, end - cost, from), of_head = __shfl_sync(0xffffffffu, a_head, from);
                h = static_cast<int>(divided(at - seq_begin, of_head));
                begin = seq_begin + h * of_head;
                if (even) {
                    r = 0;
                    return;
                }
                int lo = 0, hi = share.blocks;  // cost_upto(lo) <= at - begin < cost_upto(hi)
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (share.cost_upto(s, mid) <= at - begin) lo = mid; else hi = mid;
                }
                r = lo;
                begin += share.cost_upto(s, r);
                return;
            }
            first = __shfl_sync(0xffffffffu, end, 31);
            q_first = __shfl_sync(0xffffffffu, q_end, 31);
        }
    }
    __device__ __forceinline__ void next(const paged::Cache& c, const Shape& s, const int* starts) {
        const long long keys = static_cast<long long>(weight(s)) * share.seen_of(s, r);
        begin += even ? rounded(keys) : kBlockCost + keys;
        if (++r < share.blocks) return;
        r = 0;
        if (++h < c.kv_heads) return;
        h = 0;
        q_tile0 += q_tiles_of(s, share);
        int from = b - b0 + 1;
        for (;;) {
            const uint32_t left = from < 32 ? __ballot_sync(0xffffffffu, mine.blocks > 0) >> from << from : 0u;
            if (left) {
                from = __ffs(left) - 1;
                take(from);
                b = b0 + from;
                return;
            }
            b0 += 32;
            if (b0 >= c.sequences) {
                b = -1;
                return;
            }
            load(c, s, starts);
            from = 0;
        }
    }
    __device__ __forceinline__ static int weight_of(const Shape& s, const Share& x, int r) { return x.tokens_of(s, r) > s.tile_tokens ? 2 : 1; }
    __device__ __forceinline__ int weight(const Shape& s) const { return weight_of(s, share, r); }
    __device__ __forceinline__ long long rounded(long long cost) const { return max(1ll, divided(cost + stretch - 1, stretch)) * stretch; }
    __device__ __forceinline__ long long keys() const { return begin + (even ? 0 : kBlockCost); }
    __device__ __forceinline__ int tiles(const Shape& s) const { return (share.seen_of(s, r) + kTile - 1) / kTile; }
    __device__ __forceinline__ int tiles_before(const Shape& s, long long index) const {
        return tiles_in_front(index, stretch, keys(), tiles(s), weight(s) == 2 ? 8 : 7);
    }
};

// Where the sums of a query tile's rows lie for mass_kernel: minus their logarithms to base 2, float [query tile][key head][128].
__device__ __forceinline__ size_t lse2_row(const paged::Cache& c, long long q_tile, int h) { return (static_cast<size_t>(q_tile) * c.kv_heads + h) * kTile; }

// For a segment, or its place: not cut short when another wait has given up, because all roles then still go through all segments, and soon.
__device__ __noinline__ bool segment_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t site) {
    const long long t0 = clock64();
    while (!__all_sync(0xffffffffu, ptx::mbar_try_wait(bar, parity))) {
        if (__any_sync(0xffffffffu, clock64() - t0 > 4 * kWaitLimitCycles)) {
            *abort_flag = 1;
            atomicCAS(&g_attnw_status, 0u, 0x80000000u | site);
            return false;
        }
    }
    return true;
}

// Are there values that are not finite among rows [first, last) of a tile of values?  By one warp.  A value times zero is zero or not a number, so sums of
// such products tell, at one instruction for two values.
template <int D>
__device__ __forceinline__ bool any_not_finite(const uint8_t* rows, int first, int last) {
    constexpr int kFlight = D == 128 ? 4 : 8;
    const __nv_bfloat162 zero = __float2bfloat162_rn(0.0f);
    __nv_bfloat162 sum[4] = {zero, zero, zero, zero};
    for (int i0 = first * 8 + static_cast<int>(threadIdx.x & 31); i0 - static_cast<int>(threadIdx.x & 31) < last * 8; i0 += 32 * kFlight) {
        uint4 v[kFlight][D / 64];
#pragma unroll
        for (int x = 0; x < kFlight; ++x)
#pragma unroll
            for (int a = 0; a < D / 64; ++a)
                v[x][a] = i0 + 32 * x < last * 8 ? *reinterpret_cast<const uint4*>(rows + a * kTile * 128 + (i0 + 32 * x) * 16) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int x = 0; x < kFlight; ++x)
#pragma unroll
            for (int a = 0; a < D / 64; ++a) {
                const uint32_t w[4] = {v[x][a].x, v[x][a].y, v[x][a].z, v[x][a].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w[e]), zero, sum[e]);
            }
    }
    const __nv_bfloat162 all = __hadd2(__hadd2(sum[0], sum[1]), __hadd2(sum[2], sum[3]));
    return __any_sync(0xffffffffu, __low2float(all) != 0.0f || __high2float(all) != 0.0f);
}

// The first keys of the features' values that are not finite, among rows [first, last) of a tile of values whose first key is `key0`; those values become
// zeros.  By one warp.
template <int D>
__device__ __noinline__ void take_out_values(uint8_t* rows, int first, int last, int key0, int* first_key) {
    for (int i = first * 8 + static_cast<int>(threadIdx.x & 31); i < last * 8; i += 32)
        for (int a = 0; a < D / 64; ++a) {
            uint16_t* x = reinterpret_cast<uint16_t*>(rows + a * kTile * 128 + i * 16);
            for (int e = 0; e < 8; ++e)
                if ((x[e] & 0x7f80u) == 0x7f80u) {
                    atomicMin(&first_key[a * 64 + ((i ^ (i >> 3)) & 7) * 8 + e], key0 + (i >> 3));  // (the swizzle of 128 bytes)
                    x[e] = 0;
                }
        }
}

// A row's result, at `dst`, where it sees such a value: not a number.
template <typename T>
__device__ __noinline__ void lose_features(const int* first_key, int col0, int cols, int seen, T* dst) {
    for (int c = col0; c < col0 + cols; ++c)
        if (first_key[c] < seen) dst[c] = T(__int_as_float(0x7fc00000));
}

// The logarithm of a row's sum l 2^top: to the caller, and for mass_kernel.  (A sum is zero, where the row sees nothing, or positive, or not a number, where a
// score was none: nowhere may the last be taken for the first.)
__device__ __forceinline__ void store_lse(const paged::Cache& c, const Shape& s, float* lse, float* lse2, size_t out_row, long long q_tile, int h, int row, float top,
                                          float l) {
    const float log2_sum = l != 0.0f ? top + ptx::lg2_approx(l) : __int_as_float(0xff800000);
    if (lse) lse[out_row] = 0.69314718055994531f * log2_sum;
    if (lse2 && q_tile < s.q_tiles) lse2[lse2_row(c, q_tile, h) + row] = -log2_sum;  // (the host's bound holds for tokens of one sequence each)
}

// APART: the kernel for few tokens has the other sequences (Shape::least > 1).  A form of its own, since the question at the beginning, asked at run time by all
// calls, cost 2 % (4 x 2048 tokens over some 6000 keys 705 -> 722 us).
template <int D, bool APART>
__global__ void __launch_bounds__(kThreads, 1)
attn_paged_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ paged::Cache cache, const __grid_constant__ Shape shape, const int* starts, float scale_log2e,
                  __nv_bfloat16* O, float* lse, float* lse2, float* part_o, float2* part_stats, Join* joins) {
    using L = Smem<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    Barriers* bars = reinterpret_cast<Barriers*>(smem + L::kBarOff);
    const uint32_t bar = ptx::smem_u32(bars);
    auto bar_of = [bar](size_t field, int n) { return bar + static_cast<uint32_t>(field) + 8u * static_cast<uint32_t>(n); };
    volatile uint32_t* abort_flag = &bars->abort_flag;
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    if constexpr (APART) {
        if (nothing_to_do(cache, shape, starts)) return;
    }

    // ---- set-up ------------------------------------------------------------------------------
    if (warp == kProducer && lane == 0) {
        for (int s = 0; s < 3; ++s) {
            ptx::mbar_init(&bars->k_full[s], 1);
            ptx::mbar_init(&bars->k_empty[s], 1);
            ptx::mbar_init(&bars->v_full[s], 1);
            ptx::mbar_init(&bars->v_empty[s], 1);
        }
        for (int q = 0; q < 2; ++q) {
            ptx::mbar_init(&bars->q_full[q], 1);
            ptx::mbar_init(&bars->q_free[q], 1);
            ptx::mbar_init(&bars->s_full[q], 1);
            ptx::mbar_init(&bars->s_free[q], 8);
            ptx::mbar_init(&bars->p_full[q], 8);
            ptx::mbar_init(&bars->p_free[q], 1);
            ptx::mbar_init(&bars->o_full[q], 2);  // (by its products, and by their issuer)
            ptx::mbar_init(&bars->l_full[q], 8);
        }
        ptx::mbar_init(&bars->o_free, kSmWarps);
        ptx::mbar_init(&bars->l_both, kSmWarps);
        for (int s = 0; s < kSlots; ++s) {
            ptx::mbar_init(&bars->seg_full[s], 1);
            ptx::mbar_init(&bars->seg_free[s], kRoles);
        }
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
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem_base = bars->tmem_base;
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
    int k_loads = 0, v_loads = 0, q_loads = 0;  // producer: tiles asked for
    // Every role goes through the same segments.  One whose wait has given up goes on without waiting or computing: the Softmax warps' turns
    // need each of them, and a segment's place is free when all have been there.
    uint32_t segments = 0;  // so far
    bool ok = true;
    static_assert(kSlots == 4, "two bits of a count, and the parity above them");
    auto segment = [&]() -> Segment& { return bars->segment[segments & 3u]; };
    auto next_segment = [&]() {
        return segment_wait(bar_of(offsetof(Barriers, seg_full), static_cast<int>(segments & 3u)), (segments >> 2) & 1u, abort_flag, kSiteSegment) && segment().b >= 0;
    };
    auto done_segment = [&]() {
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&bars->seg_free[segments & 3u]);
        ++segments;
    };
    // The key tiles of a unit: all of them (whole), or every other one.
    auto steps_of = [&](const Segment& seg, int q) { return seg.whole ? seg.tile1 - seg.tile0 : (seg.tile1 - seg.tile0 + 1 - q) / 2; };
    auto key_tile = [&](const Segment& seg, int j, int q) { return seg.tile0 + (seg.whole ? j : 2 * j + q); };

    if (warp == kScheduler) {
        // ================= scheduler: the CTA's segments, one after the other =================
        Walk walk;
        const long long cta = blockIdx.x;
        walk.find(cache, shape, starts, cta);
        Join join{};
        bool first_block = true;
        for (;;) {
            bool more = walk.b >= 0 && walk.begin < (cta + 1) * walk.stretch;
            Segment s{};
            s.b = -1;
            if (more) {
                const int all = walk.tiles(shape), t0 = walk.tiles_before(shape, cta), t1 = walk.tiles_before(shape, cta + 1);
                const int i0 = walk.r * 2 * shape.tile_tokens;
                if (first_block && t0 > 0 && t0 < t1 && t1 == all)  // the last part of a block that began in front
                    join = {walk.b, walk.h, walk.share.token0 + i0, walk.share.tokens_of(shape, walk.r), walk.q_tile0 + 2 * walk.r,
                            static_cast<int>(divided(walk.begin, walk.stretch)), 0, all, walk.weight(shape) == 2 ? 8 : 7, walk.keys(), walk.stretch};
                first_block = false;
                if (t0 < t1 || (all == 0 && walk.begin >= cta * walk.stretch)) {
                    s.b = walk.b;
                    s.h = walk.h;
                    s.token0 = walk.share.token0 + i0;
                    s.tokens = walk.share.tokens_of(shape, walk.r);
                    s.seen0 = walk.share.seen0 + i0;
                    s.length = walk.share.length;
                    s.tile0 = t0;
                    s.tile1 = t1;
                    s.whole = s.tokens > shape.tile_tokens;
                    s.q_tile = walk.q_tile0 + 2 * walk.r;
                    s.part = t1 - t0 == all ? -1 : 2 * static_cast<int>(cta) + (t0 > 0 ? 0 : 1);
                }
            }
            if (!more || s.b >= 0) {
                if (!segment_wait(bar_of(offsetof(Barriers, seg_free), static_cast<int>(segments & 3u)), ((segments >> 2) & 1u) ^ 1u, abort_flag, kSiteSegmentFree))
                    more = false;
                if (lane == 0) {
                    segment() = s;
                    ptx::mbar_arrive(&bars->seg_full[segments & 3u]);
                }
                __syncwarp();
                ++segments;
            }
            if (!more) break;
            walk.next(cache, shape, starts);
        }
        if (joins && lane == 0) {
            if (join.all > 0) join.parts = static_cast<int>(cta) - join.first + 1;
            joins[cta] = join;
        }
    } else if (warp == kProducer) {
        // ================= TMA producer: the first keys, Q, then the K and V tiles in the order the MMA issuers read them =========
        // A key tile is up to 8 pages; lane i fetches the part of its page and atom.  Places behind the sequence's length, and pages
        // outside the cache, are fetched from behind the cache: the tensor map fills in zeros.
        const uint64_t first_policy = ptx::policy_evict_first(), last_policy = ptx::policy_evict_last();
        const int page_shift = min(cache.page_shift, 7), parts = kTile >> page_shift;  // boxes of a tile, and keys (log2) of a box
        const int part = lane / L::kAtoms, atom = lane % L::kAtoms;
        const bool fetches = part < parts;
        const uint32_t q_bytes = static_cast<uint32_t>(L::kAtoms * shape.tile_tokens * shape.group * 128);
        Entry ek, ev, eq;
        for (; next_segment(); done_segment()) {
            const Segment& seg = segment();
            const int tiles = seg.tile1 - seg.tile0, tile0 = seg.tile0, length = seg.length, h = seg.h;
            const uint64_t policy = seg.tokens < shape.tile_tokens ? first_policy : last_policy;
            const int* table = cache.table + static_cast<size_t>(seg.b) * cache.table_width;
            if (!ok || tiles == 0) continue;
            auto place = [&](int kt) {  // the page's place among those of all heads
                const int at = kt * kTile + (part << page_shift);
                int p = -1;
                if (fetches && kt < seg.tile1 && at < length) p = table[at >> cache.page_shift];
                return static_cast<unsigned>(p) < static_cast<unsigned>(cache.pages) ? p * cache.kv_heads + h : cache.pages * cache.kv_heads;
            };
            auto load = [&](const CUtensorMap* map, uint32_t full, uint8_t* dst, int kt, int where) {
                if (lane == 0) ptx::mbar_expect_tx(full, static_cast<uint32_t>(L::kTileBytes));
                __syncwarp();
                if (fetches)
                    ptx::tma_load_3d(dst + atom * L::kAtomBytes + (part << page_shift) * 128, map, full, atom * 64,
                                     (kt * kTile) & ((1 << cache.page_shift) - 1) & ~(kTile - 1), where, policy);
                __syncwarp();
            };
            auto load_q = [&](int q) {
                ok = ok && warp_wait(bar_of(offsetof(Barriers, q_free), eq.stage), eq.phase ^ 1u, abort_flag, kSiteQFree);
                if (!ok) return;
                if (lane == 0) {
                    ptx::mbar_expect_tx(&bars->q_full[eq.stage], q_bytes);
                    for (int a = 0; a < L::kAtoms; ++a)
                        ptx::tma_load_4d(smem + L::kQOff + eq.stage * L::kTileBytes + a * L::kAtomBytes, &tm_q, &bars->q_full[eq.stage], a * 64, 0, h,
                                         seg.token0 + q * shape.tile_tokens);
                }
                __syncwarp();
                eq.next(2);
                ++q_loads;
            };
            // Both kinds in the order of the keys (split: the units take them in turn), each as soon as it has room.
            // The table is asked four tiles ahead: its answer takes 600 cycles, as long as a tile's boxes take to issue.
            constexpr int kAhead = 4;
            int k = 0, v = 0, where_k[kAhead], where_v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) where_k[i] = place(tile0 + i);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) where_v[i] = where_k[i];
            auto advance = [&](int (&where)[kAhead], int next) {
#pragma unroll
                for (int i = 0; i + 1 < kAhead; ++i) where[i] = where[i + 1];
                where[kAhead - 1] = place(tile0 + next + kAhead - 1);
            };
            long long idle_since = 0;
            bool q_here = false;
            auto ready = [&](size_t barrier, const Entry& e) { return __all_sync(0xffffffffu, ptx::mbar_test_wait(bar_of(barrier, e.stage), e.phase ^ 1u)); };
            auto load_queries = [&]() {
                load_q(0);
                if (seg.whole) load_q(1);
                q_here = true;
            };
            if (ready(offsetof(Barriers, q_free), eq)) load_queries();  // (beside the table's answer)
            while (ok && v < tiles) {
                bool idle = true;
                if (k < tiles && ready(offsetof(Barriers, k_empty), ek)) {
                    load(&tm_k, bar_of(offsetof(Barriers, k_full), ek.stage), smem + L::kKOff + ek.stage * L::kTileBytes, tile0 + k, where_k[0]);
                    ek.next(L::kStages);
                    ++k_loads;
                    if (!q_here) load_queries();
                    advance(where_k, ++k);
                    idle = false;
                }
                if (ok && v < k && ready(offsetof(Barriers, v_empty), ev)) {
                    load(&tm_v, bar_of(offsetof(Barriers, v_full), ev.stage), smem + L::kVOff + ev.stage * L::kTileBytes, tile0 + v, where_v[0]);
                    ev.next(L::kStages);
                    ++v_loads;
                    advance(where_v, ++v);
                    idle = false;
                }
                if (!idle) {
                    idle_since = 0;
                    continue;
                }
                __nanosleep(32);
                const long long now = clock64();
                if (idle_since == 0) idle_since = now;
                bool give_up = *abort_flag != 0u;
                if (!give_up && now - idle_since > kWaitLimitCycles) {
                    *abort_flag = 1;
                    atomicCAS(&g_attnw_status, 0u, 0x80000000u | kSiteProducerEmpty);
                    give_up = true;
                }
                ok = !__any_sync(0xffffffffu, give_up);
            }
        }
    } else if (warp == kMma || warp == kMmaProduct) {
        // ================= MMA issuers (warp-uniform loops, one elected lane issues): of scores, of products =================
        constexpr uint32_t idesc_s = ptx::umma_idesc_bf16_f32(kTile, kTile);
        constexpr uint32_t idesc_o = ptx::umma_idesc_bf16_f32(kTile, D) | (1u << 16);  // B operand MN-major
        const uint32_t base = ptx::smem_u32(smem);
        // Did an earlier launch give up?  Then this one computes and writes nothing.
        if (__any_sync(0xffffffffu, *reinterpret_cast<volatile unsigned int*>(&g_attnw_status) != 0u)) {
            *abort_flag = 1;
            ok = false;
        }
        Entry e;  // of the issuer's own ring
        auto arrived = [&](size_t full) { ok = ok && warp_wait(bar_of(full, e.stage), e.phase, abort_flag, kSiteMmaKFull); };
        auto release = [&](uint64_t* empty) {  // the tile may be replaced once the MMAs issued so far are complete
            if (ok && ptx::elect_one()) ptx::umma_commit(empty + e.stage);
            __syncwarp();
            e.next(L::kStages);
        };
        uint32_t done[2] = {0, 0};  // steps of each unit so far
        if (warp == kMma) {
            Entry eq;
            int last = 0;          // kSharedS: the unit whose scores the buffer holds, and the number of its step
            uint32_t last_step = 0xffffffffu;
            auto scores = [&](int q, uint32_t step, int q_place) {
                const int before = L::kSharedS ? last : q;
                const uint32_t before_step = L::kSharedS ? last_step : step - 1u;
                ok = ok && warp_wait(bar_of(offsetof(Barriers, s_free), before), before_step & 1u, abort_flag, kSiteMmaSFree);
                if (!ok) return;
                last = q;
                last_step = step;
                ptx::tc_fence_after_sync();
                const uint32_t d_tmem = tmem_base + L::s_col(q);
                const uint64_t a_desc = ptx::umma_desc_kmajor_sw128(base + static_cast<uint32_t>(L::kQOff + q_place * L::kTileBytes));
                const uint64_t b_desc = ptx::umma_desc_kmajor_sw128(base + static_cast<uint32_t>(L::kKOff + e.stage * L::kTileBytes));
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
            for (; next_segment(); done_segment()) {
                const Segment& seg = segment();
                const bool whole = seg.whole != 0;
                const int steps[2] = {steps_of(seg, 0), steps_of(seg, 1)};
                if (!ok || steps[0] == 0) continue;
                const int place0 = eq.stage, place1 = whole ? place0 ^ 1 : place0;
                for (int q = 0; q < (whole ? 2 : 1); ++q) {
                    ok = ok && warp_wait(bar_of(offsetof(Barriers, q_full), eq.stage), eq.phase, abort_flag, kSiteMmaQ);
                    eq.next(2);
                }
                for (int j = 0; ok && j < steps[0]; ++j) {
                    for (int q = 0; ok && q < (whole ? 1 : 2); ++q) {
                        if (j >= steps[q]) continue;
                        arrived(offsetof(Barriers, k_full));
                        scores(q, done[q] + static_cast<uint32_t>(j), q == 0 ? place0 : place1);
                        if (whole) scores(1, done[1] + static_cast<uint32_t>(j), place1);
                        release(bars->k_empty);
                    }
                }
                if (ok && ptx::elect_one()) {
                    ptx::umma_commit(&bars->q_free[place0]);
                    if (whole) ptx::umma_commit(&bars->q_free[place1]);
                }
                __syncwarp();
                done[0] += static_cast<uint32_t>(steps[0]);
                done[1] += static_cast<uint32_t>(steps[1]);
            }
        } else {
            uint32_t splits = 0;  // segments so far whose O both units read
            auto product = [&](const Segment& seg, int q, int j, int steps) {  // O += P V of step j
                ok = ok && warp_wait(bar_of(offsetof(Barriers, p_full), q), (done[q] + static_cast<uint32_t>(j)) & 1u, abort_flag, kSiteMmaPFull);
                if (!ok) return;
                ptx::tc_fence_after_sync();
                const uint32_t o_tmem = tmem_base + L::o_col(q), p_tmem = tmem_base + L::p_col(q);
                const uint64_t b_desc = av::umma_desc_mnmajor_sw128(base + static_cast<uint32_t>(L::kVOff + e.stage * L::kTileBytes), L::kAtomBytes);
                if (ptx::elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < kTile / 16; ++kk)  // 16 keys per instruction
                        ptx::umma_f16_ts(o_tmem, p_tmem + static_cast<uint32_t>(kk * 8), b_desc + static_cast<uint64_t>(kk * 16 * 128 >> 4), idesc_o,
                                         (j > 0 || kk > 0) ? 1u : 0u);
                    ptx::umma_commit(&bars->p_free[q]);
                    if (j + 1 == steps) ptx::umma_commit(&bars->o_full[q]);
                }
                __syncwarp();
                if (j + 1 == steps && lane == 0) ptx::mbar_arrive(&bars->o_full[q]);  // (what has been lost is written)
            };
            // A weight of zero does not silence a value that is not finite.  So the values that none of the block's tokens sees become zeros (those behind the
            // sequence's length may be anything), and among those that only some see (the keys of its own tokens) the ones that are not finite, which the
            // rows that do see them are told of.  What all see is left as it is.  (8 prompts of 512, 32 heads on 8, d = 128, 55.3 -> 57.2 us; 4 x 2048 tokens over
            // some 6000 keys 717 -> 721; single tokens have no such keys.)
            auto silence = [&](const Segment& seg, int kt) {
                const int seen_first = min(max(seg.seen0, 0), seg.length), seen_last = min(max(seg.seen0 + seg.tokens - 1, 0), seg.length);
                const int first = max(seen_first - kt * kTile, 0), last = min(seen_last - kt * kTile, kTile);
                if (!ok || first >= kTile) return;
                uint8_t* rows = smem + L::kVOff + e.stage * L::kTileBytes;
                if (any_not_finite<D>(rows, first, last)) {
                    int* first_key = reinterpret_cast<int*>(smem + L::kLostOff) + (segments & 3u) * D;
                    if (bars->lost[segments & 3u] == 0u) {
                        __syncwarp();
                        for (int c = lane; c < D; c += 32) first_key[c] = INT_MAX;
                        if (lane == 0) bars->lost[segments & 3u] = 1u;
                        __syncwarp();
                    }
                    take_out_values<D>(rows, first, last, kt * kTile, first_key);
                }
                for (int i = max(last, 0) * 8 + lane; i < kTile * 8; i += 32)
                    for (int a = 0; a < L::kAtoms; ++a) *reinterpret_cast<uint4*>(rows + a * L::kAtomBytes + i * 16) = make_uint4(0u, 0u, 0u, 0u);
                ptx::fence_proxy_async_smem();
                __syncwarp();
            };
            for (; next_segment(); done_segment()) {
                const Segment& seg = segment();
                const bool whole = seg.whole != 0;
                const int steps[2] = {steps_of(seg, 0), steps_of(seg, 1)};
                if (!ok || steps[0] == 0) continue;
                // (a unit's own warps have read its O when its P arrives; the other unit's, of a split segment, too?)
                if (splits > 0) ok = warp_wait(bar_of(offsetof(Barriers, o_free), 0), (splits - 1u) & 1u, abort_flag, kSiteOFree);
                if (lane == 0) bars->lost[segments & 3u] = 0u;
                __syncwarp();
                for (int j = 0; ok && j < steps[0]; ++j) {
                    for (int q = 0; ok && q < (whole ? 1 : 2); ++q) {
                        if (j >= steps[q]) continue;
                        arrived(offsetof(Barriers, v_full));
                        silence(seg, key_tile(seg, j, q));
                        product(seg, q, j, steps[q]);
                        if (whole) product(seg, 1, j, steps[1]);
                        release(bars->v_empty);
                    }
                }
                if (!whole) ++splits;
                done[0] += static_cast<uint32_t>(steps[0]);
                done[1] += static_cast<uint32_t>(steps[1]);
            }
        }
    } else {
        // ================= Softmax warps: two threads per query row, 64 key columns of a tile each =================
        const int q = warp >> 3;
        const int half = (warp >> 2) & 1;
        const int quarter = warp & 3;
        const uint32_t t_quarter = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        const uint32_t t_own = t_quarter + L::s_col(q) + static_cast<uint32_t>(half * kHalf);
        const uint32_t o_own = t_quarter + L::o_col(q) + static_cast<uint32_t>(half * (D / 2));  // this thread's D/2 columns of O
        const float c2 = fmaxf(scale_log2e, 1.2e-38f);  // (a scale of zero: any finite score counts as zero all the same)
        const uint64_t c2c2 = ptx::pack2(c2, c2);
        const int row = quarter * 32 + lane;
        const uint32_t max_own = ptx::smem_u32(smem + L::kStatOff) + static_cast<uint32_t>((q * 4 * kTile + half * kTile + row) * 4);
        static_assert(L::kStatOff % 1024 == 0 && kTile * 4 == 512, "the halves' maxima lie 512 bytes apart, at one bit");
        const uint32_t lane0 = lane == 0;
        const uint32_t p_own = t_quarter + L::p_col(q) + static_cast<uint32_t>(half * 32);  // its 64 keys of P
        // The units take turns at the exponentials (see attn_onepass.cuh); the barrier of a turn is the one that the two threads of a row exchange
        // their maxima by.  Every warp takes part in all of them, also after a wait has given up.
        const uint32_t turn_own = static_cast<uint32_t>(1 + q * 4 + quarter), turn_other = static_cast<uint32_t>(1 + (q ^ 1) * 4 + quarter);
        const int behind = q == 0 ? 1 : 0;
        uint32_t phases = 0;  // bit 0: parity of the unit's steps so far; 1, 2: of its segments with a step, of the other unit's; 3, 4: of whole and split segments
        for (; next_segment(); done_segment()) {
            const Segment& seg = segment();
            const bool whole = seg.whole != 0;
            const int my_steps = steps_of(seg, q), other_steps = steps_of(seg, q ^ 1);
            const int tiles = seg.tile1 - seg.tile0;
            // The row's token (of the block), and the keys that it sees.  A row that is none's gets what its place would.
            const int tile_first = whole ? q * shape.tile_tokens : 0;  // the first token of this unit's query tile
            const int seen = min(max(seg.seen0 + tile_first + row / shape.group, 0), seg.length);
            float smax = -3.0e38f;  // running maximum of the raw scores of this row (all columns)
            float mb = -3.0e38f;    // the offset the weights, l and O's row are relative to (follows smax * c2 lazily)
            float l = 0.0f;         // sum of this thread's weights
            auto take_turn = [&](int j) { ptx::named_sync(turn_own, j >= behind && j - behind < other_steps ? 128u : 64u); };
            auto pass_turn = [&](int j) {
                if (j + 1 - behind < other_steps) ptx::named_arrive(turn_other, 128u);
            };
            // A warp without a row of its own leaves the scores and the weights as they are: decoding uses few of 128 rows, and what the others
            // would compute costs power (24 tokens over up to 32768 keys 290 -> 283 us, in a loop of a second 334 -> 320).
            const bool idle = quarter * 32 >= min(seg.tokens - tile_first, shape.tile_tokens) * shape.group;
            const int tile_step = whole ? kTile : 2 * kTile;
            int tile_begin = key_tile(seg, 0, q) * kTile + half * kHalf;
            for (int j = 0; j < my_steps; ++j, tile_begin += tile_step) {
                const uint32_t parity = (phases + static_cast<uint32_t>(j)) & 1u;
                if (ok) ok = warp_wait(bar_of(offsetof(Barriers, s_full), q), parity, abort_flag, kSiteSFull);
                if (!ok) {
                    take_turn(j);
                    pass_turn(j);
                    continue;
                }
                if (idle) {  // (P of a step is announced behind the product of the step in front, by every warp)
                    if (lane == 0) ptx::mbar_arrive(&bars->s_free[q]);
                    ok = warp_wait(bar_of(offsetof(Barriers, p_free), q), parity ^ 1u, abort_flag, kSitePFree);
                    take_turn(j);
                    pass_turn(j);
                    if (ok && lane == 0) ptx::mbar_arrive(&bars->p_full[q]);
                    continue;
                }
                ptx::tc_fence_after_sync();
                const int valid = seen - tile_begin;  // of this thread's columns
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
                if (__any_sync(0xffffffffu, valid < kHalf)) {  // weight zero: c2 > 0 and the offset is finite.  (A branch: few tiles have it.)
                    asm volatile("" ::: "memory");
#pragma unroll
                    for (int i = 0; i < kHalf; ++i)
                        if (i >= valid) s[i] = __int_as_float(0xff800000);
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
                const uint32_t place = parity * (2 * kTile * 4);
                ptx::st_shared_f32(max_own + place, m0);
                ok = static_cast<bool>(__all_sync(0xffffffffu, av1::wait_in_place(&bars->p_free[q], parity ^ 1u, abort_flag, kSitePFree)));
                take_turn(j);
                if (!ok) {
                    pass_turn(j);
                    continue;
                }
                smax = ptx::max3(smax, m0, ptx::ld_shared_f32((max_own + place) ^ 512u));
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

            // ---- the segment's result ----
            // The rows' statistics meet in shared memory: whole, those of the two threads of a row; split, of its four, who take D / 4 columns each of
            // 2^(mb_0 - mb) O_0 + 2^(mb_1 - mb) O_1.
            float* const sums = reinterpret_cast<float*>(smem + L::kSumOff) + q * 3 * kTile + row;
            const float* const peer = reinterpret_cast<const float*>(smem + L::kSumOff) + (q ^ 1) * 3 * kTile + row;
            if (tiles > 0) {
                if (ok && my_steps > 0) ok = warp_wait(bar_of(offsetof(Barriers, o_full), q), (phases >> 1) & 1u, abort_flag, kSiteOFull);
                if (ok && !whole && other_steps > 0) ok = warp_wait(bar_of(offsetof(Barriers, o_full), q ^ 1), (phases >> 2) & 1u, abort_flag, kSiteOFull);
                if (ok) {
                    // (nobody reads the last segment's any more: this one's products came behind that)
                    if (my_steps > 0) {
                        sums[half * kTile] = l;
                        if (half == 0) sums[2 * kTile] = mb;
                    }
                    __syncwarp();
                    const uint32_t l_bar = whole ? bar_of(offsetof(Barriers, l_full), q) : bar_of(offsetof(Barriers, l_both), 0);
                    ptx::mbar_arrive_if(l_bar, lane0);
                    ok = warp_wait(l_bar, (phases >> (whole ? 3 : 4)) & 1u, abort_flag, kSiteLFull);
                }
            } else if (ok) {
                ok = !__any_sync(0xffffffffu, *reinterpret_cast<volatile unsigned int*>(&g_attnw_status) != 0u);
            }
            if (ok) {
                float l_row = 0.0f, top = -3.0e38f, f_own = 0.0f, f_other = 0.0f;
                if (tiles > 0) {
                    const float l_own = my_steps > 0 ? l + sums[(half ^ 1) * kTile] : 0.0f;
                    l_row = l_own;
                    top = mb;
                    f_own = 1.0f;
                    if (!whole) {
                        const float l_other = other_steps > 0 ? peer[0] + peer[kTile] : 0.0f, mb_other = other_steps > 0 ? peer[2 * kTile] : mb;
                        // (a unit that has seen nothing of the row has a sum of zero, and its offset no say)
                        top = l_own != 0.0f ? (l_other != 0.0f ? fmaxf(mb, mb_other) : mb) : mb_other;
                        f_own = l_own != 0.0f ? ptx::ex2_approx(mb - top) : 0.0f;
                        f_other = l_other != 0.0f ? ptx::ex2_approx(mb_other - top) : 0.0f;
                        l_row = l_own * f_own + l_other * f_other;
                    }
                }
                const bool joined = seg.part >= 0;  // by combine_kernel
                if (!joined) {
                    const float inv = l_row != 0.0f ? 1.0f / l_row : 0.0f;
                    f_own *= inv;
                    f_other *= inv;
                }
                ptx::tc_fence_after_sync();
                const int in_tile = row / shape.group;  // the row's token in its query tile
                const int token = tile_first + in_tile, g = row - in_tile * shape.group;
                const bool alone = whole || tiles == 0;  // a unit's threads have their D / 2 columns; tiles == 0, split: unit 0's
                const bool stored = in_tile < shape.tile_tokens && token < seg.tokens && (whole || tiles > 0 || q == 0);
                const int cols = alone ? D / 2 : D / 4;
                const int col0 = alone ? half * (D / 2) : (q * 2 + half) * (D / 4);
                const size_t out_row = static_cast<size_t>(seg.token0 + token) * shape.heads + seg.h * shape.group + g;
                const size_t part_row = static_cast<size_t>(max(seg.part, 0)) * shape.part_rows + token * shape.group + g;
                if (stored && half == 0 && (whole || q == 0)) {
                    if (joined)
                        part_stats[part_row] = make_float2(top, l_row);
                    else
                        store_lse(cache, shape, lse, lse2, out_row, seg.q_tile + (whole ? q : 0), seg.h, row, top, l_row);
                }
                __syncwarp();
                const uint32_t o_unit = t_quarter + L::o_col(q), o_peer = t_quarter + L::o_col(q ^ 1);
                const bool has_own = my_steps > 0, has_other = !whole && other_steps > 0;
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
                if (tiles > 0 && stored && bars->lost[segments & 3u] != 0u) {
                    const int* first_key = reinterpret_cast<const int*>(smem + L::kLostOff) + (segments & 3u) * D;
                    if (joined)
                        lose_features(first_key, col0, cols, seen, part_o + part_row * D);
                    else
                        lose_features(first_key, col0, cols, seen, O + out_row * D);
                }
                ptx::tc_fence_before_sync();
                __syncwarp();
                if (!whole && tiles > 0) ptx::mbar_arrive_if(bar_of(offsetof(Barriers, o_free), 0), lane0);
            }
            if (tiles > 0) {
                phases ^= (my_steps & 1) | (my_steps > 0 ? 2u : 0u) | (other_steps > 0 ? 4u : 0u) | (whole ? 8u : 16u);
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
            land(bars->k_full, L::kStages, k_loads);
            land(bars->v_full, L::kStages, v_loads);
            land(bars->q_full, 2, q_loads);
        }
    }
    if (warp == kMma) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem_base, kTmemCols);
    }
}

// Joins the parts of the blocks that stretches of attn_paged_kernel's CTAs cut: O = sum_s 2^(mb_s - top) O_s / sum_s 2^(mb_s - top) l_s, in the order of
// the parts.  CTA (c, y): the block whose last part CTA c + 1 had, and of its rows a share.  Where a block has few rows (decoding) several warps take a row's parts in turn.
constexpr int kJoinWarps = 8;
constexpr int kJoinRows = 4;

template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32)
combine_kernel(const __grid_constant__ paged::Cache cache, const __grid_constant__ Shape shape, const int* starts, const float* part_o, const float2* part_stats,
               const Join* joins, __nv_bfloat16* O, float* lse, float* lse2) {
    constexpr int kCols = D / 32;
    __shared__ uint8_t slot_of[256];  // of each part: 0, 1; 2: the CTA has none of the block
    __shared__ float sums[kJoinWarps][32 * kCols + 2];
    ptx::grid_dependency_wait();
    if (shape.least > 1 && nothing_to_do(cache, shape, starts)) return;  // (and nobody has written a Join)
    const int lane = static_cast<int>(threadIdx.x & 31), warp = static_cast<int>(threadIdx.x >> 5);
    const Join x = joins[blockIdx.x + 1];
    if (*reinterpret_cast<volatile unsigned int*>(&g_attnw_status) != 0u || x.parts == 0) return;
    for (int i = static_cast<int>(threadIdx.x); i < x.parts; i += kJoinWarps * 32) {
        const int t0 = tiles_in_front(x.first + i, x.stretch, x.keys, x.all, x.shift), t1 = tiles_in_front(x.first + i + 1, x.stretch, x.keys, x.all, x.shift);
        slot_of[i] = t0 >= t1 ? 2 : t0 > 0 ? 0 : 1;
    }
    __syncthreads();
    const int rows = x.tokens * shape.group;
    // A part's offset and sum, and this lane's columns of its O, into what a row has so far.
    auto add = [](float2 st, const float (&o)[kCols], float& top, float& l, float (&v)[kCols]) {
        if (st.y == 0.0f) return;
        const float next = l != 0.0f ? fmaxf(top, st.x) : st.x;
        const float f_before = l != 0.0f ? ptx::ex2_approx(top - next) : 0.0f, f_new = ptx::ex2_approx(st.x - next);
        top = next;
        l = l * f_before + st.y * f_new;
#pragma unroll
        for (int c = 0; c < kCols; ++c) v[c] = fmaf(o[c], f_new, v[c] * f_before);
    };
    auto load = [&](int i, int r, float2& st, float (&o)[kCols]) {
        const int slot = i < x.parts && r < rows ? slot_of[i] : 2;
        st = make_float2(0.0f, 0.0f);
        if (slot == 2) return;
        const size_t at = static_cast<size_t>(2 * (x.first + i) + slot) * shape.part_rows + r;
        st = part_stats[at];
        const float* src = part_o + at * D + lane * kCols;
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[c] = src[c];
    };
    auto store = [&](int r, float top, float l, const float (&v)[kCols]) {
        const int token = r / shape.group, g = r - token * shape.group;
        const size_t out_row = static_cast<size_t>(x.token0 + token) * shape.heads + x.h * shape.group + g;
        const float inv = l != 0.0f ? 1.0f / l : 0.0f;
        __nv_bfloat16* dst = O + out_row * D + lane * kCols;
#pragma unroll
        for (int c = 0; c < kCols; c += 2) *reinterpret_cast<uint32_t*>(dst + c) = ptx::pack_bf16x2(v[c] * inv, v[c + 1] * inv);
        if (lane == 0)
            store_lse(cache, shape, lse, lse2, out_row, x.q_tile + token / shape.tile_tokens, x.h, token % shape.tile_tokens * shape.group + g, top, l);
    };
    int each = 1;  // warps a row
    while (each < kJoinWarps && 2 * each * rows <= kJoinWarps && 4 * each < x.parts) each *= 2;
    if (each == 1) {
        // a warp takes kJoinRows rows at once, two parts (most blocks have no more) of each on their way
        for (int r0 = (static_cast<int>(blockIdx.y) * kJoinWarps + warp) * kJoinRows; r0 < rows; r0 += static_cast<int>(gridDim.y) * kJoinWarps * kJoinRows) {
            float top[kJoinRows], l[kJoinRows], v[kJoinRows][kCols];
#pragma unroll
            for (int k = 0; k < kJoinRows; ++k) {
                top[k] = -3.0e38f;
                l[k] = 0.0f;
#pragma unroll
                for (int c = 0; c < kCols; ++c) v[k][c] = 0.0f;
            }
            for (int i = 0; i < x.parts; i += 2) {
                float2 st[2][kJoinRows];
                float o[2][kJoinRows][kCols];
#pragma unroll
                for (int f = 0; f < 2; ++f)
#pragma unroll
                    for (int k = 0; k < kJoinRows; ++k) load(i + f, r0 + k, st[f][k], o[f][k]);
#pragma unroll
                for (int f = 0; f < 2; ++f)
#pragma unroll
                    for (int k = 0; k < kJoinRows; ++k) add(st[f][k], o[f][k], top[k], l[k], v[k]);
            }
#pragma unroll
            for (int k = 0; k < kJoinRows; ++k)
                if (r0 + k < rows) store(r0 + k, top[k], l[k], v[k]);
        }
        return;
    }
    if (blockIdx.y > 0) return;  // few rows: the first CTA has all of them
    const int r = warp / each, share = warp % each;
    float top = -3.0e38f, l = 0.0f, v[kCols] = {};
    constexpr int kFlight = 4;
    for (int i0 = share; i0 < x.parts; i0 += kFlight * each) {
        float2 st[kFlight];
        float o[kFlight][kCols];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) load(i0 + f * each, r, st[f], o[f]);
#pragma unroll
        for (int f = 0; f < kFlight; ++f) add(st[f], o[f], top, l, v);
    }
    sums[warp][32 * kCols] = top;
    sums[warp][32 * kCols + 1] = l;
#pragma unroll
    for (int c = 0; c < kCols; ++c) sums[warp][lane * kCols + c] = v[c];
    __syncthreads();
    if (share > 0 || r >= rows) return;
    for (int w = warp + 1; w < warp + each; ++w) {
        float o[kCols];
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[c] = sums[w][lane * kCols + c];
        add(make_float2(sums[w][32 * kCols], sums[w][32 * kCols + 1]), o, top, l, v);
    }
    store(r, top, l, v);
}

}  // namespace pa
}  // namespace attnw
