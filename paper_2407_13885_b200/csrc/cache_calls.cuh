// Checks and launches of the calls around a paged cache (attnw_rope, attnw_cache_append, attn_paged, attnw_cache_evict).  Part of
// attnw_api.cu, whose helpers it uses.
#pragma once

namespace {

// Where a strided [n0, n1, n2, row] array lies: its bytes from `p` on, and the largest stride's period.  Strides in elements, as many
// dimensions as sizes; a dimension of size 1 has no say.
struct Extent {
    uintptr_t begin = 0, end = 0;
    unsigned long long pitch = 0;  // bytes from one token (the dimension `by`) to the next, 0 if there is one token
    unsigned long long inner = 0;  // bytes that the rows of one token, or of tokens whole pitches apart, cover of a pitch
};

// Strides of a kernel's operand: not negative, and rows on 16-byte boundaries.  `least`: of a dimension with more than one index, in elements; 0 where it
// may be broadcast, the length of a row where rows are written, which then must not lie on one another (nor along two dimensions alike).  Returns an attnw_status.
int check_strides(const long long* strides, const long long* sizes, int n, int esize, long long least) {
    for (int i = 0; i < n; ++i) {
        if (sizes[i] <= 1) continue;
        if (strides[i] < 0 || strides[i] > (1ll << 47) / (sizes[i] - 1)) return ATTNW_ERR_BAD_SHAPE;  // (an array lies within 2^48 elements)
        if (strides[i] * esize % 16 != 0) return ATTNW_ERR_MISALIGNED;
        if (strides[i] < least) return ATTNW_ERR_BAD_SHAPE;
        for (int j = 0; j < i; ++j)
            if (least > 1 && sizes[j] > 1 && strides[j] == strides[i]) return ATTNW_ERR_BAD_SHAPE;
    }
    return ATTNW_OK;
}

// `sizes` and `strides` of [.., token, .., d] without d; `token` is the index of the dimension whose rows lie side by side.
Extent extent_of(const void* p, const long long* strides, const long long* sizes, int n, int token, long long d, int esize) {
    Extent e;
    unsigned long long all = static_cast<unsigned long long>(d) * esize, inner = all;
    for (int i = 0; i < n; ++i) {
        const unsigned long long span = sizes[i] > 1 ? static_cast<unsigned long long>(sizes[i] - 1) * strides[i] * esize : 0;
        all += span;
        const bool whole_pitches = sizes[token] > 1 && strides[token] > 0 && strides[i] % strides[token] == 0;
        if (i != token && !whole_pitches) inner += span;
    }
    e.begin = reinterpret_cast<uintptr_t>(p);
    e.end = e.begin + all;
    e.pitch = sizes[token] > 1 ? static_cast<unsigned long long>(strides[token]) * esize : 0;
    e.inner = inner;
    return e;
}

// May the two share a byte?  Operands cut out of one array of tokens (queries, keys and values side by side) do not where their columns
// differ, although their extents cross.
bool may_overlap(const Extent& a, const Extent& b) {
    if (a.end <= b.begin || b.end <= a.begin) return false;
    if (a.pitch == 0 || a.pitch != b.pitch || a.inner > a.pitch || b.inner > a.pitch) return true;
    const unsigned long long at = (b.begin >= a.begin ? b.begin - a.begin : a.pitch - (a.begin - b.begin) % a.pitch) % a.pitch;
    return at < a.inner || at + b.inner > a.pitch;
}

int check_turn(const void* frequencies, int rotary, int d, int layout, float amplitude) {
    if (layout != 0 && layout != 1) return ATTNW_ERR_BAD_SHAPE;
    if (!std::isfinite(amplitude)) return ATTNW_ERR_BAD_SHAPE;
    if (rotary < 0 || rotary > d) return ATTNW_ERR_BAD_SHAPE;
    if (rotary % 16 != 0) return ATTNW_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(frequencies) % 8 != 0) return ATTNW_ERR_MISALIGNED;
    return ATTNW_OK;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Heads that one thread walks with its cosines and sines: all of them where the tokens alone fill the device (1024 threads an SM), fewer
// otherwise, since latency is what a small call spends its time on.
int heads_each(long long threads, int heads, int sm_count, int most) {
    const long long groups = std::max(1ll, static_cast<long long>(sm_count) * 1024 / std::max(1ll, threads));
    return static_cast<int>(std::min(static_cast<long long>(most), (heads + groups - 1) / groups));
}

template <typename T>
int rope_entry(const void* X, const int* positions, const double* frequencies, void* Y, int B, int H, int N, int d, int rotary,
               const long long* x_strides, const long long* y_strides, int layout, int inverse, float amplitude, void* stream) {
    if (!X || !positions || (rotary > 0 && !frequencies) || !Y || !x_strides || !y_strides) return ATTNW_ERR_NULL_POINTER;
    if (B < 1 || H < 1 || N < 1 || d < 1 || H > 65535) return ATTNW_ERR_BAD_SHAPE;
    if (d != 64 && d != 128) return ATTNW_ERR_UNSUPPORTED;
    int rc = check_turn(frequencies, rotary, d, layout, amplitude);
    if (rc != ATTNW_OK) return rc;
    const long long sizes[3] = {B, H, N};
    rc = check_strides(x_strides, sizes, 3, sizeof(T), 0);
    if (rc == ATTNW_OK) rc = check_strides(y_strides, sizes, 3, sizeof(T), d);
    if (rc != ATTNW_OK) return rc;
    if (!aligned16(X) || !aligned16(Y) || !aligned4(positions)) return ATTNW_ERR_MISALIGNED;
    const Extent x = extent_of(X, x_strides, sizes, 3, 2, d, sizeof(T)), y = extent_of(Y, y_strides, sizes, 3, 2, d, sizeof(T));
    bool in_place = X == Y;
    for (int i = 0; i < 3; ++i) in_place = in_place && (sizes[i] == 1 || x_strides[i] == y_strides[i]);
    if (!in_place && may_overlap(x, y)) return ATTNW_ERR_ALIASING;
    const unsigned long long tokens = static_cast<unsigned long long>(B) * N;
    const Extent index[2] = {extent_of(positions, sizes, sizes, 0, 0, static_cast<long long>(tokens), 4), extent_of(frequencies, sizes, sizes, 0, 0, rotary / 2, 8)};
    for (const Extent& e : index)
        if (y.begin < e.end && e.begin < y.end) return ATTNW_ERR_ALIASING;
    DeviceInfo* dev = nullptr;
    rc = current_device(&dev);
    if (rc != ATTNW_OK) return rc;
    const int parts = d / (2 * rope::Vec<T>::kN);
    const long long threads = static_cast<long long>(tokens) * parts, blocks = (threads + rope::kThreads - 1) / rope::kThreads;
    if (blocks > INT_MAX) return ATTNW_ERR_BAD_SHAPE;
    const int each = heads_each(threads, H, dev->sm_count, 8);
    const rope::Rows rows{X, Y, x_strides[0], x_strides[2], x_strides[1], y_strides[0], y_strides[2], y_strides[1], H};
    const rope::Turn turn{positions, frequencies, rotary, amplitude, inverse ? -1.0f : 1.0f};
    const auto kernel = layout == 0 ? rope::rope_kernel<T, true> : rope::rope_kernel<T, false>;
    if (launch_overlapped_3d(kernel, static_cast<unsigned>(blocks), static_cast<unsigned>((H + each - 1) / each), 1, rope::kThreads,
                             static_cast<cudaStream_t>(stream), rows, turn, static_cast<long long>(tokens), N, parts, each) != cudaSuccess) {
        (void)cudaGetLastError();
        return ATTNW_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return ATTNW_OK;
}

// Host-only checks of the cache's description.
int check_cache(const attnw_cache* c) {
    if (!c || !c->K || !c->V || !c->table || !c->lengths) return ATTNW_ERR_NULL_POINTER;
    if (c->pages < 1 || c->kv_heads < 1 || c->page < 1 || c->d < 1 || c->sequences < 1 || c->table_width < 1) return ATTNW_ERR_BAD_SHAPE;
    if (c->d != 64 && c->d != 128) return ATTNW_ERR_UNSUPPORTED;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1)) != 0) return ATTNW_ERR_UNSUPPORTED;
    if (static_cast<long long>(c->pages) * c->kv_heads >= INT_MAX) return ATTNW_ERR_BAD_SHAPE;
    if (static_cast<long long>(c->sequences) * c->kv_heads > 65535) return ATTNW_ERR_BAD_SHAPE;
    if (static_cast<long long>(c->table_width) * c->page > (1 << 28)) return ATTNW_ERR_BAD_SHAPE;
    if (!aligned16(c->K) || !aligned16(c->V) || !aligned4(c->table) || !aligned4(c->lengths)) return ATTNW_ERR_MISALIGNED;
    return ATTNW_OK;
}

struct Span {
    const void* p;
    unsigned long long bytes;
};
unsigned long long cache_bytes(const attnw_cache* c) {
    return 2ull * static_cast<unsigned long long>(c->pages) * c->kv_heads * c->page * c->d;
}
bool crosses(const Span& a, const Span& b) { return a.p && b.p && overlaps(a.p, a.bytes, b.p, b.bytes); }
Span span_of(const Extent& e) { return {reinterpret_cast<const void*>(e.begin), static_cast<unsigned long long>(e.end - e.begin)}; }

paged::Cache view_of(const attnw_cache* c) {
    int shift = 0;
    while ((1 << shift) < c->page) ++shift;
    return {static_cast<__nv_bfloat16*>(c->K), static_cast<__nv_bfloat16*>(c->V), c->table, c->lengths, c->pages, c->kv_heads, shift, c->d, c->sequences,
            c->table_width};
}

int append_entry(const attnw_cache* c, const void* Q, const void* K, const void* V, void* Q_out, const long long* strides, const int* starts,
                 const int* positions, const double* frequencies, int tokens, int heads, int rotary, int layout, float amplitude, void* stream) {
    int rc = check_cache(c);
    if (rc != ATTNW_OK) return rc;
    if (!K || !V || !strides || !starts || (!Q) != (!Q_out) || (rotary > 0 && (!positions || !frequencies))) return ATTNW_ERR_NULL_POINTER;
    if (tokens < 1 || (Q && heads < 1) || heads > 65535) return ATTNW_ERR_BAD_SHAPE;
    rc = check_turn(frequencies, rotary, c->d, layout, amplitude);
    if (rc != ATTNW_OK) return rc;
    const long long q_sizes[2] = {tokens, Q ? heads : 1}, kv_sizes[2] = {tokens, c->kv_heads};
    rc = check_strides(strides + 2, kv_sizes, 2, 2, 0);
    if (rc == ATTNW_OK) rc = check_strides(strides + 4, kv_sizes, 2, 2, 0);
    if (rc == ATTNW_OK && Q) rc = check_strides(strides, q_sizes, 2, 2, 0);
    if (rc == ATTNW_OK && Q) rc = check_strides(strides + 6, q_sizes, 2, 2, c->d);
    if (rc != ATTNW_OK) return rc;
    if (!aligned16(K) || !aligned16(V) || !aligned16(Q) || !aligned16(Q_out) || !aligned4(starts) || !aligned4(positions)) return ATTNW_ERR_MISALIGNED;
    const Extent k = extent_of(K, strides + 2, kv_sizes, 2, 0, c->d, 2), v = extent_of(V, strides + 4, kv_sizes, 2, 0, c->d, 2);
    const Span caches[2] = {{c->K, cache_bytes(c)}, {c->V, cache_bytes(c)}};
    const Span index[5] = {{c->table, 4ull * c->sequences * c->table_width}, {c->lengths, 4ull * c->sequences}, {starts, 4ull * (c->sequences + 1ull)},
                           {positions, 4ull * tokens}, {frequencies, 4ull * rotary}};
    if (crosses(caches[0], caches[1])) return ATTNW_ERR_ALIASING;
    for (const Span& s : caches) {
        if (crosses(s, span_of(k)) || crosses(s, span_of(v))) return ATTNW_ERR_ALIASING;
        for (const Span& i : index)
            if (crosses(s, i)) return ATTNW_ERR_ALIASING;
    }
    if (Q) {
        const Extent q = extent_of(Q, strides, q_sizes, 2, 0, c->d, 2), o = extent_of(Q_out, strides + 6, q_sizes, 2, 0, c->d, 2);
        bool in_place = Q == Q_out;
        for (int i = 0; i < 2; ++i) in_place = in_place && (q_sizes[i] == 1 || strides[i] == strides[6 + i]);
        if ((!in_place && may_overlap(q, o)) || may_overlap(k, o) || may_overlap(v, o)) return ATTNW_ERR_ALIASING;
        for (const Span& s : caches)
            if (crosses(s, span_of(q)) || crosses(s, span_of(o))) return ATTNW_ERR_ALIASING;
        for (const Span& i : index)
            if (crosses(span_of(o), i)) return ATTNW_ERR_ALIASING;
    }
    DeviceInfo* dev = nullptr;
    rc = current_device(&dev);
    if (rc != ATTNW_OK) return rc;
    const int parts = c->d / 16;
    const long long threads = static_cast<long long>(tokens) * parts, blocks = (threads + rope::kThreads - 1) / rope::kThreads;
    const int rows = (Q ? heads : 0) + 2 * c->kv_heads, each = std::min(heads_each(threads, rows, dev->sm_count, 16), std::max(Q ? heads : 1, c->kv_heads));
    const int q_groups = Q ? (heads + each - 1) / each : 0, kv_groups = (c->kv_heads + each - 1) / each;
    if (q_groups + 2 * kv_groups > 65535) return ATTNW_ERR_BAD_SHAPE;
    const rope::Rows q{Q, Q_out, 0, strides[0], strides[1], 0, strides[6], strides[7], heads}, k_rows{K, nullptr, 0, strides[2], strides[3], 0, 0, 0, c->kv_heads},
        v_rows{V, nullptr, 0, strides[4], strides[5], 0, 0, 0, c->kv_heads};
    const rope::Turn turn{rotary > 0 ? positions : nullptr, frequencies, rotary, amplitude, 1.0f};
    const auto kernel = layout == 0 ? rope::append_kernel<true> : rope::append_kernel<false>;
    if (launch_overlapped_3d(kernel, static_cast<unsigned>(blocks), static_cast<unsigned>(q_groups + 2 * kv_groups), 1, rope::kThreads,
                             static_cast<cudaStream_t>(stream), q, k_rows, v_rows, view_of(c), starts, turn, tokens, parts, each, q_groups,
                             kv_groups) != cudaSuccess) {
        (void)cudaGetLastError();
        return ATTNW_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return ATTNW_OK;
}

// Where the parts of attn_paged's workspace begin.
struct PagedWorkspace {
    unsigned long long lse2 = 0, joins = 0, stats = 0, o = 0, bytes = 0;
    int q_tiles = 0, part_rows = 0;  // part_rows 0: no block is long enough to be cut
};
constexpr int kPagedCtas = 148;  // CTAs of attn_paged_kernel, at most: one an SM of a B200
PagedWorkspace paged_workspace(const attnw_cache* c, int tokens, int heads, bool weigh) {
    PagedWorkspace w;
    auto take = [&w](unsigned long long bytes) {
        const unsigned long long at = w.bytes;
        w.bytes = (w.bytes + bytes + 255) / 256 * 256;
        return at;
    };
    const int group = heads / c->kv_heads, tile_tokens = 128 / group;
    w.q_tiles = tokens / tile_tokens + std::min(c->sequences, tokens);
    if (weigh) w.lse2 = take(4ull * kTile * w.q_tiles * c->kv_heads);
    const long long tiles = (static_cast<long long>(c->table_width) * c->page + kTile - 1) / kTile;
    if (tiles >= pa::kLeastCut) {  // two parts for each CTA, of a block's rows
        w.part_rows = static_cast<int>(std::min(2ll * tile_tokens * group, static_cast<long long>(tokens) * group));
        w.joins = take(sizeof(pa::Join) * kPagedCtas);
        w.stats = take(8ull * 2 * kPagedCtas * w.part_rows);
        w.o = take(4ull * 2 * kPagedCtas * w.part_rows * c->d);
    }
    return w;
}

template <int D>
int launch_paged(const attnw_cache* c, const void* Q, const long long* q_strides, const int* starts, void* O, float* lse, const float* mass, float* mass_out,
                 char* workspace, const PagedWorkspace& w, int tokens, int heads, float scale, int least, int sm_count, cudaStream_t stream) {
    using L = pa::Smem<D>;
    const int group = heads / c->kv_heads, tile_tokens = 128 / group;
    CUtensorMap tm_q, tm_k, tm_v;
    // [tokens, key heads, heads of the group, d]; a dimension of size 1 gets a stride that the encoder accepts
    const unsigned long long head = heads > 1 ? q_strides[1] : D, token = tokens > 1 ? q_strides[0] : D;
    int rc = encode_4d(&tm_q, Q, D, group, c->kv_heads, tokens, 2 * head, 2 * head * group, 2 * token, 64, group, 1, tile_tokens);
    const int box = std::min(c->page, kTile);
    const uint64_t places = static_cast<uint64_t>(c->pages) * c->kv_heads;
    if (rc == ATTNW_OK) rc = encode_3d(&tm_k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c->K, D, c->page, places, 64, box);
    if (rc == ATTNW_OK) rc = encode_3d(&tm_v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c->V, D, c->page, places, 64, box);
    if (rc != ATTNW_OK) return rc;
    if ((least > 1 ? allow_smem<pa::attn_paged_kernel<D, true>>(L::kDynamicBytes) : allow_smem<pa::attn_paged_kernel<D, false>>(L::kDynamicBytes)) != cudaSuccess) {
        (void)cudaGetLastError();
        return ATTNW_ERR_CUDA;
    }
    const paged::Cache view = view_of(c);
    // As many CTAs as may have something to do: the most that all blocks can cost, by the shortest stretches.
    const int sequences = std::min(c->sequences, tokens / least);  // at most, that have new tokens of ours
    const long long blocks = (tokens / (2 * tile_tokens) + static_cast<long long>(sequences)) * c->kv_heads;
    const long long capacity = static_cast<long long>(c->table_width) * c->page, most = blocks * (pa::kBlockCost + capacity * (tokens > tile_tokens ? 2 : 1));
    const int ctas = static_cast<int>(std::min({static_cast<long long>(kPagedCtas), static_cast<long long>(sm_count), (most + pa::kLeastEven - 1) / pa::kLeastEven}));
    const pa::Shape shape{tokens, heads, group, tile_tokens, w.part_rows, w.q_tiles, ctas, least};
    auto* stats = w.part_rows > 0 ? reinterpret_cast<float2*>(workspace + w.stats) : nullptr;
    auto* joins = w.part_rows > 0 ? reinterpret_cast<pa::Join*>(workspace + w.joins) : nullptr;
    auto* part = w.part_rows > 0 ? reinterpret_cast<float*>(workspace + w.o) : nullptr;
    const float scale_log2e = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634074);
    auto* o = static_cast<__nv_bfloat16*>(O);
    auto* lse2 = mass ? reinterpret_cast<float*>(workspace + w.lse2) : nullptr;
    const auto kernel = least > 1 ? pa::attn_paged_kernel<D, true> : pa::attn_paged_kernel<D, false>;
    cudaError_t e = launch_overlapped(kernel, static_cast<unsigned>(ctas), pa::kThreads, L::kDynamicBytes, stream, 1, tm_q, tm_k, tm_v, view,
                                      shape, starts, scale_log2e, o, lse, lse2, part, stats, joins);
    if (e == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    if (e == cudaSuccess && part && ctas > 1) {
        const unsigned slices = static_cast<unsigned>((w.part_rows + pa::kJoinRows * pa::kJoinWarps - 1) / (pa::kJoinRows * pa::kJoinWarps));
        e = launch_overlapped_3d(pa::combine_kernel<D>, static_cast<unsigned>(ctas - 1), slices, 1, pa::kJoinWarps * 32, stream, view, shape, starts, part, stats, joins, o,
                                 lse, lse2);
        if (e == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    if (e == cudaSuccess && mass) {
        // segments: at most kSegments more than one a (sequence with new tokens, key head)
        const long long segments = pm::kSegments + static_cast<long long>(sequences) * c->kv_heads;
        e = allow_smem<pm::mass_kernel<D>>(pm::Smem<D>::kDynamicBytes);
        if (e == cudaSuccess)
            e = launch_overlapped(pm::mass_kernel<D>, static_cast<unsigned>(segments), pm::kThreads, pm::Smem<D>::kDynamicBytes, stream, 1, tm_q, tm_k, view, shape,
                                  starts, lse2, scale_log2e, mass, mass_out);
        if (e == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return ATTNW_ERR_CUDA;
    }
    return ATTNW_OK;
}

// How many clusters of `ctas` CTAs of attn_few_kernel the device holds at once, one CTA an SM; at least 1.
int few_max_clusters(DeviceInfo* dev, int ctas) {
    if (ctas == 1) return dev->sm_count;
    std::atomic<int>& memo = dev->few_clusters[ctas];
    int n = memo.load(std::memory_order_relaxed);
    if (n != 0) return n;
    constexpr auto kernel = few::attn_few_kernel<128, 4, true>;  // (of the largest; where others fit twice, twice as many do)
    const int bytes = few::Smem<128, 4>::bytes(few::kMaxScores / 5 / few::kUnit * few::kUnit, true);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(ctas);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(few::kThreads, 1, 1);
    cfg.gridDim = dim3(static_cast<unsigned>(ctas * dev->sm_count), 1, 1);
    cfg.dynamicSmemBytes = static_cast<size_t>(bytes);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (allow_smem<few::attn_few_kernel<128, 4, true>>(bytes) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        (void)cudaGetLastError();
        n = 1;
    }
    memo.store(n, std::memory_order_relaxed);
    return n;
}

// How attn_few_kernel would serve a call.
struct FewShape {
    int gp = 0;  // heads of the group, rounded up to a power of two; 0: it does not
    int cluster = 1, max_keys = 0;
    long long rounds = 0;  // of clusters
};
FewShape few_shape(DeviceInfo* dev, const attnw_cache* c, int tokens, int heads, bool weigh) {
    FewShape f;
    const int group = heads / c->kv_heads;
    if (group > 8) return f;
    int gp = 1;
    while (gp < group) gp *= 2;
    // The largest clusters that all fit at once, of 64 keys a CTA at least: a second round costs as much as the first (one over 2000, 8 heads on
    // 8, d = 64: clusters of 1 ... 6 11.2 ... 6.6 us, of 8, of which 15 fit and 16 are needed, 10.7).
    const long long capacity = static_cast<long long>(c->table_width) * c->page, items = static_cast<long long>(weigh ? c->sequences : tokens) * c->kv_heads;
    if (items * few::kMaxCluster > INT_MAX) return f;
    f.cluster = few::kMaxCluster;
    while (f.cluster > 1 && (capacity < 64ll * f.cluster || items > few_max_clusters(dev, f.cluster))) --f.cluster;
    auto keys_of = [&](int cluster) { return ((capacity + few::kUnit - 1) / few::kUnit + cluster - 1) / cluster * few::kUnit; };
    while (f.cluster < few::kMaxCluster && keys_of(f.cluster) * (gp + 1) > few::kMaxScores) ++f.cluster;
    if (keys_of(f.cluster) * (gp + 1) > few::kMaxScores) return f;
    f.max_keys = static_cast<int>(keys_of(f.cluster));
    const int at_once = few_max_clusters(dev, f.cluster);
    f.rounds = (items + at_once - 1) / at_once;
    f.gp = gp;
    return f;
}

template <int D, int GP, bool WEIGH>
cudaError_t launch_few(const attnw_cache* c, const FewShape& f, const void* Q, const long long* q_strides, const int* starts, void* O, float* lse, const float* mass,
                       float* mass_out, int tokens, int heads, float scale, int turns, cudaStream_t stream) {
    constexpr int most = few::Smem<D, GP>::bytes(few::kMaxScores / (GP + 1) / few::kUnit * few::kUnit, WEIGH);
    cudaError_t e = allow_smem<few::attn_few_kernel<D, GP, WEIGH>>(most);
    if (e != cudaSuccess) return e;
    const few::Shape shape{tokens, heads, heads / c->kv_heads, f.cluster, f.max_keys, turns};
    const float scale_log2e = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634074);
    const long long items = static_cast<long long>(WEIGH ? c->sequences : tokens) * c->kv_heads;
    return launch_overlapped(few::attn_few_kernel<D, GP, WEIGH>, static_cast<unsigned>(items * f.cluster), few::kThreads,
                             static_cast<size_t>(few::Smem<D, GP>::bytes(f.max_keys, WEIGH)), stream, f.cluster, static_cast<const __nv_bfloat16*>(Q),
                             tokens > 1 ? q_strides[0] : 0, heads > 1 ? q_strides[1] : 0, view_of(c), shape, starts, scale_log2e, static_cast<__nv_bfloat16*>(O),
                             lse, mass, mass_out);
}

template <int D, bool WEIGH>
cudaError_t launch_few_group(const attnw_cache* c, const FewShape& f, const void* Q, const long long* q_strides, const int* starts, void* O, float* lse,
                             const float* mass, float* mass_out, int tokens, int heads, float scale, int turns, cudaStream_t stream) {
    const auto launch = f.gp == 1   ? launch_few<D, 1, WEIGH>
                        : f.gp == 2 ? launch_few<D, 2, WEIGH>
                        : f.gp == 4 ? launch_few<D, 4, WEIGH>
                                    : launch_few<D, 8, WEIGH>;
    return launch(c, f, Q, q_strides, starts, O, lse, mass, mass_out, tokens, heads, scale, turns, stream);
}

// Is it the faster one?  Its time goes by the bytes that a CTA reads, 25 us a MB, more with many heads, and some 3 us a round of CTAs besides; the
// other one's by the bytes in all, which it spreads evenly, after 12 us (blocks that are not cut) to 25 (cut ones, joined), and with weights 10 to 30
// more.  The lengths are on the device: caches count as full.  us per call, few -> tensor cores, 32 heads on 8, d = 128: one token over 100 keys 6.9 / 13.1,
// 1000 7.9 / 23.3, 4000 11.1 / 19.9, 16000 27.2 / 27.7, 16 over 1000 16.8 / 28.1, 8 over 4095 30.8 / 43.0, of all lengths up to that 27.6 / 28.7, 32 over 4095
// 120 / 117, 16 tokens of one sequence over 500 10.5 / 17.4, 16 each of four over 3000 130 / 31; 64 heads on 8, 8 tokens over 4000 46 / 43; 8 heads on 8
// 30 / 42.  With weights: 1 over 1000 9.9 / 32.6, 16000 31 / 47, 32 over 4095 134 / 223, 64 heads on 8, 8 over 4000 57 / 74; four tokens of one sequence
// over 100 24.7 / 21.1.
bool few_pays(const attnw_cache* c, const FewShape& f, int tokens, bool weigh) {
    if (weigh && tokens > c->sequences) return false;  // (then some sequence has several, and those take turns there: kTurns)
    long long most = f.gp <= 4 ? 1024 : 512;  // kB
    if (weigh) most = f.gp <= 4 ? 16384 : 4096;
    if (tokens > c->sequences) most = most * 3 / 4;  // (the other one reads a sequence's keys once for all its tokens)
    return f.rounds * (f.max_keys * 4ll * c->d / 1024 + 128) <= most + 128;
}

// With weights the kernel for few tokens has one cluster a (sequence, key head), and several tokens of one sequence take turns in it, each of them a pass over its
// keys.  How the new tokens are dealt out is on the device: as many as there are sequences may be one of each, or a chunk of one among others that are
// idle.  So sequences with more than kTurns are left to the other kernels, which are launched behind it and at once find out if there are none; calls of up to
// kTurnsInAll tokens are spared that.  us per call, 32 heads on 8, d = 128, alone -> with the others behind it: 64 sequences of 256 keys with one token each 36.4 ->
// 40.7, 32 of 4096 134 -> 140, 256 of 256 130 -> 136, 16 of 256 9.7 -> 14.4 (spared); a chunk of 16, 32, 64 and 256 of one among as many of 256 keys 113 -> 29
// (spared), 223 -> 25, 440 -> 33 and 1650 -> 76, of 32 among 32 of 4096 849 -> 46.  (The tensor cores for all: 65, 184, 342, 28 and 20, 23, 37, 165, 43.)
constexpr int kTurns = 8, kTurnsInAll = 16;

int paged_entry(const attnw_cache* c, const void* Q, const long long* q_strides, const int* starts, void* O, float* lse, const float* mass, float* mass_out,
                void* workspace, unsigned long long workspace_bytes, int tokens, int heads, float scale, void* stream) {
    int rc = check_cache(c);
    if (rc != ATTNW_OK) return rc;
    if (!Q || !q_strides || !starts || !O || (!mass) != (!mass_out)) return ATTNW_ERR_NULL_POINTER;
    if (tokens < 1 || heads < 1 || heads % c->kv_heads != 0) return ATTNW_ERR_BAD_SHAPE;
    if (!(scale >= 0.0f) || !std::isfinite(scale)) return ATTNW_ERR_BAD_SHAPE;
    if (heads / c->kv_heads > 128) return ATTNW_ERR_UNSUPPORTED;
    if (static_cast<long long>(tokens) * heads > INT_MAX / 4) return ATTNW_ERR_BAD_SHAPE;
    const long long sizes[2] = {tokens, heads};
    rc = check_strides(q_strides, sizes, 2, 2, 1);  // (a tensor map has no broadcast dimensions, and strides below 2^40 bytes)
    if (rc != ATTNW_OK) return rc;
    if ((tokens > 1 && q_strides[0] >= 1ll << 39) || (heads > 1 && q_strides[1] * (heads / c->kv_heads) >= 1ll << 39)) return ATTNW_ERR_BAD_SHAPE;
    if (!aligned16(Q) || !aligned16(O) || !aligned4(starts) || !aligned4(lse) || !aligned4(mass) || !aligned4(mass_out)) return ATTNW_ERR_MISALIGNED;
    const unsigned long long capacity = static_cast<unsigned long long>(c->table_width) * c->page, weights = 4ull * c->sequences * c->kv_heads * capacity;
    const PagedWorkspace w = paged_workspace(c, tokens, heads, mass != nullptr);
    if (w.bytes > 0 && !workspace) return ATTNW_ERR_NULL_POINTER;
    if (workspace_bytes < w.bytes) return ATTNW_ERR_BAD_SHAPE;
    if (w.bytes > 0 && !aligned16(workspace)) return ATTNW_ERR_MISALIGNED;
    const Span out[4] = {{O, 2ull * tokens * heads * c->d}, {lse, 4ull * tokens * heads}, {mass_out, weights}, {w.bytes ? workspace : nullptr, w.bytes}};
    const Span in[6] = {{c->K, cache_bytes(c)}, {c->V, cache_bytes(c)}, {c->table, 4ull * c->sequences * c->table_width}, {c->lengths, 4ull * c->sequences},
                        {starts, 4ull * (c->sequences + 1ull)}, span_of(extent_of(Q, q_strides, sizes, 2, 0, c->d, 2))};
    for (int i = 0; i < 4; ++i) {
        for (const Span& s : in)
            if (crosses(out[i], s)) return ATTNW_ERR_ALIASING;
        for (int j = 0; j < i; ++j)
            if (crosses(out[i], out[j])) return ATTNW_ERR_ALIASING;
        if (crosses(out[i], {mass, weights}) && !(out[i].p == mass_out && mass == mass_out)) return ATTNW_ERR_ALIASING;
    }
    DeviceInfo* dev = nullptr;
    rc = current_device(&dev);
    if (rc != ATTNW_OK) return rc;
    const int variant = g_paged_variant.load(std::memory_order_relaxed);
    const FewShape f = variant == 1 ? FewShape{} : few_shape(dev, c, tokens, heads, mass != nullptr);
    if (variant == 2 && f.gp == 0) return ATTNW_ERR_UNSUPPORTED;
    int least = 1;
    if (f.gp > 0 && (variant == 2 || few_pays(c, f, tokens, mass != nullptr))) {
        const bool both = variant == 0 && mass && tokens > kTurnsInAll;
        const auto launch = c->d == 64 ? (mass ? launch_few_group<64, true> : launch_few_group<64, false>)
                                       : (mass ? launch_few_group<128, true> : launch_few_group<128, false>);
        if (launch(c, f, Q, q_strides, starts, O, lse, mass, mass_out, tokens, heads, scale, both ? kTurns : INT_MAX, static_cast<cudaStream_t>(stream)) !=
            cudaSuccess) {
            (void)cudaGetLastError();
            return ATTNW_ERR_CUDA;
        }
        g_launches.fetch_add(1, std::memory_order_relaxed);
        if (!both) return ATTNW_OK;
        least = kTurns + 1;
    }
    rc = load_encoder();
    if (rc != ATTNW_OK) return rc;
    const auto launch = c->d == 64 ? launch_paged<64> : launch_paged<128>;
    return launch(c, Q, q_strides, starts, O, lse, mass, mass_out, static_cast<char*>(workspace), w, tokens, heads, scale, least, dev->sm_count,
                  static_cast<cudaStream_t>(stream));
}

int evict_entry(const attnw_cache* c, const int* table_out, int table_out_width, const float* mass, float* mass_out, int* kept, int* lengths_out, int budget,
                int recent, void* stream) {
    int rc = check_cache(c);
    if (rc != ATTNW_OK) return rc;
    if (!mass || !mass_out || !kept || !lengths_out) return ATTNW_ERR_NULL_POINTER;
    const bool in_place = !table_out || table_out == c->table;
    const int width_out = table_out ? table_out_width : c->table_width;
    if (width_out < 1 || (table_out == c->table && width_out != c->table_width)) return ATTNW_ERR_BAD_SHAPE;
    const long long capacity = static_cast<long long>(c->table_width) * c->page, capacity_out = static_cast<long long>(width_out) * c->page;
    if (budget < 1 || recent < 0 || recent > budget || budget > capacity_out || capacity_out > (1 << 28)) return ATTNW_ERR_BAD_SHAPE;
    if (!aligned4(mass) || !aligned4(mass_out) || !aligned4(kept) || !aligned4(lengths_out) || !aligned4(table_out)) return ATTNW_ERR_MISALIGNED;
    const unsigned long long rows = static_cast<unsigned long long>(c->sequences) * c->kv_heads;
    const Span out[5] = {{c->K, cache_bytes(c)}, {c->V, cache_bytes(c)}, {mass_out, 4ull * rows * capacity_out}, {kept, 4ull * rows * budget},
                         {lengths_out, 4ull * c->sequences}};
    const Span in[4] = {{c->table, 4ull * c->sequences * c->table_width}, {c->lengths, 4ull * c->sequences},
                        {table_out, table_out ? 4ull * c->sequences * width_out : 0}, {mass, 4ull * rows * capacity}};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < i; ++j)
            if (crosses(out[i], out[j])) return ATTNW_ERR_ALIASING;
        for (const Span& s : in)
            if (crosses(out[i], s) && !(i == 2 && s.p == mass && mass == mass_out && capacity == capacity_out)) return ATTNW_ERR_ALIASING;
    }
    DeviceInfo* dev = nullptr;
    rc = current_device(&dev);
    if (rc != ATTNW_OK) return rc;
    const paged::Cache view = view_of(c);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch_overlapped_3d(evict::evict_select_kernel, static_cast<unsigned>(rows), 1, 1, evict::kSelectThreads, s, view, mass, mass_out, kept,
                                         lengths_out, budget, recent, static_cast<int>(capacity), static_cast<int>(capacity_out));
    if (e == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    if (e == cudaSuccess) {
        // In place: as many CTAs a row as fill the device twice, of at least 32 bytes of each key.
        int slices = 1;
        while (in_place && slices < c->d / 16 && static_cast<long long>(rows) * 2 * slices < 2 * dev->sm_count) slices *= 2;
        const int keys = evict::kMoveThreads * evict::kFlight / (c->d / 8 / slices), steps = in_place ? 1 : (budget + keys - 1) / keys;
        const auto kernel = in_place ? evict::evict_move_kernel<true> : evict::evict_move_kernel<false>;
        e = launch_overlapped_3d(kernel, static_cast<unsigned>(steps * slices), static_cast<unsigned>(rows), 2, evict::kMoveThreads, s, view,
                                 in_place ? c->table : table_out, width_out, kept, budget, slices);
        if (e == cudaSuccess) g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return ATTNW_ERR_CUDA;
    }
    return ATTNW_OK;
}

}  // namespace
