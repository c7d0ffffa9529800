"""The paged cache on the GPU where tables, values or sizes are out of the ordinary."""
import math

import pytest
import torch

from paged_reference import Paged
from test_gpu_cache import check_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def attnw():
    from paper_2407_13885_b200 import binding
    yield binding
    assert binding.query_status() == 0


@pytest.fixture(params=["tensor_cores", "few"])
def variant(attnw, request):
    attnw.set_paged_variant(request.param)
    yield request.param
    attnw.set_paged_variant("auto")


def bits(x):
    return x.view(torch.int32 if x.dtype == torch.float32 else torch.int16).cpu()


# ---- eviction ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_eviction_of_keys_without_a_page(attnw, in_place, d):
    # A page that the cache does not have reads as zeros: a key of it that stays is zero in its new place, whatever was there.
    page, budget, recent = 16, 40, 10
    c = Paged([(0, 100), (0, 130)], 2, d, page, spare=9)
    c.table[0, 3], c.table[0, 6], c.table[1, 2], c.table[1, 8] = -1, c.pages, 2 ** 31 - 1, -5
    mass = torch.rand(2, 2, c.width * page, generator=c.gen).cuda()
    mass[0, :, 48:64] += 1.0                       # the keys of missing pages are among those that stay
    mass[1, 0, 32:48] += 1.0
    K0, V0 = c.K.cpu(), c.V.cpu()
    before = c.table.cpu()
    out = None if in_place else torch.tensor(c.spare[:6], dtype=torch.int32, device="cuda").view(2, 3)
    kept, lengths, _ = attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, budget, recent, table_out=out)
    assert lengths.tolist() == [40, 40] and torch.equal(c.table.cpu(), before)
    to = (c.table if in_place else out).cpu().long()
    want_K, want_V = K0.clone(), V0.clone()
    zeros = 0
    for b in range(2):
        for h in range(2):
            for t in range(budget):
                s = int(kept[b, h, t])
                source, target = int(before[b, s // page]), int(to[b, t // page])
                if not 0 <= target < c.pages:
                    continue
                there = 0 <= source < c.pages
                zeros += not there
                want_K[target, h, t % page] = K0[source, h, s % page] if there else 0.0
                want_V[target, h, t % page] = V0[source, h, s % page] if there else 0.0
    assert zeros >= 16
    assert torch.equal(bits(c.K), bits(want_K)) and torch.equal(bits(c.V), bits(want_V))


def kept_by_definition(row, length, budget, recent):
    """The last `recent` keys, and of the others those of most weight: of equal ones the first, NaN below every number."""
    if length <= budget:
        return torch.arange(length)
    old = row[:length - recent].double()
    nan = torch.isnan(old)
    by_weight = torch.argsort(old.masked_fill(nan, -math.inf), descending=True, stable=True)
    order = by_weight[torch.argsort(nan[by_weight].to(torch.int8), stable=True)]
    return torch.cat((order[:budget - recent].sort().values, torch.arange(length - recent, length)))


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("budget,recent,lengths", [
    (1000, 100, [16385 + 100, 16384 + 100, 16384 + 101]),   # keys to choose from: one more than the first turn has, and as many
    (20000, 77, [40003, 20000, 20001, 33000]),
    (33000, 0, [49153, 32768, 33001]),
    (5, 5, [40000, 3]),
    (16400, 16390, [36001]),
])
@pytest.mark.parametrize("weights", ["spread", "near", "ties", "equal", "odd", "late"])
def test_eviction_of_long_rows(attnw, budget, recent, lengths, in_place, weights):
    page, Hkv, d = 64, 2, 64
    c = Paged([(0, n) for n in lengths], Hkv, d, page, seed=budget + recent, spare=1 + len(lengths) * -(-budget // page))
    C = c.width * page
    mass = torch.randn(len(lengths), Hkv, C, generator=c.gen).mul(2).exp()
    if weights == "near":     # the same upper 13 bits for more keys than a list holds, and the same 24 for many
        mass = 1.0 + torch.randint(0, 4096, mass.shape, generator=c.gen) * 2.0 ** -23
    elif weights == "ties":   # equal to the last bit: the border lies among them, in the second or third turn
        mass = (mass * 2).floor().clamp_max(3.0)
    elif weights == "equal":
        mass = torch.full_like(mass, 0.25)
    elif weights == "late":   # the first keys have the least
        mass = torch.where(torch.arange(C) < 15000, 0.125, 0.25).expand_as(mass).contiguous()
    elif weights == "odd":
        pool = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, 1e-45, -1.0, 3e38, 1.0])
        mass = pool[torch.randint(0, 9, mass.shape, generator=c.gen)]
    mass0, mass = mass, mass.cuda()
    K0, V0 = c.K.cpu(), c.V.cpu()
    width = c.width if in_place else -(-budget // page)
    out = None if in_place else torch.tensor(c.spare[:len(lengths) * width], dtype=torch.int32, device="cuda").view(len(lengths), width)
    kept, now, mass_out = attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, budget, recent, table_out=out, mass_out=mass if in_place else None)
    assert now.tolist() == [min(n, budget) for n in lengths]
    want_K, want_V = K0.clone(), V0.clone()
    want_kept = torch.full((len(lengths), Hkv, budget), -1, dtype=torch.int32)
    want_mass = torch.zeros(len(lengths), Hkv, width * page)
    to_table = (c.table if in_place else out).cpu().long()
    for b, length in enumerate(lengths):
        for h in range(Hkv):
            src = kept_by_definition(mass0[b, h], length, budget, recent)
            t = torch.arange(len(src))
            want_kept[b, h, :len(src)] = src.to(torch.int32)
            want_mass[b, h, :len(src)] = mass0[b, h, src]
            from_page, to_page = c.table[b].cpu().long()[src // page], to_table[b][t // page]
            want_K[to_page, h, t % page], want_V[to_page, h, t % page] = K0[from_page, h, src % page], V0[from_page, h, src % page]
    assert torch.equal(kept.cpu(), want_kept)
    assert torch.equal(bits(mass_out), bits(want_mass))
    assert torch.equal(bits(c.K), bits(want_K)) and torch.equal(bits(c.V), bits(want_V))
    if not in_place:
        assert torch.equal(bits(mass), bits(mass0))


def test_a_budget_that_is_refused_takes_no_memory(attnw):
    c = Paged([(0, 100)] * 3, 2, 64, 16)
    mass = torch.rand(3, 2, c.width * 16, device="cuda")
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    for budget in (c.width * 16 + 1, 10 ** 6, 2 ** 31 - 1, 0, -1, -2 ** 31):   # (2^31 - 1: 51 GB of places)
        with pytest.raises(attnw.AttnwError) as e:
            attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, budget, 0)
        assert e.value.code == 2
    assert torch.cuda.max_memory_allocated() - before < 1 << 20
    for budget, recent in ((2 ** 31, 0), (8, 2 ** 31), (-2 ** 31 - 1, 0)):
        with pytest.raises(ValueError):
            attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, budget, recent)


# ---- values that are not finite -----------------------------------------------------------------------------------------------

def attend(attnw, c, Q, scale=0.125):
    lse = torch.full(Q.shape[:2], 7.0, device="cuda")
    mass = torch.rand(len(c.pairs), c.Hkv, c.width * c.page, generator=torch.Generator().manual_seed(3)).cuda()
    O, out = attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, scale, lse=lse, mass=mass)
    torch.cuda.synchronize()
    assert attnw.query_status() == 0
    return O, lse, out, mass


def put(c, cache, b, at, h, feature, value):
    cache[int(c.table[b, at // c.page]), h, at % c.page, feature] = value


VALUES = [  # (H, Hkv, d, page, pairs, [(sequence, key, key head, features, value)])
    (8, 2, 64, 16, [(40, 300), (200, 700), (5, 5), (1, 130)],
     [(0, 280, 0, [3], math.nan), (1, 650, 1, [0, 5, 63], math.inf), (1, 699, 0, [10], -math.inf), (2, 4, 0, list(range(64)), math.nan),
      (1, 600, 0, [20], math.inf), (1, 620, 0, [20], -math.inf), (1, 50, 1, [7], math.inf), (3, 129, 1, [1], math.nan)]),
    (4, 4, 128, 64, [(300, 300), (7, 1000)],
     [(0, 0, 0, [0], math.nan), (0, 127, 1, [64, 65, 127], math.inf), (0, 128, 2, [1, 90], math.nan), (0, 299, 3, [17], -math.inf), (0, 255, 3, [17, 18], math.nan),
      (1, 999, 0, list(range(128)), math.nan), (1, 994, 1, [5], math.inf)]),
    (6, 2, 128, 32, [(130, 3000)], [(0, 2870, 0, [2], math.nan), (0, 2999, 1, [33, 100], math.inf), (0, 2944, 1, [34], math.nan), (0, 12, 0, [50], math.nan)]),
    (3, 1, 64, 16, [(90, 80)], [(0, 79, 0, [8], math.nan), (0, 0, 0, [9], math.inf)]),
]


@pytest.mark.parametrize("H,Hkv,d,page,pairs,places", VALUES)
def test_values_that_are_not_finite_reach_only_the_tokens_that_see_them(attnw, variant, H, Hkv, d, page, pairs, places):
    c = Paged(pairs, Hkv, d, page, seed=21, front=1, behind=1)
    Q = c.normal(c.tokens, H, d)
    clean = attend(attnw, c, Q)
    starts = c.starts.tolist()
    hit = torch.zeros(c.tokens, H, d, dtype=torch.bool)
    G = H // Hkv
    for b, at, h, features, value in places:
        put(c, c.V, b, at, h, torch.tensor(features), value)
        n, length = pairs[b]
        first = max(0, at - (length - n))    # the first token that sees the key
        for f in features:
            hit[starts[b] + first:starts[b + 1], h * G:(h + 1) * G, f] = True
    for _ in range(3):
        O, lse, out, _ = attend(attnw, c, Q)
        first, last = starts[0], starts[-1]
        bad = ~torch.isfinite(O.float().cpu())[first:last]
        assert torch.equal(bad, hit[first:last])
        # rows and features have nothing to do with one another: the others are the same to the last bit
        keep = ~hit[first:last]
        assert torch.equal(O.cpu()[first:last][keep], clean[0].cpu()[first:last][keep])
        assert torch.equal(lse.cpu()[first:last], clean[1].cpu()[first:last]) and torch.equal(out, clean[2])


@pytest.mark.parametrize("H,Hkv,d,page", [(8, 2, 64, 16), (6, 2, 128, 64), (2, 2, 128, 32), (3, 3, 64, 16)])
def test_scores_that_are_not_numbers(attnw, variant, H, Hkv, d, page):
    # A score of NaN makes its row's sum NaN, and with it the row's result, its logarithm and all of its weights.
    pairs = [(1, 9000), (70, 500), (3, 300), (2, 40), (1, 64), (1, 9100)]
    if variant == "few":
        pairs[1] = (9, 500)
    c = Paged(pairs, Hkv, d, page, seed=22)
    Q = c.normal(c.tokens, H, d)
    clean = attend(attnw, c, Q)
    starts = c.starts.tolist()
    rows = torch.zeros(c.tokens, H, dtype=torch.bool)
    keys = torch.zeros(len(pairs), Hkv, c.width * page, dtype=torch.bool)
    G = H // Hkv
    n1 = pairs[1][0]
    for b, at, h in ((0, 4321, 0), (1, 500 - n1 + 4, 1), (5, 0, 1), (5, 9099, 0)):
        put(c, c.K, b, at, h, torch.tensor([5]), math.nan)
        n, length = pairs[b]
        rows[starts[b] + max(0, at - (length - n)):starts[b + 1], h * G:(h + 1) * G] = True
        keys[b, h, :length] = True
    Q[starts[2], 0, 3] = math.nan              # the first of three tokens: the last two keys are not its
    rows[starts[2], 0] = True
    keys[2, 0, :298] = True
    O, lse, out, prior = attend(attnw, c, Q)
    assert torch.equal(torch.isnan(O.float()).cpu(), rows[..., None].expand(-1, -1, d))
    assert torch.equal(torch.isnan(lse).cpu(), rows) and torch.equal(torch.isnan(out).cpu(), keys)
    assert torch.equal(O.cpu()[~rows], clean[0].cpu()[~rows]) and torch.equal(lse.cpu()[~rows], clean[1].cpu()[~rows])
    untouched = ~keys
    untouched[2, 0, 298:300] = False           # (two of three tokens: the same sums, but checked apart)
    assert torch.equal(out.cpu()[untouched], clean[2].cpu()[untouched])
    assert float((out[2, 0, 298:300] - clean[2][2, 0, 298:300]).abs().max()) <= 2.0 ** -22 * 8


def test_a_score_of_minus_infinity_weighs_nothing(attnw, variant):
    # Groups of three heads: what fills the group up has no say, also where its score of 0 times infinity is NaN.
    c = Paged([(1, 400), (2, 90)], 2, 64, 16, seed=23)
    Q = c.normal(c.tokens, 6, 64)
    Q[..., 0] = Q[..., 0].abs() + 0.5
    for b, at in ((0, 17), (1, 60)):
        put(c, c.K, b, at, slice(None), torch.tensor([0]), -1e30)
    want = attend(attnw, c, Q)
    for b, at in ((0, 17), (1, 60)):
        put(c, c.K, b, at, slice(None), torch.tensor([0]), -math.inf)
    got = attend(attnw, c, Q)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


# ---- weights of keys where some sequences have many new tokens and others few ---------------------------------------------------

DEALT_OUT = [  # (H, Hkv, d, page, pairs)
    (8, 2, 64, 16, [(0, 200)] * 30 + [(25, 300)] + [(0, 70)] * 9),                       # a chunk of one among idle ones
    (32, 8, 128, 64, [(0, 200)] * 60 + [(48, 48)] + [(0, 0), (0, 256), (0, 1)]),
    (8, 2, 128, 16, [(1, 40 + 7 * i) for i in range(40)]),                                # one of each
    (6, 3, 64, 32, [(8, 200), (0, 90), (9, 100), (1, 64), (0, 300), (17, 40)] + [(0, 100)] * 40),
    (4, 4, 128, 32, [(9, 9), (8, 8), (16, 500), (1, 1), (0, 0), (30, 20)] + [(0, 33)] * 70),
    (2, 1, 64, 16, [(1, 100)] * 20 + [(200, 1500)] + [(1, 90)] * 20 + [(0, 50)] * 250),
]


@pytest.mark.parametrize("H,Hkv,d,page,pairs", DEALT_OUT)
@pytest.mark.parametrize("apart", [False, True])
def test_weights_of_tokens_that_are_dealt_out_unevenly(attnw, H, Hkv, d, page, pairs, apart):
    c = Paged(pairs, Hkv, d, page, seed=31, behind=2)
    c.tokens = min(c.tokens, len(pairs))                 # as many tokens as sequences, at most: the rule's own condition
    assert c.tokens > 16 and sum(n for n, _ in pairs) <= c.tokens
    Q = c.normal(c.tokens, H, d)
    for _ in range(2):                                   # (the second time with what the first left in the workspace)
        check_attention(attnw, c, Q, d ** -0.5)
    if not apart:
        return
    mass = torch.rand(len(pairs), Hkv, c.width * page, generator=c.gen).cuda()
    before = attnw.launch_count()
    O, out = attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, d ** -0.5, mass=mass)   # mass_out is other memory
    assert attnw.launch_count() - before >= 2            # not all by clusters that take one token after the other
    same = mass.clone()
    P, _ = attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, d ** -0.5, mass=same, mass_out=same)
    assert torch.equal(O[:sum(n for n, _ in pairs)], P[:sum(n for n, _ in pairs)]) and torch.equal(out, same)
    untouched = torch.arange(c.width * page, device="cuda")[None] >= c.lengths[:, None] * (c.starts.diff() > 0)[:, None]
    assert torch.equal(out.masked_select(untouched[:, None]), mass.masked_select(untouched[:, None]))


def test_a_captured_call_follows_the_starts(attnw):
    # Captured with one token of each sequence, replayed with a chunk of one, and back.
    c = Paged([(1, 300)] * 40, 2, 64, 16, seed=32)
    Q, mass = c.normal(40, 8, 64), torch.rand(40, 2, c.width * 16, generator=c.gen).cuda()
    call = lambda: attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, 0.125, mass=mass)  # noqa: E731
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        got = call()
    one = torch.arange(41, dtype=torch.int32, device="cuda")
    chunk = torch.where(one <= 7, 0, 40).to(torch.int32)
    for starts in (chunk, one, chunk, one):
        c.starts.copy_(starts)
        want = call()
        for t in got:
            t.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        c.pairs = [(int(n), 300) for n in starts.diff()]
        check_attention(attnw, c, Q, 0.125)
