"""Rotary positions, the paged cache, attention over it and eviction from it on the GPU against their definitions in 64 bits."""
import math

import pytest
import torch

from paged_reference import Paged, score_error, turned

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def attnw():
    from paper_2407_13885_b200 import binding
    yield binding
    assert binding.query_status() == 0


@pytest.fixture(params=["auto", "tensor_cores", "few"])
def variant(attnw, request):
    attnw.set_paged_variant(request.param)
    yield request.param
    attnw.set_paged_variant("auto")


# ---- rotary positions ---------------------------------------------------------------------------------------------------------

def rope_tolerance(x, y, frequencies, positions, dtype):
    # Each result is a sum of two products of float32 values: cos and sin off by 2 ulp (2^-22 each, sincospif) plus the angle's rounding to float32
    # (half turns below 1: 2^-25 pi), two products and a sum (2^-24 each), in the pair's norm, and the rounding to the result's type.
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[dtype]
    return half * y.abs() + 8 * 2.0 ** -22 * x.double().abs().max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,H,N,d,rotary", [(1, 1, 1, 64, 64), (2, 3, 5, 64, 16), (1, 12, 77, 64, 32), (2, 7, 130, 128, 128), (1, 40, 33, 128, 48),
                                            (3, 2, 1, 128, 0), (1, 300, 2, 128, 112)])
def test_rope(attnw, B, H, N, d, rotary, layout, dtype):
    gen = torch.Generator().manual_seed(B * 1000 + N)
    x = torch.randn(B, H, N, d, generator=gen).to(dtype).cuda()
    pos = torch.randint(-5, 1 << 20, (B, N), generator=gen, dtype=torch.int32).cuda()
    pos.view(-1)[0] = 2 ** 31 - 1
    f = attnw.rope_frequencies(rotary, 10000.0).cuda()
    for inverse, amplitude in ((False, 1.0), (True, 1.25)):
        ref = turned(x.cpu(), pos.cpu()[:, None, :], f.cpu(), layout, amplitude, inverse)
        y = attnw.rope(x, pos, f, layout=layout, amplitude=amplitude, inverse=inverse)
        assert y.dtype == dtype and y.is_contiguous()
        assert bool(((y.cpu().double() - ref).abs() <= 1.25 * rope_tolerance(x.cpu(), ref, f, pos, dtype)).all())
        assert torch.equal(y[..., rotary:], x[..., rotary:])


def test_rope_strides_and_in_place(attnw):
    x = torch.randn(2, 50, 24 * 64 + 64, device="cuda").bfloat16()
    pos = torch.arange(50, dtype=torch.int32, device="cuda").expand(2, 50).contiguous()
    f = attnw.rope_frequencies(64).cuda()
    heads = x.view(2, 50, 25, 64).transpose(1, 2)        # token-major memory seen head by head
    want = attnw.rope(heads.contiguous(), pos, f)
    assert torch.equal(attnw.rope(heads, pos, f), want)
    out = torch.full((2, 50, 25, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    assert attnw.rope(heads, pos, f, out=out.transpose(1, 2)).data_ptr() == out.data_ptr()
    assert torch.equal(out.transpose(1, 2), want)
    part = heads[:, 3:20]
    keep = x.clone().view(2, 50, 25, 64).transpose(1, 2)
    attnw.rope(part, pos, f, out=part)                       # in place, other heads as they were
    assert torch.equal(part, want[:, 3:20])
    assert torch.equal(heads[:, :3], keep[:, :3]) and torch.equal(heads[:, 20:], keep[:, 20:])
    # columns of one array of tokens: the result may lie between the inputs' rows
    attnw.rope(heads[:, 0:3], pos, f, out=heads[:, 21:24])
    assert torch.equal(heads[:, 21:24], want[:, 0:3])
    one = keep[:, :1].expand(2, 6, 50, 64)                    # one head broadcast to six
    assert torch.equal(attnw.rope(one, pos, f), want[:, :1].expand(2, 6, 50, 64))


def test_rope_gradient(attnw):
    # <g, R x> = <R^T g, x> exactly, for R linear: the inverse call is the transpose; and it undoes R
    x, g = (torch.randn(2, 3, 40, 128, device="cuda") for _ in range(2))
    pos = torch.randint(0, 1 << 17, (2, 40), dtype=torch.int32, device="cuda")
    for layout in ("half", "interleaved"):
        f = attnw.rope_frequencies(96, 500000.0, scaling="by_parts", factor=8.0, original=8192).cuda()
        y, back = attnw.rope(x, pos, f, layout=layout, amplitude=1.5), attnw.rope(g, pos, f, layout=layout, amplitude=1.5, inverse=True)
        a, b = float((g.double() * y.double()).sum()), float((back.double() * x.double()).sum())
        assert abs(a - b) <= 2 * 1.5 * 8 * 2.0 ** -22 * float((g.double().abs() * 2 * x.double().abs().max()).sum())
        again = attnw.rope(y, pos, f, layout=layout, amplitude=1 / 1.5, inverse=True)
        assert float((again - x).abs().max()) <= 4 * 8 * 2.0 ** -22 * float(x.abs().max())
        # against differences of the forward call: linear, so any step will do
        e = torch.randn_like(x)
        diff = float((g.double() * (attnw.rope(x + e, pos, f, layout=layout).double() - attnw.rope(x - e, pos, f, layout=layout).double())).sum()) / 2
        formula = float((turned(g.cpu(), pos.cpu()[:, None], f.cpu(), layout, 1.0, True) * e.cpu().double()).sum())
        got = float((attnw.rope(g, pos, f, layout=layout, inverse=True).double() * e.double()).sum())
        bound = 16 * 2.0 ** -22 * float((g.double().abs() * 8 * (x.abs() + e.abs()).double().max()).sum())
        assert abs(diff - formula) <= bound and abs(got - formula) <= bound


# ---- new tokens into the cache --------------------------------------------------------------------------------------------------

RAGGED = [(3, 3), (1, 40), (0, 17), (7, 100), (5, 2), (0, 0), (16, 31), (1, 1)]


@pytest.mark.parametrize("Hq,Hkv,d,page,rotary,layout,pairs", [
    (4, 4, 64, 16, 64, "half", [(1, 1)]),
    (8, 2, 128, 16, 128, "half", RAGGED),
    (9, 3, 64, 32, 32, "interleaved", RAGGED),
    (2, 1, 128, 64, 48, "half", [(1, 1 + 13 * i) for i in range(70)]),
    (32, 8, 128, 128, 128, "interleaved", [(700, 1500), (513, 513)]),
    (1, 1, 64, 16, 64, "half", [(1, 3 + i % 5) for i in range(700)]),
])
def test_append(attnw, Hq, Hkv, d, page, rotary, layout, pairs):
    c = Paged(pairs, Hkv, d, page, seed=len(pairs) + d, front=2, behind=3)
    T = c.tokens
    qkv = c.normal(T, Hq + 2 * Hkv, d)  # side by side, as one projection gives them
    Q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    pos = torch.randint(0, 1 << 18, (T,), generator=c.gen, dtype=torch.int32).cuda()
    f = attnw.rope_frequencies(rotary).cuda()
    K0, V0 = c.K.clone(), c.V.clone()
    Q_out = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    assert attnw.cache_append(Q, K, V, c.K, c.V, c.table, c.lengths, c.starts, pos, f, layout=layout, Q_out=Q_out) is Q_out
    q_ref, k_ref = (turned(x.cpu(), pos.cpu()[:, None], f.cpu(), layout) for x in (Q, K))
    first, last = int(c.starts[0]), int(c.starts[-1])
    assert bool((Q_out[:first] == 7.0).all()) and bool((Q_out[last:] == 7.0).all())
    err = (Q_out.cpu().double() - q_ref).abs()[first:last]
    assert bool((err <= rope_tolerance(Q.cpu(), q_ref[first:last], f, pos, torch.bfloat16)).all())
    K_want, V_want = K0.cpu().double(), V0.cpu()
    starts = c.starts.tolist()
    written = torch.zeros(c.pages, page, dtype=torch.bool)
    for b, (n, length) in enumerate(pairs):
        for i in range(n):
            at = length - n + i
            if at < 0:
                continue
            p = int(c.table[b, at // page])
            K_want[p, :, at % page], V_want[p, :, at % page] = k_ref[starts[b] + i], V[starts[b] + i].cpu()
            written[p, at % page] = True
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731 (bits: unused places hold NaN)
    assert same(c.V.cpu(), V_want)
    mask = written[:, None, :, None].expand_as(K_want)
    assert same(c.K.cpu().masked_fill(mask, 0.0), K0.cpu().masked_fill(mask, 0.0))
    err = ((c.K.cpu().double() - K_want).abs() - rope_tolerance(K.cpu(), K_want, f, pos, torch.bfloat16))[mask]
    assert bool((err <= 0).all())
    # in place, and without rotation or queries
    K1, qkv0 = c.K.clone(), qkv.clone()
    c.K.copy_(K0)
    attnw.cache_append(Q, K, V, c.K, c.V, c.table, c.lengths, c.starts, pos, f, layout=layout, Q_out=Q)
    assert same(c.K, K1) and torch.equal(Q[first:last], Q_out[first:last])
    assert torch.equal(qkv[:, Hq:], qkv0[:, Hq:]) and torch.equal(qkv[:first], qkv0[:first]) and torch.equal(qkv[last:], qkv0[last:])
    c.K.copy_(K0)
    assert attnw.cache_append(None, K, V, c.K, c.V, c.table, c.lengths, c.starts) is None
    for b, (n, length) in enumerate(pairs):
        for i in range(max(0, n - length), n):
            at = length - n + i
            assert torch.equal(c.K[int(c.table[b, at // page]), :, at % page], K[starts[b] + i])


def test_append_ignores_bad_pages_lengths_and_starts(attnw):
    c = Paged([(4, 40), (4, 40), (4, 40)], 2, 64, 16, front=0)
    c.table[0, 2] = c.pages          # its new tokens (36 ... 39) lie there
    c.table[1, 2] = -1
    c.lengths[2] = 2 ** 31 - 1       # counts as the capacity: 48
    K, V = c.normal(12, 2, 64), c.normal(12, 2, 64)
    K0, V0 = c.K.clone(), c.V.clone()
    attnw.cache_append(None, K, V, c.K, c.V, c.table, c.lengths, c.starts)
    p = int(c.table[2, 2])
    assert torch.equal(c.K[p, :, 12:16], K[8:12].transpose(0, 1)) and torch.equal(c.V[p, :, 12:16], V[8:12].transpose(0, 1))
    c.K[p, :, 12:16], c.V[p, :, 12:16] = K0[p, :, 12:16], V0[p, :, 12:16]
    assert torch.equal(c.K.view(torch.int16), K0.view(torch.int16)) and torch.equal(c.V.view(torch.int16), V0.view(torch.int16))
    c.lengths[:] = -7
    attnw.cache_append(None, K, V, c.K, c.V, c.table, c.lengths, c.starts)
    for starts in ([0, 0, 0, 0], [5, 3, 2, 1], [-9, -8, -7, -6], [100, 200, 300, 400]):
        c.lengths[:] = 3
        attnw.cache_append(None, K[:1], V[:1], c.K, c.V, c.table, c.lengths, torch.tensor(starts, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(c.K.view(torch.int16), K0.view(torch.int16))


# ---- attention over the cache ---------------------------------------------------------------------------------------------------

def check_attention(attnw, c, Q, scale, with_mass=True):
    T, H, d = Q.shape
    O_ref, lse_ref, mass_ref, spread, most = c.attention(Q, scale)
    raw = torch.full((T + 8, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    O, lse = raw[4:-4], torch.full((T, H), 7.0, device="cuda")
    prior = torch.rand(len(c.pairs), c.Hkv, c.width * c.page, generator=c.gen).cuda()
    mass = prior.clone()
    if with_mass:
        got, out = attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, scale, O=O, lse=lse, mass=mass, mass_out=mass)
        assert got is O and out is mass
    else:
        assert attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, scale, O=O, lse=lse) is O
    torch.cuda.synchronize()
    assert attnw.query_status() == 0
    first, last = max(0, int(c.starts[0])), int(c.starts[-1])
    assert bool((raw[:4 + first] == 7.0).all()) and bool((raw[4 + last:] == 7.0).all())
    assert bool((lse[:first] == 7.0).all()) and bool((lse[last:] == 7.0).all())
    dz = score_error(most, scale, d)
    # O: the weights may be rounded to bf16 (2^-8 of each), are off by 2 dz for their scores (their own and the sum's) and some 2^-20 for the exponentials,
    # sums and the division, in float32; O is rounded once (2^-8).
    got = O.cpu().double()[first:last]
    bound = spread[first:last] * (2.0 ** -8 + 2 * dz + 2.0 ** -18) + 2.0 ** -8 * O_ref[first:last].abs() + 1e-30
    assert bool(torch.isfinite(got).all())
    worst = float(((got - O_ref[first:last]).abs() / bound).max()) if last > first else 0.0
    assert worst <= 1.0, f"O off by {worst} of its tolerance"
    empty = torch.isinf(lse_ref[first:last])
    got = lse.cpu().double()[first:last]
    assert torch.equal(torch.isinf(got) & (got < 0), empty)
    want = lse_ref[first:last][~empty]
    if want.numel():
        # the sum of up to 2^17 float32 exponentials in order, pairwise or in between: relative 2^-24 a step, at most as many steps as a thread adds up
        # (the keys over 64), then the logarithm's and the last sum's roundings
        assert float((got[~empty] - want).abs().max()) <= dz + 2.0 ** -18 + 2.0 ** -22 * float(want.abs().max())
    if with_mass:
        n = max((n for n, _ in c.pairs), default=0) * H // c.Hkv
        err = (mass.cpu().double() - prior.cpu().double() - mass_ref).abs()
        # a weight exp(z - lse): both off by dz, the exponential and the sums of lse by 2^-18 in all, then n float32 additions and the one to the prior
        assert bool((err <= mass_ref * (2 * dz + 2.0 ** -18 + n * 2.0 ** -24) + 2.0 ** -24 * (mass_ref + 1)).all()), float(err.max())
    return O, lse, mass


ATTENTION = [
    (1, 1, 64, 16, [(1, 1)]),
    (1, 1, 128, 16, [(1, 17)]),
    (12, 12, 64, 16, [(1, 501)]),
    (8, 2, 128, 16, [(1, 127), (1, 128), (1, 129), (1, 1), (1, 255), (1, 257)]),
    (14, 2, 64, 32, [(1, 1000), (1, 33), (0, 50), (1, 640)]),
    (6, 2, 128, 64, [(1, 3000)]),
    (32, 8, 128, 64, [(1, 100 + 77 * i) for i in range(9)]),
    (9, 3, 64, 16, RAGGED),
    (4, 1, 128, 32, RAGGED),
    (4, 4, 64, 16, [(130, 130)]),
    (8, 2, 128, 128, [(200, 900), (1, 300), (64, 64)]),
    (7, 1, 64, 256, [(37, 500), (129, 129)]),
    (128, 1, 64, 16, [(5, 90)]),
    (100, 1, 128, 1024, [(3, 1500), (1, 2)]),
    (12, 4, 64, 32, [(300, 301), (1, 900), (17, 18), (0, 3), (256, 512)]),
    (2, 2, 128, 16, [(513, 1030)]),
    (4, 2, 64, 64, [(3, 0), (2, 1), (1, 0)]),
    # many key tiles a segment: the ring of tiles goes round, split blocks (also with heads of 64) and whole ones
    (16, 8, 128, 64, [(1, 9000 + 100 * i) for i in range(8)]),
    (16, 8, 64, 64, [(1, 9000 + 100 * i) for i in range(8)]),
    (8, 1, 128, 128, [(300, 8500)]),
    (32, 8, 64, 32, [(300, 5000), (33, 5100)]),
    # more sequences than a warp has lanes, some without new tokens or without keys
    (4, 2, 64, 16, [(i % 3, (37 * i) % 400) for i in range(110)]),
    (2, 1, 128, 32, [(0, 50)] * 40 + [(1, 900)] + [(0, 0)] * 40 + [(70, 1500)]),
    # clusters of 7, 5 and 3 CTAs where few tokens are served by clusters
    (6, 3, 64, 16, [(1, 700 + i) for i in range(7)]),
    (5, 5, 128, 16, [(1, 900 - 33 * i) for i in range(5)]),
    (16, 16, 64, 16, [(1, 300), (1, 17), (1, 0)]),
]


@pytest.mark.parametrize("H,Hkv,d,page,pairs", ATTENTION)
@pytest.mark.parametrize("sigma", [1.0, 3.0])
def test_attention_over_the_cache(attnw, variant, H, Hkv, d, page, pairs, sigma):
    if variant == "few" and H // Hkv > 8:
        pytest.skip("more heads than it serves")
    c = Paged(pairs, Hkv, d, page, seed=7, front=1, behind=2, sigma=sigma)
    check_attention(attnw, c, c.normal(c.tokens, H, d, sigma=sigma), d ** -0.5)


@pytest.mark.parametrize("H,Hkv,d,page,pairs", [ATTENTION[3], ATTENTION[10]])
def test_attention_with_strided_queries_and_zero_scale(attnw, variant, H, Hkv, d, page, pairs):
    c = Paged(pairs, Hkv, d, page, seed=3)
    qkv = c.normal(c.tokens, H + 2 * Hkv, d)
    check_attention(attnw, c, qkv[:, :H], 0.1)
    head_major = c.normal(H, c.tokens, d)
    check_attention(attnw, c, head_major.transpose(0, 1), 0.0, with_mass=False)


def test_attention_with_bad_pages_lengths_and_starts(attnw, variant):
    c = Paged([(2, 80), (3, 80), (70, 80), (4, 30)], 2, 64, 16, width=5)
    c.table[0, 1], c.table[1, 4], c.table[2, 0] = -1, c.pages, 2 ** 31 - 1   # read as zeros
    c.lengths[3] = -5                                                     # counts as 0
    check_attention(attnw, c, c.normal(c.tokens, 4, 64), 0.125)
    c = Paged([(2, 80), (3, 80)], 2, 64, 16, width=5)
    c.lengths[0] = 2 ** 31 - 1                                            # counts as 80
    check_attention(attnw, c, c.normal(c.tokens, 4, 64), 0.125)
    Q, O = c.normal(5, 4, 64), torch.full((5, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    for starts in ([9, 9, 9], [-5, -4, -3], [5, 5, 5]):                    # nobody's tokens
        attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, torch.tensor(starts, dtype=torch.int32, device="cuda"), 0.125, O=O)
        assert bool((O == 7.0).all())
    for starts in ([0, 3, 1], [3, 0, 5], [0, 2 ** 31 - 1, 5], [-2 ** 31, 2 ** 31 - 1, -2 ** 31]):  # no order: some values, no fault
        attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, torch.tensor(starts, dtype=torch.int32, device="cuda"), 0.125, O=O,
                         mass=torch.zeros(2, 2, 80, device="cuda"))
    torch.cuda.synchronize()
    assert attnw.query_status() == 0


def test_attention_over_shared_pages_is_the_same_for_both(attnw, variant):
    # two sequences whose tables name the same pages: a prompt that both begin with
    c = Paged([(1, 300), (1, 300)], 2, 64, 16, seed=2)
    c.table[1] = c.table[0]
    Q = c.normal(2, 8, 64)
    Q[1] = Q[0]
    O, lse, mass = check_attention(attnw, c, Q, 0.125)
    assert torch.equal(O[0], O[1]) and torch.equal(lse[0], lse[1])


def test_caches_beyond_two_and_four_gigabytes(attnw, variant):
    # places whose offsets pass 2^31 elements and 2^32 bytes
    pages, Hkv, page, d = 40000, 8, 64, 128
    K, V = (torch.empty(pages, Hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = Paged([(3, 130), (1, 64)], Hkv, d, page, seed=4)
    ids = torch.tensor([[39999, 33000, 7], [39998, 0, 0]], dtype=torch.int32, device="cuda")
    for b in range(2):
        for i in range(-(-c.pairs[b][1] // page)):
            K[int(ids[b, i])], V[int(ids[b, i])] = c.K[int(c.table[b, i])], c.V[int(c.table[b, i])]
    Q = c.normal(4, 16, d)
    mass = torch.zeros(2, Hkv, 3 * page, device="cuda")
    want = attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, 0.09, mass=mass)
    got = attnw.attn_paged(Q, K, V, ids, c.lengths, c.starts, 0.09, mass=mass)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    k, v = c.normal(4, Hkv, d), c.normal(4, Hkv, d)
    attnw.cache_append(None, k, v, K, V, ids, c.lengths, c.starts)
    assert torch.equal(K[7, :, 0:2], k[1:3].transpose(0, 1)) and torch.equal(V[39998, :, 63], v[3]) and torch.equal(K[33000, :, 63], k[0])
    out = torch.tensor([[38000], [38001]], dtype=torch.int32, device="cuda")
    kept, _, _ = attnw.cache_evict(K, V, ids, c.lengths, want[1], 40, 4, table_out=out)
    for b in range(2):
        src = kept[b, 5].long()
        assert torch.equal(V[38000 + b, 5, :40], V[ids[b].long()[src // page], 5, src % page])


def test_attention_captured_replayed_and_on_two_streams(attnw, variant):
    pairs = [(1, 1000), (1, 77), (40, 300)] if variant != "few" else [(1, 1000), (1, 77), (2, 300)]
    c = Paged(pairs, 2, 64, 16, seed=9)
    Q, scale = c.normal(c.tokens, 8, 64), 0.125
    mass = torch.zeros(3, 2, c.width * 16, device="cuda")
    call = lambda q, m: attnw.attn_paged(q, c.K, c.V, c.table, c.lengths, c.starts, scale, mass=m)  # noqa: E731
    want = call(Q, mass)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graphs, results, queries = [], [], []
    for _ in range(2):
        q = Q.clone()
        with torch.cuda.stream(stream):
            call(q, mass)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            results.append(call(q, mass))
        graphs.append(g)
        queries.append(q)
    queries[1].mul_(-1)
    other = call(queries[1], mass)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(20):  # the graphs side by side, and with a plain call
        for r in results:
            r[0].fill_(7.0)
            r[1].fill_(7.0)
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        with torch.cuda.stream(stream):
            plain = call(Q, mass)
        torch.cuda.synchronize()
        for got, ref in zip((*results, plain), (want, other, want)):
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    # replays read the lengths and the table as they are then
    c.lengths[0], c.lengths[1] = 500, 64
    c.K[c.table[2, 0].long()] = 0.5
    ref = call(Q, mass)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(results[0][0], ref[0]) and torch.equal(results[0][1], ref[1])
    # a stream given by its handle, the caller's memory
    O, m = torch.empty_like(Q), mass.clone()
    torch.cuda.synchronize()
    attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, scale, O=O, mass=m, mass_out=m, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(O, ref[0]) and torch.equal(m, ref[1])


def test_the_other_calls_captured(attnw):
    c = Paged([(2, 70), (1, 40)], 2, 64, 16, seed=8, spare=8)
    f = attnw.rope_frequencies(64).cuda()
    pos = torch.tensor([68, 69, 39], dtype=torch.int32, device="cuda")
    q, k, v = c.normal(3, 4, 64), c.normal(3, 2, 64), c.normal(3, 2, 64)
    mass = torch.rand(2, 2, c.width * 16, device="cuda")
    out = torch.tensor(c.spare[:6], dtype=torch.int32, device="cuda").view(2, 3)
    x, xpos = c.normal(1, 4, 9, 64), torch.arange(9, dtype=torch.int32, device="cuda")[None]

    def run():
        return (attnw.rope(x, xpos, f), attnw.cache_append(q, k, v, c.K, c.V, c.table, c.lengths, c.starts, pos, f),
                *attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, 33, 5, table_out=out))

    want = [t.clone() for t in run()]
    K, V = c.K.clone(), c.V.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        got = run()
    for _ in range(3):
        for t in got:
            t.zero_()
        c.K[out[:, :2].long()], c.V[out[:, :2].long()] = 0.0, 0.0  # (pages that the call fills)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(c.K.view(torch.int16), K.view(torch.int16)) and torch.equal(c.V.view(torch.int16), V.view(torch.int16))


def test_results_do_not_change_from_call_to_call(attnw, variant):
    c = Paged([(1, 4000), (1, 900), (1, 2500)] if variant == "few" else [(300, 4000), (1, 900), (1, 2500), (129, 700)], 2, 128, 16, seed=12)
    Q = c.normal(c.tokens, 8, 128)
    mass = torch.rand(len(c.pairs), 2, c.width * 16, device="cuda")
    first = attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, 0.1, mass=mass)
    for _ in range(50):
        again = attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, 0.1, mass=mass)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_launches_behind_a_failure_write_nothing(attnw):
    c = Paged([(1, 2000), (200, 900), (0, 40), (2, 0)], 2, 64, 16, seed=6)
    Q = c.normal(c.tokens, 8, 64)
    O, lse = torch.full((c.tokens, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((c.tokens, 8), 7.0, device="cuda")
    mass, out = torch.zeros(4, 2, c.width * 16, device="cuda"), torch.full((4, 2, c.width * 16), 7.0, device="cuda")
    call = lambda: attnw.attn_paged(Q, c.K, c.V, c.table, c.lengths, c.starts, 0.125, O=O, lse=lse, mass=mass, mass_out=out)  # noqa: E731
    attnw.set_paged_variant("tensor_cores")
    try:
        attnw.selftest_wait_timeout(100000)
        torch.cuda.synchronize()
        for _ in range(3):
            call()
        torch.cuda.synchronize()
        assert all(bool((t == 7.0).all()) for t in (O, lse, out))
        assert attnw.query_status() & 0x80000000
        call()
        torch.cuda.synchronize()
        assert attnw.query_status() == 0 and not bool((O == 7.0).all(-1).any())
    finally:
        attnw.set_paged_variant("auto")


# ---- eviction -------------------------------------------------------------------------------------------------------------------

def evicted(c, mass, budget, recent):
    kept = torch.full((len(c.pairs), c.Hkv, budget), -1, dtype=torch.int32)
    for b, (_, length) in enumerate(c.pairs):
        for h in range(c.Hkv):
            w = mass[b, h, :length].cpu().double()
            w = torch.where(torch.isnan(w), torch.tensor(-math.inf, dtype=torch.float64), w)
            if length <= budget:
                chosen = torch.arange(length)
            else:
                nan_last = torch.isnan(mass[b, h, :length - recent].cpu()).to(torch.int64)
                order = sorted(range(length - recent), key=lambda i: (int(nan_last[i]), -float(w[i]), i))
                chosen = torch.tensor(sorted(order[:budget - recent]) + list(range(length - recent, length)))
            kept[b, h, :len(chosen)] = chosen.to(torch.int32)
    return kept


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("Hkv,d,page,budget,recent,pairs", [
    (1, 64, 16, 1, 0, [(0, 2)]),
    (2, 64, 16, 8, 8, [(0, 33), (0, 8), (0, 0), (0, 9)]),
    (3, 128, 16, 40, 5, [(0, 100), (0, 41), (0, 40), (0, 39), (0, 1)]),
    (8, 128, 64, 500, 64, [(0, 2100)]),
    (2, 128, 32, 1500, 0, [(0, 5000), (0, 1501), (0, 3000)]),
    (1, 64, 128, 4097, 1000, [(0, 9001)]),
    (40, 64, 16, 100, 17, [(0, 300 + i) for i in range(8)]),
])
@pytest.mark.parametrize("weights", ["spread", "ties", "equal", "odd"])
def test_eviction(attnw, Hkv, d, page, budget, recent, pairs, in_place, weights):
    c = Paged(pairs, Hkv, d, page, seed=budget, spare=1 + len(pairs) * -(-budget // page))
    C = c.width * page
    mass = torch.randn(len(pairs), Hkv, C, generator=c.gen).mul(2).exp()
    if weights == "ties":
        mass = (mass * 2).floor().clamp_max(3.0)
    elif weights == "equal":
        mass = torch.full_like(mass, 0.25)
    elif weights == "odd":
        pool = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, 1e-45, -1.0, 3e38, 1.0])
        mass = pool[torch.randint(0, 9, mass.shape, generator=c.gen)]
    mass = mass.cuda()
    if budget > C and in_place:
        pytest.skip("the pages in place hold fewer keys than the budget")
    kept_ref = evicted(c, mass, budget, recent)
    K0, V0, mass0 = c.K.clone(), c.V.clone(), mass.clone()
    width = c.width if in_place else -(-budget // page)
    out_table = None if in_place else torch.tensor(c.spare[:len(pairs) * width], dtype=torch.int32, device="cuda").view(len(pairs), width)
    kept, lengths, mass_out = attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, budget, recent, table_out=out_table, mass_out=mass if in_place else None)
    assert torch.equal(kept.cpu(), kept_ref)
    assert lengths.tolist() == [min(length, budget) for _, length in pairs]
    table = c.table if in_place else out_table
    bits = lambda x: x.view(torch.int32 if x.dtype == torch.float32 else torch.int16).cpu()  # noqa: E731
    want_K, want_V = K0.cpu().clone(), V0.cpu().clone()
    want_mass = torch.zeros(len(pairs), Hkv, width * page)
    for b in range(len(pairs)):
        n = int(lengths[b])
        to = torch.arange(n)
        to_page = table[b].cpu().long()[to // page]
        for h in range(Hkv):
            src = kept_ref[b, h, :n].long()
            from_page = c.table[b].cpu().long()[src // page]
            want_K[to_page, h, to % page] = K0.cpu()[from_page, h, src % page]
            want_V[to_page, h, to % page] = V0.cpu()[from_page, h, src % page]
            want_mass[b, h, :n] = mass0[b, h].cpu()[src]
    assert torch.equal(bits(c.K), bits(want_K)) and torch.equal(bits(c.V), bits(want_V))
    assert torch.equal(bits(mass_out), bits(want_mass))
    if not in_place:
        assert torch.equal(bits(mass), bits(mass0))


def test_eviction_ignores_bad_pages(attnw):
    c = Paged([(0, 100), (0, 100)], 2, 64, 16, spare=9)
    K0 = c.K.clone()
    mass = torch.rand(2, 2, c.width * 16, device="cuda")
    out = torch.tensor([[c.spare[0], -1, c.pages], [2 ** 31 - 1, c.spare[1], c.spare[2]]], dtype=torch.int32, device="cuda")
    c.table[0, 3] = -1
    kept, lengths, _ = attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, 40, 10, table_out=out)
    torch.cuda.synchronize()
    for b, i, p in ((0, 0, c.spare[0]), (1, 1, c.spare[1]), (1, 2, c.spare[2])):
        for t in range(16 * i, min(40, 16 * i + 16)):
            for h in range(2):
                s = int(kept[b, h, t])
                page = int(c.table[b, s // 16])
                if page >= 0:
                    assert torch.equal(c.K[p, h, t % 16], K0[page, h, s % 16])


# ---- a run of them together, as generating does ----------------------------------------------------------------------------------

@pytest.mark.parametrize("d,Hkv,G", [(64, 3, 4), (128, 2, 1)])
def test_generating(attnw, variant, d, Hkv, G):
    """Two prompts of different lengths go in by chunks, then some tokens one by one, with an eviction in between: each step's attention is that of the
    definition over the cache as it is, and before the eviction that of attn_fused over the whole sequence for its last token."""
    H, page, budget = Hkv * G, 16, 96
    gen = torch.Generator().manual_seed(5)
    total = [150, 61]
    x = {name: [torch.randn(n + 8, heads, d, generator=gen).bfloat16().cuda() for n in total] for name, heads in (("q", H), ("k", Hkv), ("v", Hkv))}
    f = attnw.rope_frequencies(d, 10000.0, scaling="linear", factor=2.0).cuda()
    width = 12
    K, V = (torch.full((2 * width, Hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.randperm(2 * width, generator=gen).to(torch.int32).cuda().view(2, width)
    mass = torch.zeros(2, Hkv, width * page, device="cuda")
    lengths = torch.zeros(2, dtype=torch.int32, device="cuda")
    seen = [0, 0]

    def step(counts):
        nonlocal mass, lengths
        starts = torch.tensor([0, counts[0], sum(counts)], dtype=torch.int32, device="cuda")
        lengths = lengths + torch.tensor(counts, dtype=torch.int32, device="cuda")
        q, k, v = (torch.cat([x[name][b][seen[b]:seen[b] + counts[b]] for b in range(2)]) for name in "qkv")
        pos = torch.cat([torch.arange(seen[b], seen[b] + counts[b], dtype=torch.int32) for b in range(2)]).cuda()
        q = attnw.cache_append(q, k, v, K, V, table, lengths, starts, pos, f)
        view = Paged.__new__(Paged)
        view.__dict__.update(pairs=list(zip(counts, lengths.tolist())), Hkv=Hkv, d=d, page=page, width=width, pages=2 * width, table=table, lengths=lengths,
                             starts=starts, K=K, V=V, gen=gen, tokens=sum(counts))
        O, _, _ = check_attention(attnw, view, q, d ** -0.5)
        _, mass = attnw.attn_paged(q, K, V, table, lengths, starts, d ** -0.5, mass=mass)
        for b in range(2):
            seen[b] += counts[b]
        return O

    step([100, 61])
    O = step([50, 0])
    whole = [attnw.rope(x[n][0][:150].transpose(0, 1)[None], torch.arange(150, dtype=torch.int32, device="cuda")[None], f) for n in "qk"]
    k, v = (t.repeat_interleave(G, 1) for t in (whole[1], x["v"][0][:150].transpose(0, 1)[None].contiguous()))
    same = attnw.attn_fused(whole[0], k.contiguous(), v.contiguous(), d ** -0.5)[0, :, -1]
    assert float((O[-1].float() - same.float()).abs().max()) <= 2.0 ** -6 * float(x["v"][0].float().abs().max())
    assert float((mass.sum((1, 2)).cpu() - torch.tensor([150.0, 61.0]) * H).abs().max()) <= 150 * H * 2.0 ** -16
    kept, lengths, mass = attnw.cache_evict(K, V, table, lengths, mass, budget, 10, mass_out=mass)
    assert lengths.tolist() == [96, 61]
    for _ in range(8 - 3):
        step([1, 1])
    assert lengths.tolist() == [101, 66]
