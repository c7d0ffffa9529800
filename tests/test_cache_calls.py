"""The calls around a paged cache: what they refuse, on the host, before anything touches a GPU; and the frequencies of rotary positions."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    from paper_2407_13885_b200 import build
    build.build_library()
    from paper_2407_13885_b200 import binding
    return binding


X, Y, POS, FREQ = 0x1000000, 0x9000000, 0x100, 0x200


def strides(*v):
    return (ctypes.c_longlong * len(v))(*v)


def test_rope_argument_errors(binding):
    def f(x=X, pos=POS, freq=FREQ, y=Y, B=2, H=4, N=100, d=64, rotary=64, xs=(4 * 6400, 6400, 64), ys=(4 * 6400, 6400, 64), layout=0, inverse=0, a=1.0,
          call=binding.lib.attnw_rope):
        return call(x, pos, freq, y, B, H, N, d, rotary, strides(*xs) if xs else None, strides(*ys) if ys else None, layout, inverse, a, None)
    for name in ("x", "pos", "freq", "y", "xs", "ys"):
        assert f(**{name: None}) == 1
    for name in ("B", "H", "N", "d"):
        assert f(**{name: 0}) == 2
    assert f(H=65536, xs=(0, 0, 64)) == 2
    assert f(d=32) == 4 and f(d=256) == 4 and f(rotary=8) == 4 and f(rotary=33) == 4
    assert f(rotary=80) == 2 and f(rotary=-16) == 2 and f(layout=2) == 2 and f(layout=-1) == 2
    assert f(a=math.nan) == 2 and f(a=math.inf) == 2
    assert f(x=X + 2) == 3 and f(y=Y + 8) == 3 and f(pos=POS + 2) == 3 and f(freq=FREQ + 4) == 3
    assert f(xs=(4 * 6400, 6400, 68)) == 3 and f(ys=(4 * 6400, 6400, 60)) == 3
    assert f(xs=(4 * 6400, 6400, 68), call=binding.lib.attnw_rope_f32, ys=(4 * 6400, 6400, 66)) == 3
    assert f(xs=(-25600, 6400, 64)) == 2 and f(ys=(25600, 0, 64)) == 2
    assert f(y=X + 16) == 7 and f(y=X, ys=(25600, 64, 256)) == 7
    assert f(pos=Y + 64) == 7 and f(freq=Y) == 7
    # columns of one array of tokens: four heads of 12, into the next four or into some of their own
    rows = (100 * 768, 64, 768)
    assert f(xs=rows, ys=rows, y=X + 2 * 128) == 7 and f(xs=rows, ys=rows, y=X - 2 * 128) == 7


def cache(binding, **changes):
    c = dict(K=0x10000000, V=0x20000000, table=0x1000, lengths=0x3000, pages=64, kv_heads=2, page=16, d=64, sequences=3, table_width=8)
    c.update(changes)
    return ctypes.byref(binding.Cache(**c))


BAD_CACHES = [(dict(K=None), 1), (dict(V=None), 1), (dict(table=None), 1), (dict(lengths=None), 1), (dict(pages=0), 2), (dict(kv_heads=0), 2), (dict(page=0), 2),
              (dict(d=0), 2), (dict(sequences=0), 2), (dict(table_width=0), 2), (dict(d=96), 4), (dict(page=8), 4), (dict(page=48), 4), (dict(page=2048), 4),
              (dict(pages=1 << 30), 2), (dict(sequences=40000), 2), (dict(table_width=1 << 25), 2), (dict(K=0x10000008), 3), (dict(V=0x20000002), 3),
              (dict(table=0x1001), 3), (dict(lengths=0x3002), 3)]


def append(binding, cache_ref, Q=X, K=0x2000000, V=0x3000000, Q_out=Y, s=(256, 64, 128, 64, 128, 64, 256, 64), starts=0x4000, pos=0x5000, freq=0x6000,
           tokens=40, heads=4, rotary=64, layout=0, a=1.0):
    return binding.lib.attnw_cache_append(cache_ref, Q, K, V, Q_out, strides(*s) if s else None, starts, pos, freq, tokens, heads, rotary, layout, a, None)


def paged(binding, cache_ref, Q=X, s=(256, 64), starts=0x4000, O=Y, lse=None, mass=None, mass_out=None, w=0x40000000, w_bytes=1 << 30, tokens=40, heads=4,
          scale=0.125):
    return binding.lib.attn_paged(cache_ref, Q, strides(*s) if s else None, starts, O, lse, mass, mass_out, w, w_bytes, tokens, heads, scale, None)


def evict(binding, cache_ref, table_out=0x5000, width=4, mass=X, mass_out=Y, kept=0xa000000, lengths_out=0xb000000, budget=50, recent=10):
    return binding.lib.attnw_cache_evict(cache_ref, table_out, width, mass, mass_out, kept, lengths_out, budget, recent, None)


@pytest.mark.parametrize("changes,code", BAD_CACHES)
def test_bad_caches(binding, changes, code):
    for call in (append, paged, evict):
        assert call(binding, cache(binding, **changes)) == code
        assert call(binding, None) == 1


def test_append_argument_errors(binding):
    c = cache(binding)
    f = lambda **k: append(binding, c, **k)  # noqa: E731
    for name in ("K", "V", "s", "starts", "Q", "Q_out", "pos", "freq"):
        assert f(**{name: None}) == 1
    assert f(tokens=0) == 2 and f(heads=0) == 2 and f(heads=65536) == 2 and f(layout=5) == 2 and f(a=math.inf) == 2
    assert f(rotary=72) == 2 and f(rotary=24) == 4
    for i in range(8):
        s = [256, 64, 128, 64, 128, 64, 256, 64]
        s[i] += 4
        assert f(s=s) == 3
    assert f(s=(256, 64, 128, 64, 128, 64, 0, 64)) == 2 and f(s=(256, 64, -128, 64, 128, 64, 256, 64)) == 2
    for name in ("Q", "K", "V", "Q_out"):
        assert f(**{name: X + 8}) == 3
        assert f(**{name: 0x10000000}) == 7 and f(**{name: 0x20000000 + 128}) == 7
    assert f(Q_out=X + 128) == 7 and f(Q_out=0x2000000) == 7 and f(Q_out=0x3000000) == 7
    assert f(starts=0x4002) == 3 and f(pos=0x5001) == 3 and f(freq=0x6004) == 3
    assert f(starts=Y) == 7 and f(starts=0x10000000) == 7 and f(pos=Y + 4) == 7
    assert append(binding, cache(binding, V=0x10000000 + 4096)) == 7 and append(binding, cache(binding, table=0x20000000)) == 7


def test_attention_argument_errors(binding):
    c = cache(binding)
    f = lambda **k: paged(binding, c, **k)  # noqa: E731
    for name in ("Q", "s", "starts", "O"):
        assert f(**{name: None}) == 1
    assert f(mass=0xa000000) == 1 and f(mass_out=0xa000000) == 1
    assert f(mass=0xa000000, mass_out=0xa000000, w=None) == 1
    assert f(mass=0xa000000, mass_out=0xa000000, w_bytes=0) == 2 and f(mass=0xa000000, mass_out=0xa000000, w_bytes=-5) == 2
    assert f(tokens=0) == 2 and f(heads=0) == 2 and f(heads=5) == 2 and f(heads=258, s=(258 * 64, 64)) == 4
    assert f(scale=-1.0) == 2 and f(scale=math.nan) == 2 and f(scale=math.inf) == 2
    assert f(s=(0, 64)) == 2 and f(s=(256, -64)) == 2 and f(s=(260, 64)) == 3
    assert f(Q=X + 2) == 3 and f(O=Y + 8) == 3 and f(lse=0xa000002) == 3 and f(starts=0x4001) == 3
    for at in (X, 0x10000000, 0x20000000, 0x4000 - 0x4000 % 16):
        assert f(O=at) == 7
    assert f(lse=Y) == 7 and f(lse=0x3000) == 7 and f(lse=X) == 7
    assert f(mass=0xa000000, mass_out=0xa000000 + 64) == 7 and f(mass=Y, mass_out=0xa000000) == 7 and f(mass=0xa000000, mass_out=Y) == 7
    assert f(mass=0xa000000, mass_out=0xa000000, w=Y) == 7
    assert f(tokens=1 << 29, heads=2, s=(128, 64)) == 2
    assert f(s=(1 << 39, 64)) == 2 and f(s=(1 << 62, 64)) == 2 and f(s=(256, 1 << 38)) == 2


def test_evict_argument_errors(binding):
    c = cache(binding)
    f = lambda **k: evict(binding, c, **k)  # noqa: E731
    for name in ("mass", "mass_out", "kept", "lengths_out"):
        assert f(**{name: None}) == 1
    assert f(budget=0) == 2 and f(budget=65) == 2 and f(recent=-1) == 2 and f(recent=51) == 2 and f(width=0) == 2
    assert f(table_out=0x1000, width=4) == 2   # the cache's own table has 8 columns
    assert f(mass=X + 2) == 3 and f(kept=0xa000001) == 3 and f(table_out=0x5002) == 3
    assert f(lengths_out=0x3000) == 7 and f(kept=X) == 7 and f(mass_out=X) == 7 and f(mass_out=X + 16) == 7 and f(kept=0x10000000) == 7
    assert f(kept=Y) == 7 and f(lengths_out=0xa000000) == 7 and f(lengths_out=0x5000) == 7


def test_paged_variant_knob(binding):
    lib = binding.lib
    assert lib.attnw_set_paged_variant(3) == 2 and lib.attnw_set_paged_variant(-1) == 2
    for v in (1, 2, 0):
        assert lib.attnw_set_paged_variant(v) == 0


def test_workspace_needs_a_cache(binding):
    assert binding.lib.attn_paged_workspace(None, 4, 4, 1) == 0
    assert binding.lib.attn_paged_workspace(cache(binding), 0, 4, 1) == 0 and binding.lib.attn_paged_workspace(cache(binding), 4, 5, 1) == 0
    for changes, _ in BAD_CACHES:
        assert binding.lib.attn_paged_workspace(cache(binding, **changes), 4, 4, 1) == 0
    assert binding.lib.attn_paged_workspace(cache(binding), 4, 4, 1) > 0
    # a longer table may need more, never less
    sizes = [binding.lib.attn_paged_workspace(cache(binding, table_width=w), 40, 4, 0) for w in (1, 8, 63, 64, 1000)]
    assert sizes == sorted(sizes) and sizes[0] == 0


def test_host_tensors_and_shapes_are_refused(binding):
    x = torch.zeros(1, 1, 8, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, 8, dtype=torch.int32)
    for call in (lambda: binding.rope(x, i, i), lambda: binding.cache_append(None, x[0], x[0], x, x, i, i[0], i[0]),
                 lambda: binding.attn_paged(x[0], x, x, i, i[0], i[0], 1.0), lambda: binding.cache_evict(x, x, i, i[0], i, 1, 0),
                 lambda: binding.rope(None, i, i)):
        with pytest.raises(TypeError, match="must be a CUDA tensor"):
            call()


def fake_cache(device="cuda:0"):
    e = lambda *s, t=torch.int32: torch.empty(*s, dtype=t, device=device)  # noqa: E731
    K, V = (e(16, 2, 16, 64, t=torch.bfloat16) for _ in range(2))
    return K, V, e(3, 4), e(3), e(4)


def test_shapes_types_and_devices_are_refused(binding):
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        K, V, table, lengths, starts = fake_cache()
        e = lambda *s, t=torch.bfloat16, device="cuda:0": torch.empty(*s, dtype=t, device=device)  # noqa: E731
        q, kv, mass, f = e(5, 4, 64), e(5, 2, 64), e(3, 2, 64, t=torch.float32), e(32, t=torch.float64)
        pos = e(5, t=torch.int32)
        x, xpos = e(1, 2, 5, 64), e(1, 5, t=torch.int32)
        far = e(5, 4, 64, device="cuda:1")
        for exc, call in (
                (TypeError, lambda: binding.rope(x.half(), xpos, f)), (TypeError, lambda: binding.rope(x, xpos.long(), f)),
                (TypeError, lambda: binding.rope(x, xpos, f.float())), (ValueError, lambda: binding.rope(x[0], xpos, f)),
                (ValueError, lambda: binding.rope(x, xpos[:, :4], f)), (ValueError, lambda: binding.rope(x.transpose(2, 3), xpos, f)),
                (ValueError, lambda: binding.rope(x, xpos, f, layout="rows")), (TypeError, lambda: binding.rope(x, xpos, f, out=x.float())),
                (ValueError, lambda: binding.cache_append(q, kv, kv[:, :1], K, V, table, lengths, starts, pos, f)),
                (ValueError, lambda: binding.cache_append(q[:4], kv, kv, K, V, table, lengths, starts, pos, f)),
                (ValueError, lambda: binding.cache_append(q, kv, kv, K, V, table, lengths, starts, pos)),
                (ValueError, lambda: binding.cache_append(None, kv, kv, K, V, table, lengths, starts, Q_out=q)),
                (ValueError, lambda: binding.cache_append(q, kv, kv, K, V, table, lengths, starts[:3], pos, f)),
                (ValueError, lambda: binding.cache_append(q, kv, kv, K, V[:3], table, lengths, starts, pos, f)),
                (TypeError, lambda: binding.cache_append(q, kv, kv, K.half(), V, table, lengths, starts, pos, f)),
                (ValueError, lambda: binding.attn_paged(q[..., :32], K, V, table, lengths, starts, 1.0)),
                (ValueError, lambda: binding.attn_paged(q, K, V, table, lengths[:2], starts, 1.0)),
                (ValueError, lambda: binding.attn_paged(q, K, V, table, lengths, starts, 1.0, mass=mass[..., :48])),
                (ValueError, lambda: binding.attn_paged(q, K, V, table, lengths, starts, 1.0, mass_out=mass)),
                (ValueError, lambda: binding.attn_paged(q, K, V, table, lengths, starts, 1.0, lse=mass[0])),
                (TypeError, lambda: binding.attn_paged(q, K, V, table.long(), lengths, starts, 1.0)),
                (ValueError, lambda: binding.attn_paged(far, K, V, table, lengths, starts, 1.0)),
                (ValueError, lambda: binding.cache_evict(K, V, table, lengths, mass[:2], 8, 0)),
                (ValueError, lambda: binding.cache_evict(K, V, table, lengths, mass, 8, 0, table_out=table[:2])),
                (TypeError, lambda: binding.cache_evict(K, V, table, lengths, mass.half(), 8, 0))):
            with pytest.raises(exc):
                call()


def test_frequencies(binding):
    f = binding.rope_frequencies(64, 10000.0)
    assert f.dtype == torch.float64 and f.numel() == 32 and float(f[0]) == 1.0
    assert abs(float(f[-1]) - 10000.0 ** (-62 / 64)) < 1e-18
    assert torch.equal(binding.rope_frequencies(64, scaling="linear", factor=4.0), f / 4)
    base = binding.rope_frequencies(64, scaling="base", factor=4.0)
    assert float(base[0]) == 1.0 and abs(float(base[-1] / f[-1]) - 0.25) < 1e-12
    parts = binding.rope_frequencies(64, scaling="by_parts", factor=4.0, original=2048)
    turns = 2048 * f / (2 * math.pi)
    assert torch.equal(parts[turns >= 4], f[turns >= 4]) and torch.equal(parts[turns <= 1], f[turns <= 1] / 4)
    between = (turns < 4) & (turns > 1)
    assert bool(between.any()) and bool(((parts < f) & (parts > f / 4))[between].all())
    assert binding.rope_frequencies(0).numel() == 0
    for bad in (dict(rotary=3), dict(rotary=-2), dict(rotary=64, base=0.0), dict(rotary=64, base=math.nan), dict(rotary=64, factor=0.0),
                dict(rotary=64, scaling="squares"), dict(rotary=2, scaling="base"), dict(rotary=64, scaling="by_parts"),
                dict(rotary=64, scaling="by_parts", original=8, low=4.0, high=1.0)):
        with pytest.raises(ValueError):
            binding.rope_frequencies(**bad)
