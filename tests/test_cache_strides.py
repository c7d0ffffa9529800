"""Results whose own rows would lie on one another are refused, on the host, before anything touches a GPU.  Every call here is refused: one
whose strides are in order for a pointer that is not aligned (3, looked at behind the strides), so that nothing is ever launched."""
import pytest

from test_cache_calls import Y, append, binding, cache, strides  # noqa: F401 (binding is a fixture)

X_OFF = 0x1000002


@pytest.mark.parametrize("call,least", [("attnw_rope", 8), ("attnw_rope_f32", 4)])
def test_rope_rows_on_one_another(binding, call, least):  # noqa: F811
    def f(ys, B=2, H=4, N=100, xs=(25600, 6400, 64)):
        return getattr(binding.lib, call)(X_OFF, 0x100, 0x200, Y, B, H, N, 64, 64, strides(*xs), strides(*ys), 0, 0, 1.0, None)
    for ys in ((25600, 6400, 32), (25600, 64 - least, 6400), (32, 6400, 64), (6400, 6400, 64), (25600, 64, 64), (64, 6400, 64)):
        assert f(ys) == 2
    # a dimension of one index has no say, and what X does is not looked at
    assert f((25600, 6400, 64)) == 3
    assert f((0, 6400, 64), B=1) == 3 and f((25600, 6400, 0), N=1) == 3 and f((25600, 64, 64), H=1) == 3
    assert f((25600, 6400, 64), xs=(0, 0, 0)) == 3 and f((25600, 6400, 64), xs=(64, 64, 32)) == 3


def test_append_rows_on_one_another(binding):  # noqa: F811
    c = cache(binding)
    s = (256, 64, 128, 64, 128, 64)

    def f(*out, inputs=s, **k):
        return append(binding, c, K=X_OFF, s=(*inputs, *out), **k)

    assert f(256, 32) == 2 and f(64, 64) == 2 and f(32, 4096) == 2
    assert f(256, 64) == 3 and f(256, 0, heads=1) == 3 and f(0, 64, tokens=1) == 3
    assert f(256, 64, inputs=(0,) * 6) == 3   # inputs may be broadcast
