"""Results that a call on another stream makes: whose memory they are, and how long it stays theirs."""
import pytest
import torch

from paged_reference import Paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def attnw():
    from paper_2407_13885_b200 import binding
    yield binding
    assert binding.query_status() == 0


def calls(attnw):
    """name -> (call(stream), what it must give), for every call that makes its result."""
    gen = torch.Generator().manual_seed(1)
    q = torch.randn(1, 2, 192, 64, generator=gen).bfloat16().cuda()
    x, w = torch.randn(1, 128, 128, generator=gen).bfloat16().cuda(), torch.randn(2, 64, 128, generator=gen).bfloat16().cuda()
    s = torch.randn(64, 1000, generator=gen).cuda()
    c = Paged([(2, 70), (1, 40)], 2, 64, 16, seed=8, spare=8)
    f = attnw.rope_frequencies(64).cuda()
    pos = torch.tensor([68, 69, 39], dtype=torch.int32, device="cuda")
    qn, k, v = c.normal(3, 4, 64), c.normal(3, 2, 64), c.normal(3, 2, 64)
    rows = torch.arange(192, dtype=torch.int32, device="cuda")[None]
    mass = torch.rand(2, 2, c.width * 16, device="cuda")
    out = torch.tensor(c.spare[:6], dtype=torch.int32, device="cuda").view(2, 3)
    table = {
        "attnw_fused": lambda stream: attnw.attnw_fused(q, q, 0.125, stream=stream),
        "attn_fused": lambda stream: attnw.attn_fused(q, q, q, 0.125, stream=stream),
        "project_qk": lambda stream: attnw.project_qk(x, w, w, stream=stream),
        "softmax_rows": lambda stream: attnw.softmax_rows(s, stream=stream),
        "rope": lambda stream: attnw.rope(q, rows, f, stream=stream),
        "cache_append": lambda stream: attnw.cache_append(qn, k, v, c.K, c.V, c.table, c.lengths, c.starts, pos, f, stream=stream),
        "attn_paged": lambda stream: attnw.attn_paged(qn, c.K, c.V, c.table, c.lengths, c.starts, 0.125, mass=mass, stream=stream),
        "cache_evict": lambda stream: attnw.cache_evict(c.K, c.V, c.table, c.lengths, mass, 33, 5, table_out=out, stream=stream),
    }
    return {name: (call, [t.clone() for t in all_of(call(None))]) for name, call in table.items()}


def all_of(result):
    return result if isinstance(result, tuple) else (result,)


def owner(t):
    """The stream that the block of memory under `t` belongs to."""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not torch's memory")


NAMES = ["attnw_fused", "attn_fused", "project_qk", "softmax_rows", "rope", "cache_append", "attn_paged", "cache_evict"]


@pytest.mark.parametrize("name", NAMES)
def test_results_are_memory_of_the_stream_of_the_call(attnw, name):
    call, want = calls(attnw)[name]
    torch.cuda.synchronize()
    side, current = torch.cuda.Stream(), torch.cuda.current_stream()
    for stream in (side, side.cuda_stream, None, current):
        got = all_of(call(stream))
        torch.cuda.synchronize()
        assert len(got) == len(want)
        for a, b in zip(got, want):
            assert a.shape == b.shape and torch.equal(a, b)
            assert owner(a) == (current if stream is None or stream is current else side).cuda_stream
    with torch.cuda.stream(side):          # the current stream, and the one that was current before given by name
        here, there = all_of(call(None)), all_of(call(current))
        torch.cuda.synchronize()
        assert all(owner(a) == side.cuda_stream for a in here) and all(owner(a) == current.cuda_stream for a in there)


@pytest.mark.parametrize("name", NAMES)
def test_a_dropped_result_waits_for_the_current_stream(attnw, name):
    # The result of a call on another stream is read on the current one, and dropped while that has still to be done: nobody else gets the block.
    call, want = calls(attnw)[name]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = all_of(call(side))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(100_000_000)         # some 50 ms, so that the copies are still to come
    copies = [t.clone() for t in got]
    blocks = {t.data_ptr(): t.numel() * t.element_size() for t in got}
    del got
    with torch.cuda.stream(side):
        fresh = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in blocks.values()]
    assert not {t.data_ptr() for t in fresh} & set(blocks)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(copies, want))


def test_a_call_on_a_captured_stream(attnw):
    # torch's stream is captured; the calls name it, and a stream that the capture forks to.
    both = calls(attnw)
    for name in ("attn_fused", "attn_paged", "cache_evict"):
        call, want = both[name]
        stream, fork = torch.cuda.Stream(), torch.cuda.Stream()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            first = all_of(call(stream.cuda_stream))
            fork.wait_stream(stream)
            second = all_of(call(fork))
            stream.wait_stream(fork)
        for _ in range(3):
            for t in (*first, *second):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, want)) and all(torch.equal(a, b) for a, b in zip(second, want))
