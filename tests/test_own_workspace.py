"""Calls that are given no workspace: theirs belongs to the stream that the call runs on, so that torch's allocator
neither takes it from work of another stream nor gives it away while the call's own work is under way."""
import contextlib

import pytest
import torch

from paper_2604_10235_b200 import binding as cc


class FakeContext:
    """Records on which stream each workspace is allocated and on which each call runs."""
    device = 0

    def __init__(self):
        self.at, self.made, self.ran = "current", [], []

    def workspace(self, desc, n_layers):
        self.made.append(self.at)
        return "ws"

    def cache_workspace(self, desc):
        self.made.append(self.at)
        return "ws"

    def call(self, name, desc, *args):
        assert "ws" in args or "given" in args
        self.ran.append(args[-1])

    call_cache = call


@pytest.fixture()
def ctx(monkeypatch):
    fake = FakeContext()

    @contextlib.contextmanager
    def stream(s):
        before, fake.at = fake.at, s
        yield
        fake.at = before

    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device=None: (ptr, device))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(cc, "_raw", lambda s: s)
    monkeypatch.setattr(cc, "_raw_on", lambda c, s: s)
    return fake


CALLS = {"score": lambda c, **kw: cc.cc_score_window(c, None, 1, 2, 3, **kw),
         "topk": lambda c, **kw: cc.cc_topk_select(c, None, 1, 2, 3, 4, **kw),
         "layer": lambda c, **kw: cc.cc_compress_layer(c, None, 1, 2, 3, 4, 5, 6, 7, 8, **kw),
         "layers": lambda c, **kw: cc.cc_compress_layers(c, None, [1], [2], [3], 4, [5], [6], [7], [8], **kw),
         "attention": lambda c, **kw: cc.cc_paged_attention(c, None, 1, 2, 3, 4, **kw)}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_workspace_of_the_call_s_stream(ctx, name):
    CALLS[name](ctx, stream=4096)
    assert ctx.made == [(4096, 0)] and ctx.ran == [4096] and ctx.at == "current"
    CALLS[name](ctx)
    assert ctx.made[1:] == ["current"]
    CALLS[name](ctx, stream=4096, ws="given")
    assert len(ctx.made) == 2 and ctx.ran[-1] == 4096


@pytest.mark.parametrize("handle", [0, 1])
def test_the_default_stream_has_two_handles(ctx, handle):
    """CUDA's names for it are 0 and 1; torch knows the former."""
    CALLS["attention"](ctx, stream=handle)
    assert ctx.made == [(0, 0)] and ctx.ran == [handle]


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[1, 1], [40, 90]])
def test_attention_on_a_busy_stream(new):
    from cache_util import D, Cache, assert_attention, attend_reference
    from gpu_util import ctx as context
    cache = Cache([9000, 3000], 4, 16, seed=8)
    desc = cache.desc(16, new)
    size = context().cache_workspace_bytes(desc)
    q = torch.randn((sum(new), 16, D), device="cuda").bfloat16()
    out = torch.zeros_like(q)
    lse = torch.zeros(q.shape[:2], device="cuda")
    ref = attend_reference(cache, q, new)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # memory that the current stream still uses when it is freed
    torch.cuda._sleep(20_000_000)
    before = torch.full((size,), 3, dtype=torch.uint8, device="cuda")
    copy = before.clone()
    del before
    with torch.cuda.stream(side):
        torch.cuda._sleep(10_000_000)
    cc.cc_paged_attention(context(), desc, q, cache.k, cache.v, out, lse, stream=side.cuda_stream)
    # and memory that it asks for while the call is under way
    after = [torch.full((size,), 5, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert context().poll() == 0
    assert (copy == 3).all() and all((x == 5).all() for x in after)
    assert_attention(out, lse, ref)


@pytest.mark.gpu
def test_compression_on_a_busy_stream():
    from gpu_util import ctx as context
    hq, hkv, w, n, budget = 16, 4, 8, 5000, 1000
    d = cc.Desc(hq, hkv, w, n=n, budget=budget)
    torch.manual_seed(1)
    q = torch.randn((w, hq, 128), device="cuda").bfloat16()
    k, v = (torch.randn((n, hkv, 128), device="cuda").bfloat16() for _ in range(2))
    prior = (torch.rand(n, device="cuda") < 0.1).float()

    def buffers():
        return (torch.zeros((budget, hkv, 128), dtype=torch.bfloat16, device="cuda"),
                torch.zeros((budget, hkv, 128), dtype=torch.bfloat16, device="cuda"),
                torch.zeros((hkv, budget), dtype=torch.int32, device="cuda"),
                torch.zeros((1, hkv), dtype=torch.int32, device="cuda"))

    want, got = buffers(), buffers()
    cc.cc_compress_layer(context(), d, q, k, v, prior, *want)
    side = torch.cuda.Stream()
    size = context().workspace_bytes(d, 1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(10_000_000)
    cc.cc_compress_layer(context(), d, q, k, v, prior, *got, stream=side.cuda_stream)
    after = [torch.full((size,), 5, dtype=torch.uint8, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    assert context().poll() == 0
    assert all((x == 5).all() for x in after)
    for a, b in zip(want, got):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [[1, 1], [40, 90]])
def test_streams_by_handle(new):
    """CUDA's handles of the default streams, and a stream that is being captured."""
    from cache_util import D, Cache, assert_attention, attend_reference
    from gpu_util import ctx as context
    cache = Cache([9000, 3000], 4, 16, seed=9)
    desc = cache.desc(16, new)
    q = torch.randn((sum(new), 16, D), device="cuda").bfloat16()
    ref = attend_reference(cache, q, new)
    for handle in (0, 1, 2, torch.cuda.current_stream().cuda_stream):
        out = torch.zeros_like(q)
        torch.cuda.synchronize()
        cc.cc_paged_attention(context(), desc, q, cache.k, cache.v, out, stream=handle)
        torch.cuda.synchronize()
        assert context().poll() == 0
        assert_attention(out, None, ref)
    out = torch.zeros_like(q)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cc.cc_paged_attention(context(), desc, q, cache.k, cache.v, out, stream=side.cuda_stream)
    for _ in range(3):
        out.zero_()
        x = [torch.full((1 << 20,), 5, dtype=torch.uint8, device="cuda") for _ in range(4)]
        graph.replay()
        torch.cuda.synchronize()
        assert context().poll() == 0 and all((y == 5).all() for y in x)
        assert_attention(out, None, ref)
