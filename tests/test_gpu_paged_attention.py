"""cc_paged_attention against 64 bits: lengths, heads, pages, masks, strides, lengths on the device."""
import math

import pytest
import torch

from cache_util import D, Cache, assert_attention, attend, attend_reference
from gpu_util import ctx
from paper_2604_10235_b200 import binding as cc

pytestmark = pytest.mark.gpu

HEADS = [(8, 2), (32, 8), (28, 4), (5, 5), (16, 1)]


def check(cache, hq, new, causal=True, scale=0.0, **more):
    q, out, lse = attend(ctx(), cache, hq, new, causal=causal, scale=scale, **more)
    assert ctx().poll() == 0
    assert_attention(out, lse, attend_reference(cache, q, new, causal, scale or None))


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000])
def test_one_token(hq, hkv, n):
    check(Cache([n], hkv, 16, seed=n), hq, [1])


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (28, 4)])
def test_batches_of_tokens(hq, hkv, page):
    lens = [1, 300, 0, 77, 64, 4099, 128, 9, 5, 1023]
    check(Cache(lens, hkv, page, seed=page), hq, [1] * len(lens))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new,lens", [([5], [5]), ([3, 0, 8, 2], [700, 9, 8, 2]), ([1, 130, 17], [50, 130, 400]),
                                      ([4, 4], [2, 0]), ([33], [20])])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (28, 4), (4, 4)])
def test_chunks(hq, hkv, new, lens, causal):
    """Among them chunks longer than the cache: their first tokens attend to nothing when the mask is causal."""
    check(Cache(lens, hkv, 16, seed=len(lens)), hq, new, causal)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (28, 4), (7, 1)])
@pytest.mark.parametrize("new,n", [(64, 64), (200, 1000), (257, 513), (600, 600), (129, 4000)])
def test_long_chunks(hq, hkv, new, n):
    check(Cache([n], hkv, 32, seed=n), hq, [new])


def test_all_lengths_up_to_two_tiles():
    lens = list(range(200, 264))
    check(Cache(lens, 2, 8, seed=3), 8, [1] * 64)
    check(Cache(lens, 2, 8, seed=4), 8, [(7 * i) % 40 for i in range(64)])


def test_one_head_over_a_long_cache():
    check(Cache([70001], 1, 64, seed=1), 7, [1])
    check(Cache([70001], 1, 64, seed=2), 7, [40])


@pytest.mark.parametrize("new", [1, 3, 130])
def test_many_tiles_per_sm(new):
    """Rings of tiles that go round many times."""
    check(Cache([9000, 5000, 7001, 130, 11000, 8000, 9999, 4000, 12000, 6000], 8, 16, seed=23), 32, [new] * 10)


def test_largest_batch_and_many_heads():
    check(Cache([50 + i for i in range(64)], 32, 16, seed=2), 32, [1] * 64)


@pytest.mark.parametrize("new", [1, 6, 150])
def test_strides(new):
    """Queries as a slice of a fused projection, heads outermost in the pools, a padded output."""
    hq, hkv, page, n = 16, 4, 16, 333
    rows = (-(-n // page) + 3) * page
    cache = Cache([n], hkv, page, seed=9, kv_strides=(D + 8, rows * (D + 8)))
    fused = torch.randn((new, hq + 2 * hkv, D), device="cuda").bfloat16()
    q = fused[:, 2:2 + hq]
    big = torch.full((new, hq, 2 * D), 3.0, dtype=torch.bfloat16, device="cuda")
    out = big[:, :, D:]
    desc = cache.desc(hq, [new], q_strides=(q.stride(0), q.stride(1)), out_strides=(out.stride(0), out.stride(1)))
    cc.cc_paged_attention(ctx(), desc, q, cache.k, cache.v, out)
    assert ctx().poll() == 0
    assert_attention(out, None, attend_reference(cache, q, [new]))
    assert (big[:, :, :D] == 3.0).all()


def test_rows_behind_the_last_one_stay():
    cache = Cache([200, 90], 2, 16)
    q = torch.randn((30, 8, D), device="cuda").bfloat16()
    out = torch.full_like(q, 5.0)
    lse = torch.full((30, 8), 5.0, device="cuda")
    for new in ([3, 20], [1, 1]):
        cc.cc_paged_attention(ctx(), cache.desc(8, new), q, cache.k, cache.v, out, lse)
        assert ctx().poll() == 0
        assert (out[sum(new):] == 5.0).all() and (lse[sum(new):] == 5.0).all() or sum(new) < 23
        assert_attention(out[:sum(new)], lse[:sum(new)], attend_reference(cache, q[:sum(new)], new))
    assert (out[23:] == 5.0).all() and (lse[23:] == 5.0).all()


@pytest.mark.parametrize("scale", [1.0, 0.02, -0.1])
@pytest.mark.parametrize("new", [1, 70])
def test_scales(scale, new):
    check(Cache([500], 2, 16, seed=11), 8, [new], scale=scale)


@pytest.mark.parametrize("new", [1, 5, 100])
def test_rising_logits(new):
    """Keys that grow along the cache: the reference of the softmax is replaced again and again."""
    cache = Cache([1500], 2, 16, seed=12, poison=False)
    r = cache.rows(0)
    q = torch.randn((new, 8, D), device="cuda").bfloat16()
    ramp = torch.linspace(-40, 40, 1500, device="cuda")[:, None, None]
    cache.k[r] = (ramp * q.float().mean((0, 1)).sign() * 0.3 + cache.k[r].float()).bfloat16()
    _, out, lse = attend(ctx(), cache, 8, [new], q=q)
    assert ctx().poll() == 0
    assert_attention(out, lse, attend_reference(cache, q, [new]))


def test_lengths_on_the_device_and_their_bounds():
    lens = [900, 64, 1, 333]
    cache = Cache([1000] * 4, 4, 16, seed=6)
    now = torch.tensor(lens, dtype=torch.int32, device="cuda")
    desc = cache.desc(16, [1, 3, 2, 40], dev_kv_lens=now)
    ws = ctx().cache_workspace(desc)
    for change in (0, 17, 100, -300):
        now.copy_(torch.tensor(lens, dtype=torch.int32) + change)
        now.clamp_(min=0)
        q, out, lse = attend(ctx(), cache, 16, [1, 3, 2, 40], desc=desc, ws=ws)
        assert ctx().poll() == 0
        assert_attention(out, lse, attend_reference(cache, q, [1, 3, 2, 40], lens=now.tolist()))
    now.copy_(torch.tensor([1001, -1, 50, 60], dtype=torch.int32))          # clamped, and flagged
    q, out, lse = attend(ctx(), cache, 16, [1, 3, 2, 40], desc=desc, ws=ws)
    assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
    assert_attention(out, lse, attend_reference(cache, q, [1, 3, 2, 40], lens=[1000, 0, 50, 60]))


@pytest.mark.parametrize("new", [[1, 1], [60, 3]])
def test_equal_calls_give_equal_bits_whatever_the_workspace_holds(new):
    cache = Cache([9000, 3000], 4, 16, seed=8)
    desc = cache.desc(16, new)
    ws = ctx().cache_workspace(desc)
    ws.fill_(255)
    q, out, lse = attend(ctx(), cache, 16, new, desc=desc, ws=ws)
    for fill in (0, 127):
        ws.fill_(fill)
        _, again, lse2 = attend(ctx(), cache, 16, new, q=q, desc=desc, ws=ws)
        assert torch.equal(out.view(torch.int16), again.view(torch.int16)) and torch.equal(lse, lse2)
    assert ctx().poll() == 0


@pytest.mark.parametrize("new", [1, 90])
def test_sequences_that_share_pages(new):
    cache = Cache([500, 500], 2, 16, seed=5)
    cache.table[1] = cache.table[0]
    check(cache, 8, [new, new])


def test_far_rows_of_a_large_pool():
    """Offsets beyond 2^31 elements."""
    page, hkv = 128, 8
    pool = (1 << 31) // (page * hkv * D) + 40
    k = torch.empty((pool * page, hkv, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    for new in (1, 40):
        cache = Cache([300], hkv, page, seed=21, spare=0)
        ids = torch.tensor([pool - 1, 0, pool - 7], dtype=torch.int32, device="cuda")
        for i in range(3):
            k[ids[i] * page:(ids[i] + 1) * page] = cache.k[cache.table[0, i] * page:(cache.table[0, i] + 1) * page]
            v[ids[i] * page:(ids[i] + 1) * page] = cache.v[cache.table[0, i] * page:(cache.table[0, i] + 1) * page]
        cache.table, cache.pool, cache.k, cache.v = ids[None], pool, k, v
        check(cache, 32, [new])


def test_side_stream_and_graph_replays():
    cache = Cache([3000, 170], 4, 16, seed=14)      # bounds of the lengths that `now` takes below
    now = torch.tensor([2000, 50], dtype=torch.int32, device="cuda")
    for new in ([1, 1], [20, 30]):
        desc = cache.desc(16, new, dev_kv_lens=now)
        ws = ctx().cache_workspace(desc)
        q = torch.randn((sum(new), 16, D), device="cuda").bfloat16()
        out = torch.empty_like(q)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            cc.cc_paged_attention(ctx(), desc, q, cache.k, cache.v, out, ws=ws)
        side.synchronize()
        assert_attention(out, None, attend_reference(cache, q, new, lens=now.tolist()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            cc.cc_paged_attention(ctx(), desc, q, cache.k, cache.v, out, ws=ws)
        for step in range(3):
            now += 11
            q.normal_()
            out.zero_()
            graph.replay()
            assert ctx().poll() == 0
            assert_attention(out, None, attend_reference(cache, q, new, lens=now.tolist()))


@pytest.mark.parametrize("new", [1, 50])
def test_bad_pages_are_flagged_and_skipped(new):
    cache = Cache([400, 100], 2, 16, seed=15, poison=False)
    good = cache.table.clone()
    for bad in (-1, cache.pool, 2 ** 31 - 1, -2 ** 31):
        cache.table.copy_(good)
        cache.table[0, 7] = bad
        q, out, lse = attend(ctx(), cache, 8, [new, new])
        assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
        cache.table.copy_(good)
        ref = attend_reference(cache, q, [new, new])
        assert_attention(out[new:], lse[new:], tuple(x[new:] for x in ref))       # the other sequence is untouched
    q, out, lse = attend(ctx(), cache, 8, [new, new])
    assert ctx().poll() == 0
    assert_attention(out, lse, attend_reference(cache, q, [new, new]))


@pytest.mark.parametrize("new", [1, 50])
def test_tiles_without_a_good_page(new):
    cache = Cache([1000, 100], 2, 128, seed=15, poison=False)
    good = cache.table.clone()
    cache.table[0] = -1
    q, out, lse = attend(ctx(), cache, 8, [new, new])
    assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
    cache.table.copy_(good)
    ref = attend_reference(cache, q, [new, new])
    assert_attention(out[new:], lse[new:], tuple(x[new:] for x in ref))


@pytest.mark.parametrize("new", [1, 20])
def test_not_a_number_where_it_is_attended_to_and_only_there(new):
    cache = Cache([100, 90], 2, 16, seed=16)
    cache.k[cache.rows(0)[3], 0, 5] = math.nan
    cache.v[cache.rows(1)[4], 1, 9] = math.inf
    q, out, lse = attend(ctx(), cache, 8, [new, new])
    assert ctx().poll() == 0
    assert out[:new, :4].isnan().all() and lse[:new, :4].isnan().all()
    assert not out[:new, 4:].isnan().any()
    assert out[new:, 4:, 9].isinf().all() and torch.isfinite(out[new:, :4]).all()
    rest = [c for c in range(D) if c != 9]
    assert torch.isfinite(out[new:, 4:][..., rest]).all() and torch.isfinite(lse[new:]).all()


@pytest.mark.parametrize("heads,new,n", [((8, 2), 4, 70), ((8, 2), 3, 64), ((28, 4), 2, 129), ((8, 2), 40, 300), ((28, 4), 33, 1000),
                                         ((4, 4), 300, 700), ((16, 1), 70, 70)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_later_tokens_of_a_chunk_do_not_reach_earlier_ones(heads, new, n, bad):
    """Infinities and NaN in K and V of a token are seen by the tokens that attend to it only."""
    hq, hkv = heads
    cache = Cache([n, n + 5], hkv, 16, seed=n)
    for token in (new - 1, new // 2):
        clean_k, clean_v = cache.k.clone(), cache.v.clone()
        row = cache.rows(0)[n - new + token]
        cache.v[row, 0, 3] = bad
        cache.v[row, 0, 77] = bad
        cache.k[cache.rows(1)[n + 5 - new + token], hkv - 1, 9] = math.nan
        q, out, lse = attend(ctx(), cache, hq, [new, new])
        assert ctx().poll() == 0
        cache.k.copy_(clean_k)
        cache.v.copy_(clean_v)
        ref = attend_reference(cache, q, [new, new])
        g = hq // hkv
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        hit[token:new, :g, 3] = hit[token:new, :g, 77] = True
        if math.isnan(bad):
            assert out[hit].isnan().all()
        else:
            assert (out[hit] == bad).all()
        hit[new + token:, hq - g:] = True
        assert out[new + token:, hq - g:].isnan().all() and lse[new + token:, hq - g:].isnan().all()
        out, lse = out.clone(), lse.clone()
        out[hit] = ref[0].bfloat16()[hit]
        lse[new + token:, hq - g:] = ref[1].float()[new + token:, hq - g:]
        assert_attention(out, lse, ref)


@pytest.mark.parametrize("hq,hkv", [(17, 1), (48, 2), (64, 1), (100, 1), (128, 1), (12, 1)])
@pytest.mark.parametrize("new,n", [(1, 300), (5, 5), (9, 1000)])
def test_wide_groups(hq, hkv, new, n):
    check(Cache([n, n + 1], hkv, 16, seed=hq), hq, [new, 1])


@pytest.mark.parametrize("causal", [True, False])
def test_chunks_over_nothing_and_next_to_nothing(causal):
    check(Cache([0, 1, 0, 130], 2, 16, seed=1), 8, [40, 70, 1, 50], causal)


@pytest.mark.parametrize("page", [8, 128])
@pytest.mark.parametrize("new", [[30, 1, 200], [513]])
def test_chunks_on_small_and_large_pages(page, new):
    check(Cache([700 + 3 * t for t in new], 4, page, seed=page), 28, new)


@pytest.mark.parametrize("new", [1, 3, 64, 300])
@pytest.mark.parametrize("scale", [2.0, 40.0])
def test_logits_of_hundreds(new, scale):
    """Probabilities that underflow and references that jump by more than a probability's range from tile to tile."""
    cache = Cache([1200], 2, 16, seed=31)
    r = cache.rows(0)
    cache.k[r[::130]] *= 8
    check(cache, 8, [new], scale=scale)


@pytest.mark.parametrize("new", [1, 5, 90])
def test_equal_keys_give_the_mean(new):
    cache = Cache([777], 2, 16, seed=32)
    r = cache.rows(0)
    cache.k[r] = cache.k[r[:1]].clone()
    check(cache, 8, [new])


def test_mixed_batches_in_one_and_in_two_launches():
    """Single tokens beside chunks: together where they have few keys, in launches of their own where they have many."""
    check(Cache([500, 300, 90, 1000], 8, 16, seed=33), 32, [1, 100, 1, 1])
    check(Cache([30000, 300, 40000, 1000], 8, 16, seed=34), 32, [1, 100, 1, 1])


def test_two_streams_with_a_workspace_each():
    caches = [Cache([20000, 50], 4, 16, seed=35), Cache([9000], 4, 32, seed=36)]
    news = [[1, 1], [260]]
    descs = [c.desc(16, t) for c, t in zip(caches, news)]
    spaces = [ctx().cache_workspace(d) for d in descs]
    qs = [torch.randn((sum(t), 16, D), device="cuda").bfloat16() for t in news]
    outs = [torch.empty_like(q) for q in qs]
    streams = [torch.cuda.Stream() for _ in news]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, d, ws, q, out, st in zip(caches, descs, spaces, qs, outs, streams):
            with torch.cuda.stream(st):
                cc.cc_paged_attention(ctx(), d, q, c.k, c.v, out, ws=ws)
    torch.cuda.synchronize()
    assert ctx().poll() == 0
    for c, t, q, out in zip(caches, news, qs, outs):
        assert_attention(out, None, attend_reference(c, q, t))


def test_out_off_the_32_byte_grid():
    cache = Cache([100], 2, 16, seed=37)
    for new in (1, 40):
        q = torch.randn((new, 8, D), device="cuda").bfloat16()
        big = torch.full((new * 8 * D + 8,), 9.0, dtype=torch.bfloat16, device="cuda")
        out = big[8:].view(new, 8, D)
        cc.cc_paged_attention(ctx(), cache.desc(8, [new]), q, cache.k, cache.v, out)
        assert ctx().poll() == 0
        assert_attention(out, None, attend_reference(cache, q, [new]))
        assert (big[:8] == 9.0).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,new,lens", [
    (8, 2, [92], [256]), (32, 8, [26, 227, 251], [848, 655, 251]),            # a problem per CTA
    (28, 4, [41], [571]), (8, 2, [84], [728]),                               # a few CTAs per problem
    (8, 2, [300], [300]), (8, 2, [180], [40]),                               # blocks with fewer tiles than CTAs, or none
    (8, 2, [40, 40], [5000, 0]), (8, 2, [40, 70], [5000, 1]),
    (8, 2, [44, 31], [454, 16271]), (28, 4, [27], [9151]), (5, 1, [130], [14000])])      # many parts of a problem
def test_few_problems(hq, hkv, new, lens, causal):
    check(Cache(lens, hkv, 16, seed=len(new) + lens[0]), hq, new, causal)


@pytest.mark.parametrize("new", [[38], [90], [90, 3]])
def test_few_problems_shorter_on_the_device(new):
    cache = Cache([9000] * len(new), 2, 16, seed=31)
    now = torch.zeros(len(new), dtype=torch.int32, device="cuda")
    desc = cache.desc(8, new, dev_kv_lens=now)
    ws = ctx().cache_workspace(desc)
    for n in (9000, 0, 1, 128, 129, 1000, 8999):
        now.fill_(n)
        q, out, lse = attend(ctx(), cache, 8, new, desc=desc, ws=ws)
        assert ctx().poll() == 0
        assert_attention(out, lse, attend_reference(cache, q, new, lens=now.tolist()))
