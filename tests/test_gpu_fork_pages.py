"""cc_fork_pages: bit copies of last pages, rows of the child table, and the way from a compression to forked decoding."""
import numpy as np
import pytest
import torch

from cache_util import D, Cache, assert_attention, attend_reference
from gpu_util import ctx
from paper_2604_10235_b200 import binding as cc

pytestmark = pytest.mark.gpu


def fork_reference(cache, parents, free, k, v, width, lens=None):
    table = torch.full((len(parents), width), -1, dtype=torch.int32)
    src = cache.table.cpu()
    k, v = k.clone(), v.clone()
    for f, s in enumerate(parents):
        n = cache.lens[s] if lens is None else lens[s]
        full, rest = divmod(n, cache.page)
        table[f, :full] = src[s, :full]
        if rest:
            table[f, full] = int(free[f])
            a, b = int(src[s, full]) * cache.page, int(free[f]) * cache.page
            k[:, b:b + rest], v[:, b:b + rest] = k[:, a:a + rest], v[:, a:a + rest]
    return table, k, v


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("layers,hkv", [(1, 8), (3, 4), (70, 1)])
def test_against_the_definition(page, layers, hkv):
    lens = [0, 1, page - 1, page, page + 1, 5 * page + 3]
    parents = [5, 5, 0, 1, 2, 3, 4, 5]
    cache = Cache(lens, hkv, page, seed=page, spare=len(parents) + 2)
    shape = (layers,) + tuple(cache.k.shape)
    k, v = (torch.randint(-2 ** 15, 2 ** 15, shape, device="cuda", dtype=torch.int16) for _ in range(2))
    for width in (6, 9):
        child = torch.full((len(parents) + 1, width), 55, dtype=torch.int32, device="cuda")
        ref = fork_reference(cache, parents, cache.free, k, v, width)
        kk, vv = k.clone(), v.clone()
        cc.cc_fork_pages(ctx(), cache.desc(hkv), [x.view(torch.bfloat16) for x in kk], [x.view(torch.bfloat16) for x in vv],
                         parents, child[:-1], cache.free)
        assert ctx().poll() == 0
        assert torch.equal(child[:-1].cpu(), ref[0]) and (child[-1] == 55).all()
        assert torch.equal(kk, ref[1]) and torch.equal(vv, ref[2])


def test_children_as_rows_of_the_same_table_lengths_on_the_device_and_strides():
    page, hkv = 16, 2
    cache = Cache([100, 200], hkv, page, seed=1, spare=6, extra_cols=2, kv_strides=(D, 40 * page * D), poison=False)
    table = torch.full((6, cache.table.shape[1]), -1, dtype=torch.int32, device="cuda")
    table[:2] = cache.table
    cache.table = table
    now = torch.tensor([35, 200], dtype=torch.int32, device="cuda")
    k0, v0 = cache.k[None].clone(), cache.v[None].clone()
    ref = fork_reference(cache, [0, 1, 1, 0], cache.free, k0, v0, table.shape[1], lens=[35, 200])
    cc.cc_fork_pages(ctx(), cache.desc(hkv, dev_kv_lens=now), [cache.k], [cache.v], [0, 1, 1, 0], table[2:], cache.free)
    assert ctx().poll() == 0
    assert torch.equal(table[2:].cpu(), ref[0])
    assert torch.equal(cache.k, ref[1][0]) and torch.equal(cache.v, ref[2][0])
    with pytest.raises(cc.CodecompError) as e:
        cc.cc_fork_pages(ctx(), cache.desc(hkv), [cache.k], [cache.v], [0, 1, 1, 0], table[1:5], cache.free)
    assert e.value.status == cc.CC_ERR_INVALID_ARG


def test_bad_pages_are_flagged_and_skipped():
    cache = Cache([20, 37], 2, 8, seed=4, spare=3, poison=False)
    k0, v0 = cache.k.clone(), cache.v.clone()
    child = torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    free = cache.free.clone()
    for where in ("free", "last", "full"):
        cache.k.copy_(k0)
        cache.v.copy_(v0)
        table = cache.table.clone()
        f = free.clone()
        if where == "free":
            f[0] = cache.pool
        else:
            cache.table[0, 2 if where == "last" else 0] = -3
        cc.cc_fork_pages(ctx(), cache.desc(2), [cache.k], [cache.v], [0, 1], child, f)
        assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
        cache.table.copy_(table)
        ref = fork_reference(cache, [0, 1], free, k0[None], v0[None], 5)
        rows = torch.arange(8, device="cuda") + free[1].long() * 8
        assert torch.equal(child[1].cpu(), ref[0][1]) and torch.equal(cache.k[rows], ref[1][0][rows])
        rows0 = torch.arange(8, device="cuda") + free[0].long() * 8
        if where == "full":
            assert child[0].tolist() == [-1] + ref[0][0].tolist()[1:]
        else:
            assert torch.equal(cache.k[rows0], k0[rows0])


def test_from_a_compression_to_forked_decoding():
    """A prompt is compressed into pages, forked, continued by a chunk and then token by token from a captured graph:
    every output equals attention over the rows that were retained and appended, in 64 bits."""
    hq, hkv, page, n, budget = 16, 4, 16, 1000, 203
    steps, children, chunk = 5, 3, 37
    torch.manual_seed(3)
    pages_in, room = -(-n // page), -(-(budget + chunk + steps) // page)
    pool = pages_in + room * (children + 1) + 2
    perm = torch.randperm(pool).int().cuda()
    k, v = (torch.randn((pool * page, hkv, D), device="cuda").bfloat16() for _ in range(2))
    q_win = torch.randn((1, 8, hq, D), device="cuda").bfloat16()
    prior = (torch.rand(n, device="cuda") < 0.1).float()
    prompt = perm[:pages_in][None].contiguous()
    d = cc.Desc(hq, hkv, 8, seq_lens=[n], budgets=[budget], force_threshold=0.5, page_size=page, page_table=prompt,
                pool_pages=pool, out_page_table_stride=room)
    idx = torch.empty((hkv, budget), dtype=torch.int32, device="cuda")
    count = torch.empty((1, hkv), dtype=torch.int32, device="cuda")
    kept = torch.empty((1, room), dtype=torch.int32, device="cuda")
    fresh = perm[pages_in:].contiguous()
    k_before, v_before = k.clone(), v.clone()
    cc.cc_compress_layer(ctx(), d, q_win, k, v, prior, k, v, idx, count, fresh, kept)
    used = -(-budget // page)
    rest = fresh[used:].contiguous()
    table = torch.empty((children, room), dtype=torch.int32, device="cuda")
    parent = cc.CacheDesc(hq, hkv, [budget], page_size=page, page_table=kept, pool_pages=pool)
    cc.cc_fork_pages(ctx(), parent, [k], [v], [0] * children, table, rest)
    # pages for the tokens to come
    table[:, used:] = rest[children:children + children * (room - used)].view(children, room - used)
    rope = cc.RopePlan(128, base=1e6)
    # the rows as each child should see them, [children][slots][heads][d]
    tok = prompt[0].long()[idx.long() // page] * page + idx.long() % page
    heads = torch.arange(hkv, device="cuda")[:, None]
    seen_k = k_before[tok, heads].transpose(0, 1)[None].repeat(children, 1, 1, 1).double()
    seen_v = v_before[tok, heads].transpose(0, 1)[None].repeat(children, 1, 1, 1).double()
    freq = torch.from_numpy(np.array([1e6 ** (-2 * i / 128) for i in range(64)])).cuda()

    def turn(x, pos):
        z = torch.complex(x[..., :64].double(), x[..., 64:].double())
        z = z * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), pos.double()[:, None] * freq)[:, None]
        return torch.cat((z.real, z.imag), -1)

    now = torch.zeros(children, dtype=torch.int32, device="cuda")
    now.fill_(budget)

    def step(desc, t, bufs, ws):
        q_new, k_new, v_new, pos, q, out, lse = bufs
        cc.cc_rope_append(ctx(), desc, q_new, k_new, v_new, pos, q, k, v)
        cc.cc_paged_attention(ctx(), desc, q, k, v, out, lse, ws=ws)

    def buffers(t):
        total = children * t
        x = [torch.empty((total, h, D), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv, hq, hq)]
        return [x[0], x[1], x[2], torch.empty(total, dtype=torch.int32, device="cuda"), x[3], x[4],
                torch.empty((total, hq), device="cuda")]

    def fill(bufs, t, at):
        for b in bufs[:3]:
            b.normal_()
        bufs[3].copy_((at + torch.arange(t)).repeat(children))

    def verify(bufs, t):
        nonlocal seen_k, seen_v
        q_new, k_new, v_new, pos, q, out, lse = bufs
        # the cache holds bf16: the appended keys are rounded once
        seen_k = torch.cat((seen_k, turn(k_new, pos).bfloat16().double().view(children, t, hkv, D)), 1)
        seen_v = torch.cat((seen_v, v_new.double().view(children, t, hkv, D)), 1)
        total = seen_k.shape[1]
        rows = (table[:, :, None].long() * page + torch.arange(page, device="cuda")).reshape(children, -1)[:, :total]
        got = k[rows].double()
        off = (got - seen_k).abs()
        # Both sides are rounded to bf16: of a value next to a border one goes up and one down, each by half a step (2^-8 of the
        # value) at most, so they are a whole step apart.  Where x cos a and y sin a cancel, f32 leaves 1e-5.
        assert (off <= 2 * 2.0 ** -8 * seen_k.abs() + 1e-5).all().item()
        assert torch.equal(v[rows].double(), seen_v)
        cache = Cache([total] * children, hkv, page, poison=False)
        cache.table, cache.k, cache.v = table, k, v
        assert_attention(out, lse, attend_reference(cache, q, [t] * children))

    bound = [room * page] * children
    desc = cc.CacheDesc(hq, hkv, bound, [chunk] * children, page_size=page, page_table=table, pool_pages=pool, rope=rope,
                        dev_kv_lens=now)
    bufs = buffers(chunk)
    fill(bufs, chunk, n)
    now += chunk
    step(desc, chunk, bufs, ctx().cache_workspace(desc))
    assert ctx().poll() == 0
    verify(bufs, chunk)
    desc = cc.CacheDesc(hq, hkv, bound, page_size=page, page_table=table, pool_pages=pool, rope=rope, dev_kv_lens=now)
    bufs, ws = buffers(1), ctx().cache_workspace(desc)
    fill(bufs, 1, n + chunk)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(desc, 1, bufs, ws)
    for i in range(steps):
        fill(bufs, 1, n + chunk + i)
        now += 1
        graph.replay()
        assert ctx().poll() == 0
        verify(bufs, 1)
