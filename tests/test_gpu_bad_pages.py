"""cc_paged_attention where pages are missing: their slots take no part, in the sequence that has them as in the others."""
import math

import pytest
import torch

from cache_util import D, Cache, assert_attention, attend
from gpu_util import ctx
from paper_2604_10235_b200 import binding as cc

pytestmark = pytest.mark.gpu


def reference(cache, table, q, new, causal, lens=None):
    """As cache_util.attend_reference, over the slots whose page in ``table`` belongs to the pool."""
    hq, page = q.shape[1], cache.page
    g = hq // cache.hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(out)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    reach = torch.zeros_like(lse)
    at = 0
    for s, T in enumerate(new):
        n = cache.lens[s] if lens is None else lens[s]
        j = torch.arange(n, device="cuda")
        ids = table[s].long()[j // page]
        slots = j[(ids >= 0) & (ids < cache.pool)]
        if T and len(slots):
            rows = table[s].long()[slots // page] * page + slots % page
            k = cache.k[rows].double().repeat_interleave(g, 1)
            v = cache.v[rows].double().repeat_interleave(g, 1)
            t = torch.arange(T, device="cuda")
            qq = q[at + t].double()
            x = torch.einsum("thd,nhd->thn", qq, k) / math.sqrt(D)
            seen = slots[None, :] <= ((n - T + t)[:, None] if causal else n)
            x = x.masked_fill(~seen[:, None, :], -math.inf)
            some = seen.any(-1)
            p = torch.where(some[:, None, None], torch.softmax(x, -1), torch.zeros_like(x))
            out[at + t] = torch.einsum("thn,nhd->thd", p, v)
            size[at + t] = torch.einsum("thn,nhd->thd", p, v.abs())
            lse[at + t] = torch.where(some[:, None], torch.logsumexp(x, -1), lse[at + t])
            reach[at + t] = (torch.einsum("thd,nhd->thn", qq.abs(), k.abs())).amax(-1) / math.sqrt(D)
        at += T
    return out, lse, size, reach


def check(cache, hq, new, causal=True, **more):
    q, out, lse = attend(ctx(), cache, hq, new, causal=causal, **more)
    assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
    ref = reference(cache, cache.table, q, new, causal, more.get("lens"))
    none = ref[1] == -math.inf
    assert (out[none] == 0).all() and (lse[none] == -math.inf).all()
    assert_attention(out, lse, ref)


def lose(cache, s, pages):
    """Replaces entries of a row of the page table by ids outside the pool, each of another kind."""
    bad = [-1, cache.pool, 2 ** 31 - 1, -2 ** 31]
    for i, p in enumerate(pages):
        cache.table[s, p] = bad[i % 4]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("new", [1, 3, 50, 300])
def test_missing_pages_are_left_out(new, page, causal):
    """Pages anywhere, the first and the last among them, beside a sequence that has all its pages."""
    cache = Cache([1000, 700, 333], 2, page, seed=page)
    used = -(-1000 // page)
    lose(cache, 0, [0, 1, used // 2, used - 1])
    lose(cache, 2, range(0, -(-333 // page), 2))
    check(cache, 8, [new] * 3, causal)


@pytest.mark.parametrize("hq,hkv", [(28, 4), (16, 1), (128, 1), (5, 5)])
@pytest.mark.parametrize("new", [1, 2, 90])
def test_heads(hq, hkv, new):
    cache = Cache([515, 90], hkv, 16, seed=hq)
    lose(cache, 0, [3, 8, 9, 10, 11, 12, 13, 14, 15, 16, 32])
    check(cache, hq, [new, new])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new", [1, 4, 40, 200])
def test_sequences_without_a_page(new, causal):
    """Tokens that are left without a slot, in sequences of one tile and of many."""
    cache = Cache([500, 20, 9000], 2, 16, seed=3)
    lose(cache, 0, range(-(-500 // 16)))
    lose(cache, 1, range(2))
    check(cache, 8, [new] * 3, causal)
    lose(cache, 2, range(-(-9000 // 16)))
    check(cache, 8, [new] * 3, causal)


@pytest.mark.parametrize("n", [40, 130, 300])
def test_first_tokens_of_a_chunk_without_a_slot(n):
    """The pages of the first tokens are missing: later tokens see the rest."""
    cache = Cache([n, n], 2, 8, seed=n)
    lose(cache, 0, range(3))
    check(cache, 8, [n, n])
    check(cache, 2, [n, n])


@pytest.mark.parametrize("new", [[1], [7], [60], [513]])
def test_long_caches_cut_between_blocks(new):
    """Parts of a problem with and without slots are joined, also where whole parts have none."""
    cache = Cache([30000], 2, 64, seed=9)
    lose(cache, 0, list(range(100, 140)) + list(range(300, 460, 3)))
    check(cache, 8, new)
    lose(cache, 0, range(0, 460))
    check(cache, 8, new)


@pytest.mark.parametrize("new", [1, 80])
def test_lengths_on_the_device(new):
    cache = Cache([2000, 2000], 4, 16, seed=10)
    lose(cache, 0, [0, 5, 61, 62])
    now = torch.tensor([1000, 1500], dtype=torch.int32, device="cuda")
    q, out, lse = attend(ctx(), cache, 16, [new, new], desc=cache.desc(16, [new, new], dev_kv_lens=now))
    assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
    assert_attention(out, lse, reference(cache, cache.table, q, [new, new], True, [1000, 1500]))


@pytest.mark.parametrize("new", [1, 60])
def test_what_shared_memory_held_before_is_not_seen(new):
    """The missing page's place in the ring holds rows of other sequences, infinite ones among them."""
    cache = Cache([3000, 3000], 2, 16, seed=11)
    rows = cache.rows(1)
    cache.k[rows] = math.nan
    cache.v[rows] = math.inf
    clean = Cache([3000, 3000], 2, 16, seed=11)
    lose(cache, 0, range(1, 188, 2))
    q, out, lse = attend(ctx(), cache, 8, [new, new])
    assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
    ref = reference(clean, cache.table, q, [new, new], True)
    assert_attention(out[:new], lse[:new], tuple(x[:new] for x in ref))


@pytest.mark.parametrize("new", [1, 60])
def test_infinite_logits_alone_are_not_a_row_without_slots(new):
    cache = Cache([100], 2, 16, seed=12)
    cache.k[cache.rows(0), 0, 5] = -math.inf
    q = torch.randn((new, 8, D), device="cuda").bfloat16()
    q[..., 5] = 1.0
    _, out, lse = attend(ctx(), cache, 8, [new], q=q)
    assert ctx().poll() == 0
    assert out[:, :4].isnan().all() and torch.isfinite(out[:, 4:]).all() and torch.isfinite(lse[:, 4:]).all()


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, "pool"])
def test_forks_of_a_parent_without_its_last_page(bad):
    """The child's fresh page receives nothing, so the child does not get it: its old rows belong to nobody."""
    cache = Cache([20, 37], 2, 8, seed=4, spare=3, poison=False)
    cache.table[0, 2] = cache.pool if bad == "pool" else bad
    child = torch.full((2, 5), 55, dtype=torch.int32, device="cuda")
    k0, v0 = cache.k.clone(), cache.v.clone()
    cc.cc_fork_pages(ctx(), cache.desc(2), [cache.k], [cache.v], [0, 1], child, cache.free)
    assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
    assert child[0].tolist() == cache.table[0, :2].tolist() + [-1] * 3
    assert child[1].tolist() == cache.table[1, :4].tolist() + [int(cache.free[1])]
    rows = torch.arange(8, device="cuda") + cache.free[0].long() * 8
    assert torch.equal(cache.k[rows], k0[rows]) and torch.equal(cache.v[rows], v0[rows])
