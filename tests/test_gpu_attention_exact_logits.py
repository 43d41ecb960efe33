"""cc_paged_attention on logits of hundreds that are exact, so that nothing but the softmax and the sums can be off."""
import math

import pytest
import torch

from cache_util import D, Cache, assert_attention, attend, attend_reference
from gpu_util import ctx

pytestmark = pytest.mark.gpu


def check(cache, hq, new, scale, seed, causal=True):
    """q and K are small integers, so products sum exactly in f32 in any order, and the scale is a power of two.  What is left of
    a logit's error: its product with scale * log2(e) in f32 is rounded once, 2^-24 of it, and the factor itself is off by 2^-24
    of what lies between a logit and its row's largest one, at most as much.  Both together in the place of the error that sums of
    products have."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-2, 3, (sum(new), hq, D), generator=g, device="cuda").bfloat16()
    _, out, lse = attend(ctx(), cache, hq, new, q=q, causal=causal, scale=scale)
    assert ctx().poll() == 0
    o, l, size, reach = attend_reference(cache, q, new, causal, scale)
    largest = torch.zeros_like(l)
    at = 0
    for s, t in enumerate(new):
        k = cache.k[cache.rows(s)].double().repeat_interleave(hq // cache.hkv, 1)
        for i in range(at, at + t, 64):
            j = min(at + t, i + 64)
            largest[i:j] = abs(scale) * torch.einsum("thd,nhd->thn", q[i:j].double(), k).abs().amax(-1)
        at += t
    assert_attention(out, lse, (o, l, size, largest * 2.0 ** -23 / 2.0 ** -16))


def integers(cache, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    for s, n in enumerate(cache.lens):
        cache.k[cache.rows(s)] = torch.randint(-4, 5, (n, cache.hkv, D), generator=g, device="cuda").bfloat16()
    return cache


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("scale", [0.125, 1.0, -1.0])
@pytest.mark.parametrize("new", [1, 3, 40, 64, 300])
def test_keys_far_above_their_neighbours(new, scale, causal):
    """Every 130th key eight times as large: references jump by hundreds, in either half of a tile and in the middle of a problem."""
    cache = integers(Cache([1200, 700], 2, 16, seed=31), 41)
    for s in range(2):
        cache.k[cache.rows(s)[5::130]] *= 8
    check(cache, 8, [new, new], scale, new, causal)


@pytest.mark.parametrize("new", [1, 4, 50, 200])
def test_ascending_logits(new):
    """Keys that grow along the cache, up to 16 times: nearly every tile replaces the reference."""
    cache = integers(Cache([1500], 2, 16, seed=32), 42)
    r = cache.rows(0)
    cache.k[r] = cache.k[r] * (1 + torch.arange(1500, device="cuda") // 100)[:, None, None]
    check(cache, 8, [new], 0.5, new)


@pytest.mark.parametrize("new", [[1], [5], [38], [130]])
def test_parts_of_a_problem_with_references_far_apart(new):
    """A long cache is cut between blocks, whose references differ by more than a probability's range."""
    cache = integers(Cache([20000], 2, 64, seed=33), 43)
    r = cache.rows(0)
    cache.k[r[7000:9000]] *= 4
    cache.k[r[15000:15100]] *= 4
    check(cache, 8, new, 1.0, new[0])


@pytest.mark.parametrize("group", [7, 16])
@pytest.mark.parametrize("new", [1, 30])
def test_equal_largest_logits(group, new):
    """Several keys share the largest logit exactly: the result is near the mean of their values, the smallest step counts."""
    cache = integers(Cache([900], 1, 16, seed=34), 44)
    r = cache.rows(0)
    cache.k[r[[3, 70, 300, 301, 555]]] = 32.0
    g = torch.Generator(device="cuda").manual_seed(9)
    q = torch.randint(1, 3, (new, group, D), generator=g, device="cuda").bfloat16()
    _, out, lse = attend(ctx(), cache, group, [new], q=q, scale=0.25)
    assert ctx().poll() == 0
    mean = cache.v[r[[3, 70, 300, 301, 555]], 0].double().mean(0)
    # probabilities of 1, exact sums: one rounding of the output, the others' share is below 2^-100
    assert ((out.double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 1e-6).all()
    top = q.double().sum(-1) * 32 * 0.25 + math.log(5)
    assert ((lse.double() - top).abs() <= top.abs() * 2.0 ** -22).all()
