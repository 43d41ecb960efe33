"""cc_rope_append against 64 bits: layouts, scalings, far positions, slots, strides, refusals of bad slots."""
import math

import numpy as np
import pytest
import torch

from cache_util import D, Cache
from gpu_util import ctx
from paper_2604_10235_b200 import binding as cc

pytestmark = pytest.mark.gpu

KINDS = {"plain": {}, "linear": dict(kind=cc.CC_ROPE_LINEAR, factor=3.0), "base": dict(kind=cc.CC_ROPE_BASE, factor=4.0),
         "bands": dict(kind=cc.CC_ROPE_BANDS, factor=8.0, base=5e5, attn_factor=1.2),
         "given": dict(kind=cc.CC_ROPE_GIVEN)}


def plan(dims, interleaved, kind):
    kw = dict(KINDS[kind])
    if kind == "given":
        kw["inv_freq"] = np.linspace(0.0, 9.0, dims // 2)
    return cc.RopePlan(dims, interleaved=interleaved, **kw), frequencies(dims, kind, kw), kw.get("attn_factor", 1.0)


def frequencies(dims, kind, kw):
    if kind == "given":
        return kw["inv_freq"]
    base, s = kw.get("base", 10000.0), kw.get("factor", 1.0)
    if kind == "base":
        base *= s ** (dims / (dims - 2))
    f = np.array([base ** (-2 * i / dims) for i in range(dims // 2)])
    if kind == "linear":
        f = f / s
    if kind == "bands":
        g = np.clip((8192 * f / (2 * math.pi) - 1.0) / 3.0, 0, 1)
        f = (1 - g) * f / s + g * f
    return f


def rotated(x, pos, f, dims, interleaved, factor):
    """64 bits, and the size of what each value is summed from."""
    a = pos.double()[:, None] * torch.from_numpy(f).cuda()
    c, s = (factor * a.cos())[:, None], (factor * a.sin())[:, None]
    y, size = x.double().clone(), x.double().abs()
    i = torch.arange(dims // 2, device="cuda")
    u, w = (2 * i, 2 * i + 1) if interleaved else (i, i + dims // 2)
    y[..., u] = x.double()[..., u] * c - x.double()[..., w] * s
    y[..., w] = x.double()[..., u] * s + x.double()[..., w] * c
    both = factor * (x.double()[..., u].abs() + x.double()[..., w].abs())
    size[..., u], size[..., w] = both, both
    return y, size


def close(got, ref, pos, f):
    """One rounding to bf16 (2^-8), the angle to 2^-24 of a turn and a half in f32 (1e-6), the reference's own angle
    (positions times a frequency in 64 bits: 2^-52 of it), and a few f32 roundings of what is summed."""
    y, size = ref
    angle = (pos.abs().max().double() * float(np.max(f)) * 2.0 ** -51).item()
    tol = 2.0 ** -8 * y.abs() + (2e-6 + 2 * angle) * size + 1e-38
    err = (got.double() - y).abs()
    assert (err <= tol).all().item(), f"{(err / tol).max().item():.3g} of the tolerance"


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("dims,interleaved", [(128, False), (128, True), (64, False), (64, True), (16, False), (48, True),
                                              (112, False)])
def test_layouts_and_scalings(dims, interleaved, kind):
    rope, f, factor = plan(dims, interleaved, kind)
    hq, hkv, new, lens = 28, 4, [5, 1, 0, 70], [5, 300, 33, 1000]
    cache = Cache(lens, hkv, 16, seed=dims)
    k0, v0 = cache.k.clone(), cache.v.clone()
    total = sum(new)
    q_new, k_new, v_new = (torch.randn((total, h, D), device="cuda").bfloat16() for h in (hq, hkv, hkv))
    pos = torch.randint(0, 200000, (total,), device="cuda", dtype=torch.int32)
    q = torch.empty_like(q_new)
    cc.cc_rope_append(ctx(), cache.desc(hq, new, rope=rope), q_new, k_new, v_new, pos, q, cache.k, cache.v)
    assert ctx().poll() == 0
    close(q, rotated(q_new, pos, f, dims, interleaved, factor), pos, f)
    assert torch.equal(q[..., dims:], q_new[..., dims:])
    rows = torch.cat([cache.rows(s)[n - t:] for s, (n, t) in enumerate(zip(lens, new))])
    close(cache.k[rows], rotated(k_new, pos, f, dims, interleaved, factor), pos, f)
    assert torch.equal(cache.v[rows], v_new)
    k0[rows], v0[rows] = cache.k[rows], cache.v[rows]              # and nothing else
    assert torch.equal(k0.view(torch.int16), cache.k.view(torch.int16))
    assert torch.equal(v0.view(torch.int16), cache.v.view(torch.int16))


def test_far_and_negative_positions():
    rope, f, _ = plan(128, False, "plain")
    cache = Cache([4], 2, 8)
    pos = torch.tensor([2 ** 31 - 1, -5, 10 ** 9 + 7, -2 ** 31], dtype=torch.int32, device="cuda")
    q_new = torch.randn((4, 8, D), device="cuda").bfloat16()
    q = torch.empty_like(q_new)
    cc.cc_rope_append(ctx(), cache.desc(8, [4], rope=rope), q_new, None, None, pos, q, None, None)
    assert ctx().poll() == 0
    close(q, rotated(q_new, pos, f, 128, False, 1.0), pos, f)


@pytest.mark.parametrize("total", [1, 3, 64, 5000])
def test_slots_as_positions_in_place_and_strided(total):
    """q in place in a fused projection, keys and values from the same rows; positions left out."""
    rope, f, _ = plan(128, False, "plain")
    hq, hkv, page = 12, 3, 32
    lens, new = [total + 100, 70], [total, 2]
    cache = Cache(lens, hkv, page, seed=total)
    fused = torch.randn((total + 2, hq + 2 * hkv + 1, D), device="cuda").bfloat16()
    before = fused.clone()
    q, k_new, v_new = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:hq + 2 * hkv]
    st = (fused.stride(0), D)
    desc = cache.desc(hq, new, rope=rope, q_new_strides=st, q_strides=st, kv_new_strides=st)
    cc.cc_rope_append(ctx(), desc, q, k_new, v_new, None, q, cache.k, cache.v)
    assert ctx().poll() == 0
    pos = torch.cat([torch.arange(n - t, n, device="cuda") for n, t in zip(lens, new)]).int()
    close(q, rotated(before[:, :hq], pos, f, 128, False, 1.0), pos, f)
    assert torch.equal(fused[:, hq:], before[:, hq:])
    rows = torch.cat([cache.rows(s)[n - t:] for s, (n, t) in enumerate(zip(lens, new))])
    close(cache.k[rows], rotated(before[:, hq:hq + hkv], pos, f, 128, False, 1.0), pos, f)
    assert torch.equal(cache.v[rows], v_new)


def test_keys_only_and_no_rotation():
    cache = Cache([9], 2, 8, seed=2)
    k_new, v_new = torch.randn((2, 9, 2, D), device="cuda").bfloat16()
    cc.cc_rope_append(ctx(), cache.desc(2, [9]), None, k_new, v_new, None, None, cache.k, cache.v)
    assert ctx().poll() == 0
    assert torch.equal(cache.k[cache.rows(0)], k_new) and torch.equal(cache.v[cache.rows(0)], v_new)


def test_slots_that_do_not_exist_are_flagged_and_skipped():
    cache = Cache([40, 20], 2, 8, seed=3, poison=False)
    k_new, v_new = torch.randn((2, 12, 2, D), device="cuda").bfloat16()
    k0 = cache.k.clone()
    now = torch.tensor([3, 20], dtype=torch.int32, device="cuda")                 # three slots for ten new tokens
    cc.cc_rope_append(ctx(), cache.desc(2, [10, 2], dev_kv_lens=now), None, k_new, v_new, None, None, cache.k, cache.v)
    assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
    rows = torch.cat([cache.rows(0)[:3], cache.rows(1)[18:]])
    k0[rows] = k_new[7:]
    assert torch.equal(k0, cache.k)
    for bad in (-1, cache.pool):
        cache.table[1, 2] = bad
        cc.cc_rope_append(ctx(), cache.desc(2, [0, 2]), None, k_new[:2], v_new[:2], None, None, cache.k, cache.v)
        assert ctx().poll() == cc.CC_ERR_DEVICE_FLAG
        assert torch.equal(k0, cache.k)
