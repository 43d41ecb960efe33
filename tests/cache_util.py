"""Paged caches with poisoned surroundings and 64-bit references for the calls that work on them."""
from __future__ import annotations

import math

import torch

from paper_2604_10235_b200 import binding as cc

D = 128


class Cache:
    """Sequences of the given lengths in a pool whose pages lie anywhere; rows that no sequence has hold NaN."""

    def __init__(self, lens, hkv, page, seed=0, spare=3, poison=True, extra_cols=0, kv_strides=None, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        used = [-(-n // page) for n in lens]
        self.lens, self.hkv, self.page = list(lens), hkv, page
        self.pool = sum(used) + spare
        perm = torch.randperm(self.pool, generator=g).int()
        table = torch.full((len(lens), max(used + [1]) + extra_cols), -77, dtype=torch.int32)
        at = 0
        for s, u in enumerate(used):
            table[s, :u] = perm[at:at + u]
            at += u
        self.free = perm[at:].cuda()
        self.table = table.cuda()
        rows = self.pool * page
        tok, head = kv_strides or (hkv * D, D)
        self.strides = (tok, head)
        size = (rows - 1) * tok + (hkv - 1) * head + D
        self.k_mem = torch.full((size,), math.nan if poison else 0.0, dtype=torch.bfloat16, device="cuda")
        self.v_mem = self.k_mem.clone()
        self.k = self.k_mem.as_strided((rows, hkv, D), (tok, head, 1))
        self.v = self.v_mem.as_strided((rows, hkv, D), (tok, head, 1))
        gd = torch.Generator(device="cuda").manual_seed(seed + 1)
        for s, n in enumerate(lens):
            if n:
                r = self.rows(s)
                self.k[r] = (torch.randn((n, hkv, D), generator=gd, device="cuda") * scale).bfloat16()
                self.v[r] = torch.randn((n, hkv, D), generator=gd, device="cuda").bfloat16()

    def rows(self, s, n=None):
        """Pool rows of the first n slots of sequence s."""
        j = torch.arange(self.lens[s] if n is None else n, device="cuda")
        return self.table[s].long()[j // self.page] * self.page + j % self.page

    def desc(self, hq, new=None, **more):
        return cc.CacheDesc(hq, self.hkv, self.lens, new, page_size=self.page, page_table=self.table, pool_pages=self.pool,
                            kv_strides=self.strides, **more)


def attend_reference(cache, q, new, causal=True, scale=None, lens=None, rows=None):
    """out, lse, sum_j softmax |v_j| and the largest scale * sum |q| |k| of every row, in 64 bits."""
    scale = 1 / math.sqrt(D) if scale is None else scale
    hq = q.shape[1]
    g = hq // cache.hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(out)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    reach = torch.zeros_like(lse)
    at = 0
    for s, T in enumerate(new):
        n = cache.lens[s] if lens is None else lens[s]
        if n and T:
            r = cache.rows(s, n)
            k = cache.k[r].double().repeat_interleave(g, 1)
            v = cache.v[r].double().repeat_interleave(g, 1)
            for t0 in range(0, T, 256):
                t = torch.arange(t0, min(T, t0 + 256), device="cuda")
                qq = q[at + t].double()
                x = torch.einsum("thd,nhd->thn", qq, k) * scale
                seen = torch.ones((len(t), n), dtype=torch.bool, device="cuda")
                if causal:
                    seen = torch.arange(n, device="cuda")[None, :] <= (n - T + t)[:, None]
                x = x.masked_fill(~seen[:, None, :], -math.inf)
                p = torch.softmax(x, -1)
                some = seen.any(-1)
                p = torch.where(some[:, None, None], p, torch.zeros_like(p))
                out[at + t] = torch.einsum("thn,nhd->thd", p, v)
                size[at + t] = torch.einsum("thn,nhd->thd", p, v.abs())
                lse[at + t] = torch.where(some[:, None], torch.logsumexp(x, -1), lse[at + t])
                reach[at + t] = (abs(scale) * torch.einsum("thd,nhd->thn", qq.abs(), k.abs())).amax(-1)
        at += T
    return out, lse, size, reach


def assert_attention(out, lse, ref):
    """Tolerances.  A probability is rounded to bf16 once (2^-8 of its size), the output once (2^-8).  A logit is a sum of
    128 products in f32: 128 roundings of 2^-23 (the tensor core may truncate) of what they sum, and one of the scaling; its error
    is the relative error of the probability, beside 1e-4 for the exponential (8e-5 where a polynomial computes it)."""
    o, l, size, reach = ref
    eta = reach * 2.0 ** -16 + 1.0e-4
    tol = 2.0 ** -8 * o.abs() + (2.0 ** -8 * 1.01 + 2 * eta)[..., None] * size + 1e-30
    err = (out.double() - o).abs()
    assert torch.isfinite(out.float()).all()
    worst = (err / tol).max().item()
    assert worst <= 1, f"{worst:.3g} of the tolerance at {torch.nonzero(err > tol)[:3].tolist()}"
    if lse is not None:
        none = l == -math.inf
        assert torch.equal(lse == -math.inf, none)
        e = (lse.double() - l).abs()[~none]
        bound = (eta + l.abs() * 2.0 ** -22)[~none]
        assert (e <= bound).all().item(), f"lse off by {(e / bound).max().item():.3g} of the tolerance"


def attend(ctx, cache, hq, new, q=None, causal=True, scale=0.0, seed=5, desc=None, ws=None, with_lse=True):
    total = sum(new)
    if q is None:
        g = torch.Generator(device="cuda").manual_seed(seed)
        q = torch.randn((total, hq, D), generator=g, device="cuda").bfloat16()
    out = torch.full((total, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((total, hq), 7.0, device="cuda") if with_lse else None
    desc = desc or cache.desc(hq, new, causal=causal, scale=scale)
    cc.cc_paged_attention(ctx, desc, q, cache.k, cache.v, out, lse, ws=ws)
    return q, out, lse
