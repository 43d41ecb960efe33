"""The operators around a compacted, paged KV cache whose speed counts: rotating and appending new tokens, attention of
new tokens over the cache, and forking sequences.

A case is a dict of plain values.  ``listed()`` names twelve, ``draw(rng)`` gives more of the same ranges; ``prepare``
makes what a program holds before the call, ``run`` is the call: of this package where ``own`` is true, else the same
operator in elementary torch operations.  ``exact`` gives the results from the definitions in 64 bits.

Inputs.  Keys carry a few outlier channels (one in a hundred, scaled by eight), the queries of neighbouring tokens share
most of their direction, pages of a sequence lie anywhere in the pool (a seeded permutation), and positions of new
tokens are those of the uncompressed prompt, ahead of the slots that a compacted cache gives them.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

HEAD_DIM = 128
#: (query heads, KV heads) of the package's workloads
HEADS = ((8, 2), (32, 8), (28, 4))
PAGES = (8, 16, 16, 32, 64, 128)


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


# ------------------------------------------------------------------------------- cases
def _attend(name, heads, new, kv, page=16, causal=True):
    return {"name": name, "op": "attend", "heads_q": heads[0], "heads_kv": heads[1], "new": _text(new), "kv": _text(kv),
            "page_size": page, "causal": causal}


def _rope(name, heads, new, kv, dims=128, interleaved=False, kind="plain", page=16):
    return {"name": name, "op": "rope", "heads_q": heads[0], "heads_kv": heads[1], "new": _text(new), "kv": _text(kv),
            "page_size": page, "dims": dims, "interleaved": interleaved, "kind": kind}


def _fork(name, heads, kv, children, layers, page=16):
    return {"name": name, "op": "fork", "heads_kv": heads[1], "kv": _text(kv), "children": children, "layers": layers,
            "page_size": page}


def listed():
    rng = np.random.Generator(np.random.PCG64(7007))
    served = np.exp(rng.uniform(math.log(300), math.log(16384), size=64))
    drafts = rng.integers(1, 9, size=16)
    return [
        # one request, one token after a prompt compressed to 2048 tokens: latency
        _attend("token_short", (32, 8), [1], [2305]),
        # one token of every request of a served batch, caches of 300 to 16384 tokens
        _attend("tokens_served", (32, 8), [1] * 64, served),
        # one token over a whole uncompressed repository
        _attend("token_long", (28, 4), [1], [131071], page=64),
        # a few drafted tokens per request, checked together
        _attend("drafts", (28, 4), drafts, rng.integers(1500, 9000, size=16)),
        # the query of a request behind its compressed chunks (Section 4.6): prefill over the cache
        _attend("query_chunk", (32, 8), [517], [8709]),
        # prefill of several requests in one batch, chunks of odd lengths
        _attend("chunks_ragged", (28, 4), [1003, 77, 512, 640, 9], [9007, 4100, 512, 12001, 3001], page=32),
        # a chunk of a long prompt: the largest work
        _attend("prefill_long", (32, 8), [2048], [32768], page=64),
        # the tokens of a served batch, before their attention
        _rope("rotate_tokens", (32, 8), [1] * 64, served),
        # a prefill batch: all heads, positions far out, frequencies scaled by bands
        _rope("rotate_chunks", (32, 8), [4096, 1021, 2500, 515], [30001, 1021, 9000, 2055], kind="bands"),
        # neighbouring pairs, half of the head
        _rope("rotate_partial", (28, 4), [5003], [20011], dims=64, interleaved=True, kind="linear", page=64),
        # four continuations of one prompt, one layer
        _fork("fork_one", (32, 8), [2309], 4, 1),
        # eight continuations of each request of a batch, all layers of the model
        _fork("fork_batch", (32, 8), rng.integers(500, 6000, size=8), 64, 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: lengths spread over their logarithm, odd ones among them."""
    op = rng.choices(("token", "drafts", "chunk", "all", "rope", "fork"), (25, 15, 25, 5, 20, 10))[0]
    heads, page = rng.choice(HEADS), rng.choice(PAGES)
    if op == "fork":
        parents = _log_int(rng, 1, 8)
        kv = [_log_int(rng, 100, 6000) for _ in range(parents)]
        layers = rng.choice((1, 4, 28, 32))
        most = max(1, 32 * 16 * 64 // (layers * page))          # children that copy as much as those of the listed batch
        c = _fork("", heads, kv, min(parents * rng.randint(1, 8), most), layers, page)
    elif op == "rope":
        count = _log_int(rng, 1, 64)
        new = [_log_int(rng, 1, 8000 // count) for _ in range(count)]
        kv = [t + rng.choice((0, _log_int(rng, 1, 8000))) for t in new]
        c = _rope("", heads, new, kv, rng.choice((128, 128, 64, 32, 96)), rng.random() < 0.4,
                  rng.choice(("plain", "linear", "base", "bands")), page)
    else:
        count = _log_int(rng, 1, {"token": 64, "drafts": 32, "chunk": 6, "all": 4}[op])
        most = {"token": 1, "drafts": 16, "chunk": 2048, "all": 600}[op]
        new = [_log_int(rng, 1 if most < 20 else 20, most) for _ in range(count)]
        room = 240000 * 8 // heads[1] if op == "token" else 120000 if op == "drafts" else 32768
        kv = [_log_int(rng, 100, min(131072, room)) for _ in range(count)]
        if op != "all":
            kv = [t + n for t, n in zip(new, kv)]
        # no more keys, and no more products, than the largest listed cases have
        scale = min(1.0, room / sum(kv), 2048 * 31744 / sum(t * n for t, n in zip(new, kv)))
        kv = [max(t, int(n * scale)) for t, n in zip(new, kv)]
        while sum(t * n for t, n in zip(new, kv)) > 2048 * 31744:
            new = [max(1, t // 2) for t in new]
        c = _attend("", heads, new, kv, page, op != "all")
    del c["name"]
    return c


# ------------------------------------------------------------------------------- inputs
def _rng(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _keys(g, rows, heads):
    scale = torch.ones((heads, HEAD_DIM), device="cuda")
    scale[torch.arange(heads, device="cuda"), torch.randint(HEAD_DIM, (heads,), generator=g, device="cuda")] = 8.0
    return (_normal(g, rows, heads, HEAD_DIM) * scale).bfloat16()


def _tables(g, kv, page, spare):
    """Page table of sequences of the given lengths (-1 beyond their pages), ids of the spare pages, pages of the pool."""
    used = [-(-n // page) for n in kv]
    pool = sum(used) + spare
    perm = torch.randperm(pool, generator=g, device="cuda").int()
    table = torch.full((len(kv), max(used)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, u in enumerate(used):
        table[s, :u] = perm[at:at + u]
        at += u
    return table, perm[at:].contiguous(), pool



def _scaling(kind):
    """base, factor, low, high, original length and the factor of the rotated values."""
    if kind == "bands":
        return 500000.0, 8.0, 1.0, 4.0, 8192.0, 1.2079441541679836          # 0.1 ln 8 + 1
    return 1e6 if kind == "base" else 10000.0, 4.0 if kind != "plain" else 1.0, 1.0, 4.0, 8192.0, 1.0


def prepare(case, seed):
    g = _rng(seed)
    st = {"case": case}
    kv, page, hkv = _ints(case["kv"]), case["page_size"], case["heads_kv"]
    if case["op"] == "fork":
        f, layers = case["children"], case["layers"]
        table, free, pool = _tables(g, kv, page, f)
        shape = (layers, pool * page, hkv, HEAD_DIM)
        st["k"] = torch.randint(-32768, 32767, shape, generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
        st["v"] = torch.randint(-32768, 32767, shape, generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
        parents = [i % len(kv) for i in range(f)]
        st.update(table=table, free=free, parents=np.asarray(parents, np.int32),
                  parents_dev=torch.tensor(parents, device="cuda"), lens=torch.tensor(kv, device="cuda"),
                  child=torch.empty((f, table.shape[1]), dtype=torch.int32, device="cuda"))
        if own:
            st["call"] = _own_fork(case, st, pool)
        return st
    new, hq = _ints(case["new"]), case["heads_q"]
    total = sum(new)
    table, _, pool = _tables(g, kv, page, 2)
    st["k"], st["v"] = _keys(g, pool * page, hkv), _normal(g, pool * page, hkv, HEAD_DIM).bfloat16()
    st["table"] = table
    # sequence, place in it, slot of the cache of every new token
    st["seq"] = torch.tensor([s for s, t in enumerate(new) for _ in range(t)], device="cuda")
    st["place"] = torch.tensor([i for t in new for i in range(t)], device="cuda")
    st["slot"] = torch.tensor([n - t + i for t, n in zip(new, kv) for i in range(t)], device="cuda")
    st["lens"] = torch.tensor(kv, device="cuda")
    shared = _normal(g, 1, hq, HEAD_DIM)
    q = (0.6 * shared + 0.8 * _normal(g, total, hq, HEAD_DIM)).bfloat16()
    if case["op"] == "attend":
        st.update(q=q, out=torch.empty_like(q), lse=torch.empty((total, hq), device="cuda"))
    else:
        ahead = torch.tensor([(n * 3) // 2 for n in kv], device="cuda")       # tokens that the compression dropped
        st.update(q=q, k_new=_keys(g, total, hkv), v_new=_normal(g, total, hkv, HEAD_DIM).bfloat16(),
                  positions=(st["slot"] + ahead[st["seq"]]).int(), out=torch.empty_like(q))
    if own:
        st["call"] = (_own_attend if case["op"] == "attend" else _own_rope)(case, st, pool)
    return st


# ------------------------------------------------------------------------------- the package's calls
_CTX = []


def _context():
    from paper_2604_10235_b200 import binding as cc
    if not _CTX:
        _CTX.append(cc.Context(0))
    return cc, _CTX[0]


def _desc(cc, case, st, pool, **more):
    return cc.CacheDesc(case.get("heads_q", case["heads_kv"]), case["heads_kv"], _ints(case["kv"]),
                        page_size=case["page_size"], page_table=st["table"], pool_pages=pool, **more)


def _own_attend(case, st, pool):
    cc, ctx = _context()
    desc = _desc(cc, case, st, pool, new_lens=_ints(case["new"]), causal=case["causal"])
    return cc, ctx, desc, ctx.cache_workspace(desc)


def _own_rope(case, st, pool):
    cc, ctx = _context()
    base, factor, low, high, original, attn = _scaling(case["kind"])
    kind = {"plain": cc.CC_ROPE_PLAIN, "linear": cc.CC_ROPE_LINEAR, "base": cc.CC_ROPE_BASE, "bands": cc.CC_ROPE_BANDS}
    rope = cc.RopePlan(case["dims"], base=base, kind=kind[case["kind"]], factor=factor, low=low, high=high,
                       original=original, attn_factor=attn, interleaved=case["interleaved"])
    return cc, ctx, _desc(cc, case, st, pool, new_lens=_ints(case["new"]), rope=rope)


def _own_fork(case, st, pool):
    cc, ctx = _context()
    st["k_layers"], st["v_layers"] = list(st["k"].unbind(0)), list(st["v"].unbind(0))
    return cc, ctx, _desc(cc, case, st, pool)


# ------------------------------------------------------------------------------- the plain forms
def _slot_rows(st, page, seq, slot):
    """Pool rows of slots of sequences."""
    return st["table"][seq, slot // page].long() * page + slot % page


def _plain_attend(case, st):
    page, hkv = case["page_size"], case["heads_kv"]
    table, lens = st["table"].long().clamp(min=0), st["lens"]
    n_seq, n_max = table.shape[0], table.shape[1] * page
    hq = case["heads_q"]
    t_max = max(_ints(case["new"]))
    rows = (table[:, :, None] * page + torch.arange(page, device="cuda")).reshape(n_seq, n_max)
    k, v = st["k"][rows].float().permute(0, 2, 3, 1), st["v"][rows].float().permute(0, 2, 1, 3)
    q = torch.zeros((n_seq, t_max, hq, HEAD_DIM), device="cuda")
    q[st["seq"], st["place"]] = st["q"].float()
    # the first slot that a token does not see; tokens that a sequence does not have see nothing
    limit = torch.zeros((n_seq, t_max), dtype=torch.int64, device="cuda")
    limit[st["seq"], st["place"]] = st["slot"] + 1 if case["causal"] else lens[st["seq"]]
    q = q.view(n_seq, t_max, hkv, hq // hkv, HEAD_DIM).permute(0, 2, 3, 1, 4).reshape(n_seq, hkv, -1, HEAD_DIM)
    s = torch.matmul(q, k).mul_(1.0 / math.sqrt(HEAD_DIM)).view(n_seq, hkv, hq // hkv, t_max, n_max)
    seen = torch.arange(n_max, device="cuda") < limit[:, None, None, :, None]
    s.masked_fill_(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n_seq, hkv, -1, n_max), v).view(n_seq, hkv, hq // hkv, t_max, HEAD_DIM)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(n_seq, t_max, hq, HEAD_DIM)
    lse = (m + total.log())[..., 0].permute(0, 3, 1, 2).reshape(n_seq, t_max, hq)
    st["out"].copy_(o[st["seq"], st["place"]])
    st["lse"].copy_(lse[st["seq"], st["place"]])
    return {"out": st["out"], "lse": st["lse"]}


def _frequencies(case):
    base, factor, low, high, original, attn = _scaling(case["kind"])
    dims = case["dims"]
    i = torch.arange(dims // 2, dtype=torch.float64, device="cuda")
    if case["kind"] == "base":
        base *= factor ** (dims / (dims - 2))
    f = base ** (-2.0 * i / dims)
    if case["kind"] == "linear":
        f = f / factor
    if case["kind"] == "bands":
        turns = original * f / (2 * math.pi)
        share = ((turns - low) / (high - low)).clamp(0.0, 1.0)
        f = f * share + f / factor * (1 - share)
    return f, attn


def _rotate(x, cos, sin, dims, interleaved):
    a, b = (x[..., 0:dims:2], x[..., 1:dims:2]) if interleaved else (x[..., :dims // 2], x[..., dims // 2:dims])
    c, s = cos[:, None, :], sin[:, None, :]
    u, w = a * c - b * s, a * s + b * c
    turned = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., dims:]), -1)


def _plain_rope(case, st):
    f, attn = _frequencies(case)
    angle = st["positions"].double()[:, None] * f
    cos, sin = (angle.cos() * attn).float(), (angle.sin() * attn).float()
    rows = _slot_rows(st, case["page_size"], st["seq"], st["slot"])
    st["out"].copy_(_rotate(st["q"].float(), cos, sin, case["dims"], case["interleaved"]))
    st["k"][rows] = _rotate(st["k_new"].float(), cos, sin, case["dims"], case["interleaved"]).bfloat16()
    st["v"][rows] = st["v_new"]
    return {"q": st["out"], "k": st["k"], "v": st["v"]}


def _plain_fork(case, st):
    page = case["page_size"]
    parents, lens, table = st["parents_dev"], st["lens"], st["table"]
    n = lens[parents]
    full, rest = n // page, n % page
    at = torch.arange(table.shape[1], device="cuda")
    child = torch.where(at < full[:, None], table[parents], torch.full_like(table[parents], -1))
    st["child"].copy_(torch.where((at == full[:, None]) & (rest[:, None] > 0), st["free"][:, None].expand_as(child), child))
    off = torch.arange(page, device="cuda")
    last = table[parents, full.clamp(max=table.shape[1] - 1)].long()
    to = st["free"].long()[:, None] * page + off
    src = torch.where(off < rest[:, None], last[:, None] * page + off, to)
    for pool in (st["k"], st["v"]):
        bits = pool.view(torch.int16)
        bits[:, to.flatten()] = bits[:, src.flatten()]
    return {"table": st["child"], "k": st["k"].view(torch.int16), "v": st["v"].view(torch.int16)}


def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"attend": _plain_attend, "rope": _plain_rope, "fork": _plain_fork}[op](case, st)
    if op == "attend":
        cc, ctx, desc, ws = st["call"]
        cc.cc_paged_attention(ctx, desc, st["q"], st["k"], st["v"], st["out"], st["lse"], ws=ws)
        return {"out": st["out"], "lse": st["lse"]}
    if op == "rope":
        cc, ctx, desc = st["call"]
        cc.cc_rope_append(ctx, desc, st["q"], st["k_new"], st["v_new"], st["positions"], st["out"], st["k"], st["v"])
        return {"q": st["out"], "k": st["k"], "v": st["v"]}
    cc, ctx, desc = st["call"]
    cc.cc_fork_pages(ctx, desc, st["k_layers"], st["v_layers"], st["parents"], st["child"], st["free"])
    return {"table": st["child"], "k": st["k"].view(torch.int16), "v": st["v"].view(torch.int16)}


# ------------------------------------------------------------------------------- work and exact results
def work(case):
    kv, page, hkv = _ints(case["kv"]), case["page_size"], case["heads_kv"]
    row = HEAD_DIM * 2
    if case["op"] == "fork":
        lens = [kv[i % len(kv)] for i in range(case["children"])]
        width = max(-(-n // page) for n in kv)
        return {"bytes": 4 * row * hkv * case["layers"] * sum(n % page for n in lens) + 8 * width * len(lens), "flops": 0}
    new, hq = _ints(case["new"]), case["heads_q"]
    pages = sum(-(-n // page) for n in kv)
    if case["op"] == "rope":
        per = 2 * row * (hq + 2 * hkv) + 8
        return {"bytes": sum(new) * per, "flops": 6 * sum(new) * (hq + hkv) * case["dims"] // 2}
    pairs = sum(t * n - (t * (t - 1) // 2 if case["causal"] else 0) for t, n in zip(new, kv))
    return {"bytes": 2 * row * hkv * sum(kv) + sum(new) * hq * (2 * row + 4) + 4 * pages,
            "flops": 4 * HEAD_DIM * hq * pairs}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    kv, page, hkv = _ints(case["kv"]), case["page_size"], case["heads_kv"]
    if case["op"] == "fork":
        return None                                             # bit copies: no computed numbers
    new, hq = _ints(case["new"]), case["heads_q"]
    pages = st["table"].cpu().numpy()
    rows = [torch.from_numpy((pages[s, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page)).cuda()
            for s, n in enumerate(kv)]
    if case["op"] == "attend":
        out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        at = 0
        for s, (t, n) in enumerate(zip(new, kv)):
            for h in range(hkv):
                k, v = st["k"][rows[s], h].double(), st["v"][rows[s], h].double()
                for i0 in range(0, t, 512):
                    i1 = min(t, i0 + 512)
                    heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                    x = torch.einsum("tgd,nd->tgn", st["q"][at + i0:at + i1, heads].double(), k) / math.sqrt(HEAD_DIM)
                    if case["causal"]:
                        own_slot = torch.arange(n - t + i0, n - t + i1, device="cuda")
                        x[(torch.arange(n, device="cuda")[None, :] > own_slot[:, None])[:, None, :].expand_as(x)] = -math.inf
                    lse[at + i0:at + i1, heads] = torch.logsumexp(x, -1)
                    out[at + i0:at + i1, heads] = torch.einsum("tgn,nd->tgd", torch.softmax(x, -1), v)
            at += t
        return {"out": out, "lse": lse}
    # rotation of the complex numbers that the pairs are
    base, factor, low, high, original, attn = _scaling(case["kind"])
    dims = case["dims"]
    if case["kind"] == "base":
        base = base * factor ** (dims / (dims - 2))
    f = np.array([math.pow(base, -2.0 * i / dims) for i in range(dims // 2)])
    if case["kind"] == "linear":
        f = f / factor
    elif case["kind"] == "bands":
        wave = 2 * math.pi / f
        share = np.minimum(1.0, np.maximum(0.0, (original / wave - low) / (high - low)))
        f = (1 - share) * f / factor + share * f
    turn = torch.polar(torch.full((1, 1), attn, dtype=torch.float64, device="cuda"),
                       st["positions"].double()[:, None] * torch.from_numpy(f).cuda())[:, None, :]

    def turned(x):
        y = x.double().clone()
        lo, hi = (slice(0, dims, 2), slice(1, dims, 2)) if case["interleaved"] else (slice(0, dims // 2), slice(dims // 2, dims))
        z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * turn
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    k, v = st["k"].double(), st["v"].double()
    at = 0
    for s, (t, n) in enumerate(zip(new, kv)):
        k[rows[s][n - t:]] = turned(st["k_new"])[at:at + t]
        v[rows[s][n - t:]] = st["v_new"][at:at + t].double()
        at += t
    return {"q": turned(st["q"]), "k": k, "v": v}
