"""Tensors of the calls on a paged cache hold what the descriptor describes.  No GPU: tensors on the host stand for those
of a device (-1), and every call that passes the checks is refused by the library afterwards, before it would use one."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from test_cache_step import Call
from paper_2604_10235_b200 import binding as cc

HQ, HKV, ROWS, PAGE, POOL = 8, 2, 7, 16, 100


class Sub(torch.Tensor):
    """What is not exactly a torch.Tensor is described by its methods."""


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def tensors():
    return {"q_new": bf(ROWS, HQ, 128), "k_new": bf(ROWS, HKV, 128), "v_new": bf(ROWS, HKV, 128),
            "positions": torch.zeros(ROWS, dtype=torch.int32), "q": bf(ROWS, HQ, 128), "k": bf(POOL * PAGE, HKV, 128),
            "v": bf(POOL * PAGE, HKV, 128), "out": bf(ROWS, HQ, 128), "lse": torch.zeros(ROWS, HQ)}


def invoke(name, t, strides=(), parents=(99,)):
    call = Call((40, 20), (5, 2))
    for field, value in strides:
        setattr(call.d, field, value)
    at, desc, calls = C.addressof(call.ctx), C.addressof(call.d), call.lib.calls
    if name == "rope":
        call.d.rope_scale = math.inf
        return calls["cc_rope_append"](at, desc, -1, t["q_new"], t["k_new"], t["v_new"], t["positions"], t["q"], t["k"], t["v"], 0)
    if name == "attend":
        call.d.scale = math.nan
        return calls["cc_paged_attention"](at, desc, -1, t["q"], t["k"], t["v"], t["out"], t["lse"], None, 0)
    p = np.array(parents, np.int32)
    table = torch.zeros((len(p), 4), dtype=torch.int32)
    return calls["cc_fork_pages"](at, desc, -1, 2, [t["k"]] * 2, [t["v"]] * 2, p, len(p), table, 4, table, 0)


USES = [("rope", n) for n in ("q_new", "k_new", "v_new", "positions", "q", "k", "v")] + \
       [("attend", n) for n in ("q", "k", "v", "out", "lse")] + [("fork", n) for n in ("k", "v")]


@pytest.mark.parametrize("sub", [False, True])
@pytest.mark.parametrize("name", ["rope", "attend", "fork"])
def test_tensors_that_fit_reach_the_library(name, sub):
    t = tensors()
    more = {"q_new": bf(ROWS + 3, HQ, 128), "q": bf(1, ROWS, HQ * 128), "k": bf(POOL, PAGE, HKV, 128),
            "v": bf(POOL * PAGE * HKV * 128 + 5), "lse": torch.zeros(ROWS * HQ), "positions": torch.zeros((1, ROWS), dtype=torch.int32)}
    for x in (t, {**t, **more}, {**t, "positions": None, "lse": None}):
        if sub:
            x = {k: None if v is None else v.as_subclass(Sub) for k, v in x.items()}
        assert invoke(name, x) == cc.CC_ERR_INVALID_ARG


@pytest.mark.parametrize("sub", [False, True])
@pytest.mark.parametrize("name,arg", USES)
def test_tensors_that_are_too_small_are_refused(name, arg, sub):
    t = tensors()
    for short in (t[arg][:-1], t[arg].flatten()[1:].clone(), t[arg][:0]):
        x = short.as_subclass(Sub) if sub else short
        with pytest.raises(ValueError, match="fewer than"):
            invoke(name, {**t, arg: x})


@pytest.mark.parametrize("sub", [False, True])
@pytest.mark.parametrize("name,arg", USES)
def test_tensors_with_strides_of_their_own_need_them_in_the_descriptor(name, arg, sub):
    t = tensors()
    x = t[arg]
    wide = torch.zeros(x.shape[:-1] + (2 * x.shape[-1],), dtype=x.dtype)[..., :x.shape[-1]]
    swapped = torch.zeros((x.shape[1], x.shape[0]) + x.shape[2:], dtype=x.dtype).transpose(0, 1) if x.dim() > 1 else x.expand(1, -1)
    if x.dim() == 1:
        wide = torch.zeros(2 * len(x), dtype=x.dtype)[::2]
    for y in (wide, swapped, x[:1].expand(x.shape)):
        if y.is_contiguous():
            continue
        y = y.as_subclass(Sub) if sub else y
        with pytest.raises(ValueError, match="contiguous"):
            invoke(name, {**t, arg: y})


@pytest.mark.parametrize("sub", [False, True])
def test_strides_of_the_descriptor(sub):
    """A fused projection, a pool with its heads outermost, a padded output: what the last row needs and no more."""
    t = tensors()
    fused = bf(ROWS, HQ + 2 * HKV, 128)
    st = fused.stride(0)
    pool = bf(HKV, POOL * PAGE, 136)
    padded = bf(ROWS, HQ, 256)
    own = {"q_new": fused[:, :HQ], "q": fused[:, :HQ], "k_new": fused[:, HQ:HQ + HKV], "v_new": fused[:, HQ + HKV:],
           "k": pool[..., :128], "v": pool[..., :128].transpose(0, 1), "out": padded[..., :128]}
    strides = [("q_new_stride_tok", st), ("kv_new_stride_tok", st), ("q_stride_tok", st), ("q_stride_head", 128),
               ("kv_stride_tok", 136), ("kv_stride_head", POOL * PAGE * 136), ("out_stride_tok", HQ * 256), ("out_stride_head", 256)]
    view = (lambda x: x.as_subclass(Sub)) if sub else (lambda x: x)
    own = {k: view(v) for k, v in own.items()}
    for name in ("rope", "attend", "fork"):
        assert invoke(name, {**t, **own}, strides) == cc.CC_ERR_INVALID_ARG
    for name, arg in (("rope", "q_new"), ("rope", "k_new"), ("rope", "q"), ("rope", "k"), ("attend", "out"), ("attend", "q"),
                      ("attend", "v"), ("fork", "k")):
        short = own[arg][..., :-1]
        with pytest.raises(ValueError, match="fewer than"):
            invoke(name, {**t, **own, arg: short}, strides)
    # strides that reach beyond a dense tensor
    with pytest.raises(ValueError, match="fewer than"):
        invoke("attend", t, [("q_stride_tok", 2048)])
    with pytest.raises(ValueError, match="fewer than"):
        invoke("rope", t, [("kv_stride_head", 2 ** 32)])


def test_nothing_is_asked_of_tensors_that_are_not_used():
    call = Call((40, 20), (0, 0))
    x = bf(1)
    at, desc, calls = C.addressof(call.ctx), C.addressof(call.d), call.lib.calls
    assert calls["cc_rope_append"](at, desc, -1, x, x, x, None, x, x, x, 0) == cc.CC_OK
    assert calls["cc_paged_attention"](at, desc, -1, x, x, x, x, None, None, 0) == cc.CC_OK
    # descriptors that the library refuses say so themselves
    for field, value in (("num_seqs", 0), ("num_seqs", 65), ("n_heads_q", -8), ("q_stride_tok", -8)):
        call = Call((40, 20), (5, 2))
        setattr(call.d, field, value)
        at, desc = C.addressof(call.ctx), C.addressof(call.d)
        x = tensors()
        assert calls["cc_paged_attention"](at, desc, -1, x["q"], x["k"], x["v"], x["out"], None, None, 0) in (
            cc.CC_ERR_INVALID_ARG, cc.CC_ERR_UNSUPPORTED)


def test_tensors_that_require_gradients_are_tensors():
    t = tensors()
    t["q"].requires_grad_(True)
    t["k"] = torch.nn.Parameter(t["k"])
    assert invoke("attend", t) == cc.CC_ERR_INVALID_ARG


def test_rows_of_a_descriptor():
    class Table:
        dtype, is_cuda, device, shape = torch.int32, True, "cuda:0", (3, 200)
        is_contiguous = staticmethod(lambda: True)
        dim = staticmethod(lambda: 2)
        data_ptr = staticmethod(lambda: 4096)
        get_device = staticmethod(lambda: 0)
    more = dict(page_size=16, page_table=Table, pool_pages=9)
    assert cc.CacheDesc(32, 8, [2065, 1233], [17, 1], **more).n_new == 18
    d = cc.CacheDesc(32, 8, [5, 0, 7], **more)
    assert d.n_new == 3 and d.lens == [5, 0, 7]
