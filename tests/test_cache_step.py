"""Calls on a paged cache without a GPU: rotation frequencies, refusals, the descriptor's layout."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest

from paper_2604_10235_b200 import binding as cc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def words(dims=128, kind=cc.CC_ROPE_PLAIN, **kw):
    return cc.RopePlan(dims, kind=kind, **kw).freqs[:dims // 2]


@pytest.mark.parametrize("dims", [16, 64, 96, 128])
def test_frequencies(dims):
    """A frequency in 64 bits has 2^-53, the powers and products of this formula a few of them."""
    i = np.arange(dims // 2)
    plain = 10000.0 ** (-2 * i / dims)
    stretched = (10000.0 * 4.0 ** (dims / (dims - 2))) ** (-2 * i / dims)
    turns = 8192.0 * plain / (2 * math.pi)
    g = np.clip((turns - 1) / 3, 0, 1)
    for got, f in ((words(dims), plain), (words(dims, cc.CC_ROPE_LINEAR, factor=4.0), plain / 4),
                   (words(dims, cc.CC_ROPE_BASE, factor=4.0), stretched),
                   (words(dims, cc.CC_ROPE_BANDS, factor=4.0), (1 - g) * plain / 4 + g * plain),
                   (words(dims, cc.CC_ROPE_GIVEN, inv_freq=plain), plain)):
        np.testing.assert_allclose(got.astype(np.float64) / 2.0 ** 64, f / (2 * math.pi), rtol=64 * 2.0 ** -53)


def test_frequencies_are_places_on_the_circle():
    two_pi = 2 * math.pi
    got = words(16, cc.CC_ROPE_GIVEN, inv_freq=[0.0, two_pi / 4, two_pi * 5.5, 1.0, 0.5, 100.0, 3.0, 1e6])
    assert got[0] == 0
    # (2 pi in 64 bits is off by 2.4e-16 of 6.28)
    assert abs(float(got[1]) / 2.0 ** 64 - 0.25) < 1e-15 and abs(float(got[2]) / 2.0 ** 64 - 0.5) < 1e-14
    for w, f in zip(got[3:], (1.0, 0.5, 100.0, 3.0, 1e6)):
        assert abs(float(w) / 2.0 ** 64 - math.fmod(f / two_pi, 1.0)) < 1e-9


@pytest.mark.parametrize("kw,status", [
    (dict(dims=8), cc.CC_ERR_UNSUPPORTED), (dict(dims=136), cc.CC_ERR_UNSUPPORTED), (dict(dims=24), cc.CC_ERR_UNSUPPORTED),
    (dict(kind=9), cc.CC_ERR_INVALID_ARG), (dict(kind=-1), cc.CC_ERR_INVALID_ARG), (dict(base=1.0), cc.CC_ERR_INVALID_ARG),
    (dict(base=math.nan), cc.CC_ERR_INVALID_ARG), (dict(base=math.inf), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_LINEAR, factor=0.5), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_BASE, factor=math.nan), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_BANDS, low=4.0, high=4.0), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_BANDS, low=0.0), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_BANDS, original=0.0), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_GIVEN), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_GIVEN, inv_freq=[1.0] * 63 + [math.nan]), cc.CC_ERR_INVALID_ARG),
    (dict(kind=cc.CC_ROPE_GIVEN, inv_freq=[-1.0] * 64), cc.CC_ERR_INVALID_ARG)])
def test_frequencies_refused(kw, status):
    with pytest.raises(cc.CodecompError) as e:
        cc.RopePlan(**kw)
    assert e.value.status == status


class Call:
    """Argument checks with a context that was never created and addresses that nothing reads."""

    def __init__(self, lens=(40, 20), new=None):
        self.lib = cc.load_library()
        self.ctx = C.create_string_buffer(4096)
        self.lens = np.array(lens, np.int32)
        self.new = None if new is None else np.array(new, np.int32)
        d = self.d = cc.cc_cache_desc()
        d.n_heads_q, d.n_heads_kv, d.head_dim, d.dtype, d.num_seqs = 8, 2, 128, cc.CC_BF16, len(lens)
        d.page_size, d.pool_pages, d.page_table_stride, d.page_table = 16, 100, 3, 4096
        d.kv_lens = self.lens.ctypes.data_as(C.POINTER(C.c_int32))
        if new is not None:
            d.new_lens = self.new.ctypes.data_as(C.POINTER(C.c_int32))
        d.causal = 1
        self.freqs = np.zeros(64, np.uint64)
        d.rope_dims, d.rope_freqs = 128, self.freqs.ctypes.data_as(C.POINTER(C.c_uint64))

    def attend(self, q=4096, k=4096, v=4096, out=4096, ws=4096, ws_bytes=1 << 40, ctx=True):
        return self.lib.cc_paged_attention(self.ctx if ctx else None, C.byref(self.d), q, k, v, out, None, ws, ws_bytes, None)

    def rope(self, q_new=4096, k_new=4096, v_new=4096, q=8192, k=4096, v=4096):
        return self.lib.cc_rope_append(self.ctx, C.byref(self.d), q_new, k_new, v_new, None, q, k, v, None)

    def fork(self, layers=1, parents=(0, 1), table=1 << 20, stride=3, free=4096, pool=4096):
        k = (C.c_void_p * max(layers, 1))(*[pool] * max(layers, 1))
        p = np.array(parents, np.int32)
        return self.lib.cc_fork_pages(self.ctx, C.byref(self.d), layers, k, k, p.ctypes.data, len(p), table, stride, free, None)

    @property
    def text(self):
        return self.lib.cc_last_error(self.ctx).decode()


@pytest.mark.parametrize("field,value,status", [
    ("n_heads_q", 0, cc.CC_ERR_INVALID_ARG), ("n_heads_q", 7, cc.CC_ERR_INVALID_ARG), ("n_heads_kv", -2, cc.CC_ERR_INVALID_ARG),
    ("n_heads_q", 2 * 129, cc.CC_ERR_UNSUPPORTED), ("head_dim", 64, cc.CC_ERR_UNSUPPORTED), ("dtype", cc.CC_F32, cc.CC_ERR_UNSUPPORTED),
    ("num_seqs", 0, cc.CC_ERR_UNSUPPORTED), ("num_seqs", 65, cc.CC_ERR_UNSUPPORTED), ("page_size", 0, cc.CC_ERR_UNSUPPORTED),
    ("page_size", 24, cc.CC_ERR_UNSUPPORTED), ("page_size", 256, cc.CC_ERR_UNSUPPORTED), ("pool_pages", 0, cc.CC_ERR_INVALID_ARG),
    ("pool_pages", 2 ** 31 - 1, cc.CC_ERR_UNSUPPORTED), ("page_table", None, cc.CC_ERR_INVALID_ARG),
    ("page_table_stride", 2, cc.CC_ERR_INVALID_ARG), ("kv_lens", None, cc.CC_ERR_INVALID_ARG),
    ("q_stride_tok", 1025, cc.CC_ERR_UNSUPPORTED), ("kv_stride_head", 64, cc.CC_ERR_INVALID_ARG),
    ("kv_new_stride_tok", -8, cc.CC_ERR_INVALID_ARG), ("out_stride_tok", 2 ** 40, cc.CC_ERR_UNSUPPORTED)])
def test_descriptors_refused(field, value, status):
    c = Call()
    setattr(c.d, field, value)
    assert c.attend() == status and c.rope() == status and c.fork() == status
    assert c.lib.cc_attention_workspace_bytes(c.ctx, C.byref(c.d)) == 0
    assert c.text


def test_lengths_refused():
    for lens, new in (((40, -1), None), ((40, 20), (1, -1)), ((40, 49), None), ((2 ** 31 - 1, 20), None)):
        assert Call(lens, new).attend() == cc.CC_ERR_INVALID_ARG
    assert Call((40, 20), (2 ** 30, 2 ** 30)).attend() == cc.CC_ERR_UNSUPPORTED
    # appending needs a slot for every new token; attention does not, nor do queries alone
    assert Call((40, 20), (1, 21)).rope() == cc.CC_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["q", "k", "v", "out"])
def test_attention_pointers_refused(name):
    assert Call().attend(**{name: None}) == cc.CC_ERR_INVALID_ARG
    assert Call().attend(**{name: 4104}) == cc.CC_ERR_INVALID_ARG


def test_attention_workspace_and_scale_refused():
    assert Call().attend(ws=None) == cc.CC_ERR_WORKSPACE
    assert Call().attend(ws=4096 + 128) == cc.CC_ERR_WORKSPACE
    c = Call()
    c.ctx = C.create_string_buffer(bytes(4) + (148).to_bytes(4, "little") + bytes(4088), 4096)     # its SM count
    need = c.lib.cc_attention_workspace_bytes(c.ctx, C.byref(c.d))
    assert need >= 256
    assert c.attend(ws_bytes=255) == cc.CC_ERR_WORKSPACE
    for scale in (math.nan, math.inf):
        c = Call()
        c.d.scale = scale
        assert c.attend() == cc.CC_ERR_INVALID_ARG
    assert Call().attend(ctx=False) == cc.CC_ERR_INVALID_ARG


def test_rotation_refused():
    for kw in (dict(q=None), dict(v_new=None), dict(k=None), dict(v=None), dict(q_new=4100), dict(k=4104)):
        assert Call().rope(**kw) == cc.CC_ERR_INVALID_ARG, kw
    for dims, status in ((8, cc.CC_ERR_UNSUPPORTED), (40, cc.CC_ERR_UNSUPPORTED), (144, cc.CC_ERR_UNSUPPORTED)):
        c = Call()
        c.d.rope_dims = dims
        assert c.rope() == status
    c = Call()
    c.d.rope_freqs = None
    assert c.rope() == cc.CC_ERR_INVALID_ARG
    c = Call()
    c.d.rope_scale = math.inf
    assert c.rope() == cc.CC_ERR_INVALID_ARG
    c = Call()
    c.d.q_stride_tok = 2048
    assert c.rope(q=4096) == cc.CC_ERR_INVALID_ARG               # in place with other strides
    assert Call().rope(q_new=None, k_new=None) == cc.CC_OK       # nothing to do
    assert Call((40, 20), (0, 0)).rope() == cc.CC_OK and Call((40, 20), (0, 0)).attend() == cc.CC_OK


def test_forks_refused():
    for kw in (dict(parents=(0, 2)), dict(parents=(-1,)), dict(stride=2), dict(stride=0), dict(table=None), dict(free=None),
               dict(layers=-1), dict(pool=None), dict(pool=4104)):
        assert Call().fork(**kw) == cc.CC_ERR_INVALID_ARG, kw
    assert Call().fork(parents=[0] * 257) == cc.CC_ERR_UNSUPPORTED
    # the rows of the children on those of the parents, which begin at address 4096 and have 12 bytes each
    assert Call().fork(table=4096) == cc.CC_ERR_INVALID_ARG
    assert Call().fork(table=4096 + 12, parents=(1, 1)) == cc.CC_ERR_INVALID_ARG
    assert Call().fork(parents=()) == cc.CC_OK and Call().fork(layers=0) == cc.CC_OK


def test_binding_struct_matches_header_field_order():
    text = open(os.path.join(ROOT, "include", "codecomp.h")).read()
    for name, struct in (("cc_cache_desc", cc.cc_cache_desc), ("cc_rope_params", cc.cc_rope_params)):
        body = text[text.index(f"typedef struct {name} {{"):text.index(f"}} {name};")].split("{", 1)[1]
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = []
        for decl in body.split(";"):
            words_ = [w for w in decl.replace("*", " ").split() if w not in ("const", "int32_t", "int64_t", "uint64_t", "float", "double")]
            fields += [f.strip() for f in " ".join(words_).split(",") if f.strip()]
        assert fields == [f[0] for f in struct._fields_]


def test_too_much_work_for_one_call_is_refused():
    c = Call((2 ** 30, 2 ** 30), (2 ** 29, 2 ** 29))
    c.d.n_heads_q, c.d.n_heads_kv, c.d.page_table_stride = 64, 1, 2 ** 26
    c.ctx = C.create_string_buffer(bytes(4) + (148).to_bytes(4, "little") + bytes(4088), 4096)
    assert c.lib.cc_attention_workspace_bytes(c.ctx, C.byref(c.d)) == 0
    assert c.attend() == cc.CC_ERR_UNSUPPORTED and "tiles" in c.text


def test_typed_arguments_are_checked():
    """bfloat16 tensors of the context's device; what is on the host is on device -1, which stands for any other here."""
    import torch
    call = Call()
    lib, at = call.lib, C.addressof(call.ctx)
    bf, f32, i32 = torch.zeros(4, dtype=torch.bfloat16), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    attend = lib.calls["cc_paged_attention"]
    desc = C.addressof(call.d)
    for args in ((f32, bf, bf, bf, f32), (bf, i32, bf, bf, f32), (bf, bf, bf, bf, bf)):
        with pytest.raises(ValueError):
            attend(at, desc, -1, *args, None, 0)
    with pytest.raises(ValueError):
        attend(at, desc, 0, bf, bf, bf, bf, f32, None, 0)
    with pytest.raises(AttributeError):
        attend(at, desc, -1, object(), bf, bf, bf, f32, None, 0)
    rope = lib.calls["cc_rope_append"]
    assert rope(at, desc, -1, None, None, None, None, None, None, None, 0) == cc.CC_OK
    for positions in (f32, torch.zeros((4, 2), dtype=torch.int32)[:, 0]):
        with pytest.raises(ValueError):
            rope(at, desc, -1, None, None, None, positions, None, None, None, 0)
    fork = lib.calls["cc_fork_pages"]
    parents = np.array([0, 5], np.int32)
    assert fork(at, desc, -1, 0, [], [], parents, 2, i32, 3, i32, 0) == cc.CC_OK
    with pytest.raises(ValueError):
        fork(at, desc, -1, 1, [f32], [bf], parents, 2, i32, 3, i32, 0)
    with pytest.raises(ValueError):
        fork(at, desc, -1, 1, [bf], [bf], parents.astype(np.int64), 2, i32, 3, i32, 0)
    with pytest.raises(AttributeError):
        fork(at, desc, -1, 1, [None], [bf], parents, 2, i32, 3, i32, 0)
    with pytest.raises((TypeError, BufferError)):
        fork(at, desc, -1, 1, [bf], [bf], [0, 5], 2, i32, 3, i32, 0)


def test_one_workspace_for_all_lengths():
    """What the header promises: no more than 266496 bytes per SM, whatever the batch."""
    rng = np.random.default_rng(3)
    for _ in range(2000):
        seqs = int(rng.integers(1, 65))
        lens = np.exp(rng.uniform(0, math.log(200000), seqs)).astype(np.int32)
        c = Call(lens, np.minimum(lens, np.exp(rng.uniform(0, math.log(4000), seqs)).astype(np.int32)))
        c.d.n_heads_kv = int(rng.choice([1, 2, 4, 8, 32]))
        c.d.n_heads_q = c.d.n_heads_kv * int(rng.choice([1, 4, 7, 16]))
        c.d.page_table_stride = 200000 // 16
        sms = int(rng.choice([1, 2, 20, 148]))
        c.ctx = C.create_string_buffer(bytes(4) + sms.to_bytes(4, "little") + bytes(4088), 4096)
        assert 256 <= c.lib.cc_attention_workspace_bytes(c.ctx, C.byref(c.d)) <= 266496 * sms
