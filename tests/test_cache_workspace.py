"""The workspace of cc_paged_attention is memory of the context's device.  No GPU: tensors on the host stand for those of a
device (-1), and the calls are refused before they would use one."""
import ctypes as C
import math

import pytest
import torch

from test_cache_step import Call
from paper_2604_10235_b200 import binding as cc


def attend(device, ws, scale=math.nan):
    call = Call()
    call.d.scale = scale
    return call.lib.calls["cc_paged_attention"](C.addressof(call.ctx), C.addressof(call.d), device, None, None, None, None, None, ws, 0)


def test_workspace_of_another_device_is_refused():
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    assert attend(-1, ws) == cc.CC_ERR_INVALID_ARG               # (the scale)
    with pytest.raises(ValueError):
        attend(0, ws)


def test_workspace_is_contiguous_or_none():
    for ws in (torch.zeros(1 << 16, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.uint8).expand(1 << 16)):
        with pytest.raises(ValueError):
            attend(-1, ws)
    assert attend(-1, None) == cc.CC_ERR_INVALID_ARG             # the library's own refusal
