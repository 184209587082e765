"""Windows that ``tra_packed_create`` refuses, on the CPU (the checks come before any CUDA call)."""
import ctypes

import pytest

from paper_2608_02504_b200 import build

build.build()
from paper_2608_02504_b200 import api  # noqa: E402

BAD, UNSUPPORTED = api.TRA_ERR_INVALID_ARG, api.TRA_ERR_UNSUPPORTED


@pytest.mark.parametrize("causal,window,sinks,rc", [
    (1, -1, 0, BAD), (1, 0, 1, BAD), (1, 5, -1, BAD), (0, 5, 0, UNSUPPORTED), (0, 0, 2, BAD), (1, (1 << 30) + 1, 0, UNSUPPORTED),
    (1, 1, (1 << 30) + 1, UNSUPPORTED)])
def test_create(causal, window, sinks, rc):
    cfg = api.tra_packed_config_t(4, 2, 64, api.TRA_BF16, causal, window, sinks)
    h = ctypes.c_void_p(5)
    assert api._lib.tra_packed_create(ctypes.byref(h), ctypes.byref(cfg)) == rc and not h.value


def test_workspace_follows_the_window():
    """A window shortens what a call walks: one token over a long cache then needs no second launch."""
    class Handle(ctypes.Structure):
        _fields_ = [("cfg", api.tra_packed_config_t), ("device", ctypes.c_int), ("sm_count", ctypes.c_int), ("status", ctypes.c_void_p)]
    size = lambda window: api._lib.tra_packed_attn_workspace_bytes(
        ctypes.byref(Handle(api.tra_packed_config_t(40, 8, 128, 0, 1, window, 0), -7, 148, None)), 1, 1, 1, 100000)
    assert size(0) > 0 and size(100000) == size(0) and size(500) == 0


@pytest.mark.parametrize("sizes", [dict(window=2 ** 32 + 5), dict(window=5, sinks=2 ** 32), dict(window=-2 ** 32)])
def test_numbers_that_a_c_int_would_wrap(sizes):
    with pytest.raises(ValueError):
        api.PackedAttn(4, 2, 64, **sizes)
