"""Arguments that the calls around the 4-bit cache refuse, on the CPU: the checks come before any CUDA call, so a handle made up here (of a
device that does not exist: nothing is ever launched through it) is enough."""
import ctypes

import pytest

from paper_2608_02504_b200 import build

build.build()
from paper_2608_02504_b200 import api  # noqa: E402
from tests.test_packed_refusals import A, BAD, UNSUPPORTED, Handle, arguments, passed  # noqa: E402

STRIDE = ctypes.c_int64 * 2


def handle(window=0, sinks=0, heads=4, kv_heads=2, head_dim=64, dtype=0):
    return Handle(api.tra_packed_config_t(heads, kv_heads, head_dim, dtype, 1, window, sinks), -7, 148, None)


def cache(**kw):
    c = api.tra_cache4_t(A, A, A, A, 120)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def rows(name, c, k=A, v=A, ks=(128, 64), vs=(128, 64), slots=A, n=10, h=None):
    h = handle() if h is None else h
    return getattr(api._lib, name)(ctypes.byref(h), ctypes.byref(c), k, v, STRIDE(*ks), STRIDE(*vs), slots, n, None)


@pytest.mark.parametrize("name", ["tra_cache4_write", "tra_cache4_read"])
def test_rows(name):
    call = getattr(api._lib, name)
    assert passed(rows(name, cache()))
    assert rows(name, cache(), n=0) == api.TRA_OK and rows(name, cache(tokens=0, k=None, v=None, k_step=None, v_step=None), n=0) == api.TRA_OK
    # a dimension of one entry has no stride
    assert passed(rows(name, cache(), n=1, ks=(3, 64)))
    for c in (cache(k=None), cache(v=None), cache(k_step=None), cache(v_step=None), cache(k=A + 8), cache(v_step=A + 2), cache(tokens=-2), cache(tokens=121)):
        assert rows(name, c) == BAD
    for kw in (dict(k=None), dict(v=None), dict(k=A + 8), dict(v=A + 4), dict(ks=(128, 60)), dict(vs=(0, 64)), dict(ks=(128, -64)), dict(vs=(1 << 38, 64)),
               dict(slots=None), dict(slots=A + 2), dict(n=-1)):
        assert rows(name, cache(), **kw) == BAD, kw
    assert rows(name, cache(tokens=(1 << 30) + 2)) == UNSUPPORTED and rows(name, cache(), n=(1 << 30) + 1) == UNSUPPORTED
    assert call(None, ctypes.byref(cache()), A, A, STRIDE(128, 64), STRIDE(128, 64), A, 1, None) == BAD
    assert call(ctypes.byref(handle()), None, A, A, STRIDE(128, 64), STRIDE(128, 64), A, 1, None) == BAD
    assert call(ctypes.byref(handle()), ctypes.byref(cache()), A, A, None, STRIDE(128, 64), A, 1, None) == BAD


def attend(a, c, h=None, ws=A, ws_bytes=1 << 40):
    h = handle() if h is None else h
    return api._lib.tra_packed_attn_cache4(ctypes.byref(h), ctypes.byref(a), ctypes.byref(c), ws, ws_bytes, None)


def test_attention():
    assert passed(attend(arguments(k=None, v=None), cache()))
    assert passed(attend(arguments(k=A + 1, k_stride=(1, 1)), cache()))              # not looked at
    assert passed(attend(arguments(lse=None), cache())) and passed(attend(arguments(), cache(), handle(10, 3)))
    assert attend(arguments(), cache(tokens=121)) == BAD and attend(arguments(), cache(k=None)) == BAD
    assert attend(arguments(o_rest=A), cache()) == BAD
    for kw in (dict(q=None), dict(o=None), dict(q=A + 8), dict(cu_q=None), dict(k_begin=None), dict(k_end=A + 2), dict(lse=A + 1), dict(n_seq=0),
               dict(total_q=-1), dict(max_q=101), dict(max_k=121), dict(max_k=-1), dict(sm_scale=0.0), dict(q_stride=(256, 60)), dict(o_stride=(1 << 38, 64))):
        assert attend(arguments(**kw), cache()) == BAD, kw
    assert attend(arguments(total_q=(1 << 30) + 1), cache()) == UNSUPPORTED
    lib = api._lib
    assert lib.tra_packed_attn_cache4(None, ctypes.byref(arguments()), ctypes.byref(cache()), A, 1 << 40, None) == BAD
    assert lib.tra_packed_attn_cache4(ctypes.byref(handle()), None, ctypes.byref(cache()), A, 1 << 40, None) == BAD
    assert lib.tra_packed_attn_cache4(ctypes.byref(handle()), ctypes.byref(arguments()), None, A, 1 << 40, None) == BAD


@pytest.mark.parametrize("dtype", [api.TRA_BF16, api.TRA_FP16])
def test_workspace_follows_the_sizes(dtype):
    size = lambda n_seq, total_q, max_q, max_k, h=handle(heads=40, kv_heads=8, head_dim=128, dtype=dtype): \
        api._lib.tra_packed_attn_cache4_workspace_bytes(ctypes.byref(h), n_seq, total_q, max_q, max_k)
    assert size(1, 1, 1, 1000) == 0                                                   # one cluster
    assert size(64, 64, 1, 32768) % (4 * 64 * 40 * 130) == 0 < size(64, 64, 1, 32768)  # parts
    many = size(4, 2048, 512, 16384)
    assert 2 * 4 * 16384 * 8 * 128 * 2 <= many < (1 << 30)                            # keys and values read back
    assert size(400, 400 * 512, 512, 16384) < (3 << 30)                              # in passes
    assert size(0, 1, 1, 1) == 0 and size(1, 1, 2, 1) == 0 and size(1, 1, 1, -1) == 0 and size(1, 0, 0, 5) == 0
    assert api._lib.tra_packed_attn_cache4_workspace_bytes(None, 1, 1, 1, 1) == 0
    # a window bounds what is read back
    h = handle(1000, 16, heads=40, kv_heads=8, head_dim=128, dtype=dtype)
    assert size(4, 2048, 512, 1 << 20, h) < 1 << 28
