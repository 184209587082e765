"""Arguments that the packed-attention calls refuse, on the CPU.  The checks come before any CUDA call, so a handle made up here
(of a device that does not exist: nothing is ever launched through it) is enough: what passes them ends at the device
check."""
import ctypes

import pytest

from paper_2608_02504_b200 import build

build.build()
from paper_2608_02504_b200 import api  # noqa: E402

A = 1 << 20          # an aligned address that is never read
BAD, UNSUPPORTED = api.TRA_ERR_INVALID_ARG, api.TRA_ERR_UNSUPPORTED


class Handle(ctypes.Structure):
    _fields_ = [("cfg", api.tra_packed_config_t), ("device", ctypes.c_int), ("sm_count", ctypes.c_int), ("status", ctypes.c_void_p)]


def handle(heads=4, kv_heads=2, head_dim=64, dtype=0, causal=1):
    return Handle(api.tra_packed_config_t(heads, kv_heads, head_dim, dtype, causal), -7, 148, None)


def arguments(**kw):
    a = api.tra_packed_args_t()
    a.q, a.k, a.v, a.o, a.lse = A, A, A, A, A
    for n, heads in (("q", 4), ("k", 2), ("v", 2), ("o", 4)):
        getattr(a, n + "_stride")[:] = (heads * 64, 64)
    a.cu_q, a.k_begin, a.k_end = A, A, A + 4
    a.n_seq, a.total_q, a.total_k, a.max_q, a.max_k, a.sm_scale = 2, 100, 120, 60, 70, 0.125
    for name, value in kw.items():
        if name.endswith("stride"):
            getattr(a, name)[:] = value
        else:
            setattr(a, name, value)
    return a


def grads(**kw):
    g = api.tra_packed_grads_t()
    g.d_o, g.dq, g.dk, g.dv = A, A, A, A
    for n, heads in (("do", 4), ("dq", 4), ("dk", 2), ("dv", 2)):
        getattr(g, n + "_stride")[:] = (heads * 64, 64)
    for name, value in kw.items():
        if name.endswith("stride"):
            getattr(g, name)[:] = value
        else:
            setattr(g, name, value)
    return g


def forward(a, h=None, ws=A, ws_bytes=1 << 40):
    h = handle() if h is None else h
    return api._lib.tra_packed_attn(ctypes.byref(h), ctypes.byref(a), ws, ws_bytes, None)


def backward(a, g, ws=A, ws_bytes=1 << 40):
    return api._lib.tra_packed_attn_backward(ctypes.byref(handle()), ctypes.byref(a), ctypes.byref(g), ws, ws_bytes, None)


def passed(rc):
    """The argument checks were passed: no CUDA device here, or not the handle's."""
    import torch
    return rc == (BAD if torch.cuda.is_available() else api.TRA_ERR_CUDA)


@pytest.mark.parametrize("kw,rc", [
    (dict(heads=0), BAD), (dict(kv_heads=0), BAD), (dict(heads=4, kv_heads=3), BAD), (dict(dtype=api.TRA_FP32), BAD),
    (dict(dtype=9), BAD), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(heads=258, kv_heads=2), UNSUPPORTED),
    (dict(heads=8192, kv_heads=8192), UNSUPPORTED)])
def test_create(kw, rc):
    cfg = handle(**kw).cfg
    h = ctypes.c_void_p(5)
    assert api._lib.tra_packed_create(ctypes.byref(h), ctypes.byref(cfg)) == rc and not h.value


def test_null_handles():
    assert api._lib.tra_packed_create(None, None) == BAD
    assert api._lib.tra_packed_destroy(None) == BAD
    assert api._lib.tra_packed_status(None, None) == BAD
    assert api._lib.tra_packed_attn(None, ctypes.byref(arguments()), None, 0, None) == BAD
    assert api._lib.tra_packed_attn_backward(None, ctypes.byref(arguments()), ctypes.byref(grads()), None, 0, None) == BAD
    assert api._lib.tra_packed_attn_workspace_bytes(None, 1, 1, 1, 1) == 0
    assert api._lib.tra_packed_attn_backward_workspace_bytes(None, 1) == 0
    h = handle()
    assert api._lib.tra_packed_attn(ctypes.byref(h), None, None, 0, None) == BAD
    assert api._lib.tra_packed_attn_backward(ctypes.byref(h), ctypes.byref(arguments()), None, A, 1 << 40, None) in (BAD, api.TRA_ERR_CUDA)


def test_good_arguments_reach_the_device_check():
    assert passed(forward(arguments()))
    assert passed(forward(arguments(lse=None)))
    assert passed(forward(arguments(o_rest=A))) and forward(arguments(o_rest=A, lse=None)) == BAD
    assert passed(backward(arguments(), grads()))
    assert passed(forward(arguments(total_k=0, max_k=0, k=None, v=None)))
    # a dimension of one entry has no stride
    assert passed(forward(arguments(total_q=1, max_q=1, q_stride=(3, 64))))


@pytest.mark.parametrize("kw,rc", [
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(o=None), BAD), (dict(q=A + 8), BAD),
    (dict(o=A + 2), BAD), (dict(cu_q=None), BAD), (dict(k_begin=None), BAD), (dict(k_end=None), BAD), (dict(cu_q=A + 2), BAD),
    (dict(lse=A + 1), BAD), (dict(o_rest=A + 8), BAD), (dict(n_seq=0), BAD), (dict(total_q=-1), BAD), (dict(total_k=-1), BAD), (dict(max_q=-1), BAD),
    (dict(max_q=101), BAD), (dict(max_k=121), BAD), (dict(sm_scale=0.0), BAD), (dict(sm_scale=-1.0), BAD),
    (dict(sm_scale=float("nan")), BAD), (dict(sm_scale=float("inf")), BAD), (dict(q_stride=(256, 60)), BAD),
    (dict(k_stride=(0, 64)), BAD), (dict(v_stride=(128, -64)), BAD), (dict(o_stride=(1 << 38, 64)), BAD),
    (dict(total_q=(1 << 30) + 1), UNSUPPORTED), (dict(total_k=(1 << 30) + 1), UNSUPPORTED)])
def test_arguments(kw, rc):
    assert forward(arguments(**kw)) == rc
    assert backward(arguments(**kw), grads()) == rc


@pytest.mark.parametrize("n_seq,total_q,max_q,max_k,parts", [(1, 1, 1, 100000, True), (1, 1, 1, 2000, False), (64, 64, 1, 4000, False),
                                                            (1, 97, 97, 65500, True), (8, 20000, 8000, 8000, False)])
def test_workspace_follows_the_sizes(n_seq, total_q, max_q, max_k, parts):
    h = handle(heads=40, kv_heads=8, head_dim=128)
    n = api._lib.tra_packed_attn_workspace_bytes(ctypes.byref(h), n_seq, total_q, max_q, max_k)
    assert (n > 0) == parts and n % (4 * total_q * 40 * 130) == 0
    assert api._lib.tra_packed_attn_workspace_bytes(ctypes.byref(h), n_seq, total_q, max_q, -1) == 0
    assert api._lib.tra_packed_attn_workspace_bytes(ctypes.byref(h), 0, total_q, max_q, max_k) == 0
    assert api._lib.tra_packed_attn_backward_workspace_bytes(ctypes.byref(h), total_q) == 4 * 40 * total_q
