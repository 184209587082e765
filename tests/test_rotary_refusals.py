"""Arguments that the rotary calls refuse, on the CPU: handles, descriptors and the binding's own checks come before
any CUDA call."""
import ctypes

import pytest
import torch

from paper_2608_02504_b200 import build

build.build()
from paper_2608_02504_b200 import api  # noqa: E402


def rotary_create(head_dim=64, n_axes=3, axis=None, freq=None, norm=0, eps=1e-6, null=None):
    cfg = api.tra_rotary_config_t()
    n = max(head_dim, 0) // 2
    axis = [i % max(n_axes, 1) for i in range(n)] if axis is None else axis
    freq = [1.0] * n if freq is None else freq
    cfg.head_dim, cfg.n_axes, cfg.norm, cfg.eps = head_dim, n_axes, norm, eps
    cfg.axis, cfg.inv_freq = (ctypes.c_int * len(axis))(*axis), (ctypes.c_double * len(freq))(*freq)
    if null:
        setattr(cfg, null, None)
    h = ctypes.c_void_p()
    rc = api._lib.tra_rotary_create(ctypes.byref(h), ctypes.byref(cfg))
    assert (rc == api.TRA_OK) == bool(h.value)
    return rc, h


@pytest.mark.parametrize("kw,rc", [
    (dict(), api.TRA_OK), (dict(head_dim=16), api.TRA_OK), (dict(head_dim=256, n_axes=4), api.TRA_OK),
    (dict(head_dim=0), api.TRA_ERR_UNSUPPORTED), (dict(head_dim=-16), api.TRA_ERR_UNSUPPORTED),
    (dict(head_dim=72), api.TRA_ERR_UNSUPPORTED), (dict(head_dim=272), api.TRA_ERR_UNSUPPORTED),
    (dict(n_axes=0), api.TRA_ERR_INVALID_ARG), (dict(n_axes=5), api.TRA_ERR_INVALID_ARG),
    (dict(axis=[3] * 32), api.TRA_ERR_INVALID_ARG), (dict(axis=[-1] * 32), api.TRA_ERR_INVALID_ARG),
    (dict(freq=[float("nan")] * 32), api.TRA_ERR_INVALID_ARG), (dict(freq=[float("inf")] * 32), api.TRA_ERR_INVALID_ARG),
    (dict(norm=3), api.TRA_ERR_INVALID_ARG), (dict(eps=-1.0), api.TRA_ERR_INVALID_ARG),
    (dict(eps=float("nan")), api.TRA_ERR_INVALID_ARG),
    (dict(null="axis"), api.TRA_ERR_INVALID_ARG), (dict(null="inv_freq"), api.TRA_ERR_INVALID_ARG)])
def test_rotary_create(kw, rc):
    got, h = rotary_create(**kw)
    assert got == rc
    if h.value:
        assert api._lib.tra_rotary_destroy(h) == api.TRA_OK


def test_rotary_null_handles():
    assert api._lib.tra_rotary_create(None, None) == api.TRA_ERR_INVALID_ARG
    assert api._lib.tra_rotary_destroy(None) == api.TRA_ERR_INVALID_ARG
    assert api._lib.tra_rotary_backward_workspace_bytes(None) == 0
    assert api._lib.tra_rotary_forward(None, None, None, None, 1, 1, 1, 0, None) == api.TRA_ERR_INVALID_ARG


A = 1 << 20          # an aligned address that is never read


def tensor(**kw):
    t = api.tra_rotary_tensor_t()
    t.src, t.dst, t.heads, t.flags = A, A, 2, api.TRA_ROTARY_ROTATE
    t.src_stride[:], t.dst_stride[:], t.x_stride[:] = (1280, 128, 64), (1280, 128, 64), (1280, 128, 64)
    for name, value in kw.items():
        if name.endswith("stride"):
            getattr(t, name)[:] = value
        else:
            setattr(t, name, value)
    return t


def call(backward, tensors, norm=0, n=None, pos=A, B=1, tokens=10, dtype=0, ws=A, ws_bytes=1 << 30):
    _, h = rotary_create(norm=norm)
    arr = (api.tra_rotary_tensor_t * 3)(*tensors)
    n = len(tensors) if n is None else n
    args = [h, None, pos, ctypes.byref(arr), n, B, tokens, dtype]
    rc = api._lib.tra_rotary_backward(*args, ws, ws_bytes, None) if backward else api._lib.tra_rotary_forward(*args, None)
    api._lib.tra_rotary_destroy(h)
    return rc


BAD = api.TRA_ERR_INVALID_ARG


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,call_kw", [
    (dict(src=None), {}), (dict(dst=None), {}), (dict(heads=0), {}), (dict(src=A + 8), {}), (dict(dst=A + 4), {}),
    (dict(src_stride=(1280, 100, 64)), {}), (dict(dst_stride=(1280, 128, 60)), {}), (dict(flags=4), {}),
    (dict(flags=3), {}), (dict(weight=A), {}), (dict(bias=A), {}), (dict(x=A), {}), (dict(weight_grad=A), {}),
    (dict(bias_grad=A), dict(norm=1)), (dict(bias=A), dict(norm=1)), (dict(weight=A + 2), dict(norm=1)),
    ({}, dict(pos=None)), ({}, dict(pos=A + 2)), ({}, dict(B=0)), ({}, dict(tokens=0)), ({}, dict(dtype=3)),
    ({}, dict(dtype=-1)), ({}, dict(n=0)), ({}, dict(n=4))])
def test_rotary_descriptors(backward, kw, call_kw):
    if backward and call_kw.get("norm") and "x" not in kw:
        kw = dict(kw, x=A)
    assert call(backward, [tensor(**kw)], **call_kw) == BAD


def test_rotary_backward_needs_input_and_workspace():
    assert call(True, [tensor()], norm=1) == BAD                                    # x is missing
    assert call(True, [tensor(x=A, weight_grad=A)], norm=1, ws=None) == BAD
    assert call(True, [tensor(x=A, weight_grad=A)], norm=1, ws_bytes=1000) == api.TRA_ERR_CAPACITY
    assert call(True, [tensor(x=A, x_stride=(1280, 128, 60))], norm=1) == BAD
    assert call(True, [tensor(flags=0, x=A)], norm=1) == BAD                        # only moved: nothing to norm


def test_rotary_binding():
    with pytest.raises(ValueError):
        api.Rotary(64)
    with pytest.raises(ValueError):
        api.Rotary(64, (24, 20, 20), axis=[0] * 32, inv_freq=[1.0] * 32)
    with pytest.raises(ValueError):
        api.Rotary(64, (24, 20, 22))
    with pytest.raises(ValueError):
        api.Rotary(64, (23, 21, 20))
    with pytest.raises(ValueError):
        api.Rotary(64, (64,), norm="batch")
    with pytest.raises(ValueError):
        api.Rotary(64, axis=[0] * 31, inv_freq=[1.0] * 31)
    with pytest.raises(api.TraError):
        api.Rotary(72, (24, 24, 24))
    rot = api.Rotary(64, (24, 20, 20), norm="rms")
    x = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rot.forward(x, pos=torch.zeros(4, 3, dtype=torch.int32))          # not on a GPU
    rot.close()
    rot.close()
