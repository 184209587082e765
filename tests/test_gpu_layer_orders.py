"""Rotary calls whose tensors differ in token order (raster-order plans, positions from the grid), and a plan's rotary call followed
by packed attention and all the way back."""
import math

import pytest
import torch

from tests.packed_reference import i32
from tests.test_gpu_rotary import (AXES, check_backward, check_forward, cpu64, grid_pos, make, params, plan_order, reference)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.mark.parametrize("flags", ["TRA_ORDER_RASTER", "TRA_ORDER_RASTER_QO"])
@pytest.mark.parametrize("grid", [(2, 16, 32, 0), (3, 16, 16, 48), (7, 48, 80, 16)])
@pytest.mark.parametrize("dtype,norm,heads,d", [(torch.bfloat16, "rms", 3, 64), (torch.float16, None, 4, 128),
                                                (torch.float32, "layer", 5, 64)])
def test_grid_positions_of_raster_plans(api, flags, grid, dtype, norm, heads, d):
    """RASTER: nothing is reordered.  RASTER_QO: K and V are, Q is not, though both have the grid's positions."""
    T, H, W, n_text = grid
    plan = api.Plan(T, H, W, d, 128, 8, 16, flags=getattr(api, flags), n_text=n_text)
    rot = api.Rotary(d, AXES[d], norm=norm)
    qkv = make(api, (1, plan.N, heads, heads, d), dtype, 35)
    w = params(d, dtype, norm, 36)
    pos, turned = grid_pos(T, H, W, n_text), plan.N_video
    raster, tiles = torch.arange(plan.N), plan_order(plan)
    orders = (raster, raster, raster) if flags == "TRA_ORDER_RASTER" else (raster, tiles, tiles)
    outs = rot.forward(*qkv, plan=plan, **w)
    # (the helpers take all tensors in one order: each is turned back to the raster order first)
    back = [torch.empty_like(o) for o in orders]
    for b, o in zip(back, orders):
        b[o] = raster
    in_raster = [y[:, :, b.cuda()] for y, b in zip(outs, back)]
    check_forward(in_raster, qkv, pos, norm, w, False, dtype, turned, raster)
    dys = tuple(torch.randn(o.shape, device="cuda").to(dtype) for o in outs)
    weights = {n: t for n, t in w.items() if n.endswith("weight")}
    x = dict(q=qkv[0], k=qkv[1]) if norm else {}
    dxs, grads = rot.backward(*dys, plan=plan, **x, **weights)
    check_backward(dxs, grads, [dy[:, :, b.cuda()] for dy, b in zip(dys, back)], qkv, pos, norm, w, False, dtype, turned, raster)
    # Q alone, and V alone beside it, give the same bits
    alone = rot.forward(qkv[0], plan=plan, **{n: t for n, t in w.items() if n[0] == "q"})
    assert torch.equal(alone[0], outs[0]) and alone[1] is None and alone[2] is None
    pair = rot.forward(qkv[0], None, qkv[2], plan=plan, **{n: t for n, t in w.items() if n[0] == "q"})
    assert torch.equal(pair[0], outs[0]) and torch.equal(pair[2], outs[2])
    plan.close()


@pytest.mark.parametrize("flags", [None, "TRA_ORDER_RASTER_QO"])
@pytest.mark.parametrize("T,H,W,n_text,heads,d", [(2, 16, 16, 0, 2, 64), (3, 8, 16, 21, 3, 128)])
def test_plan_rotary_then_packed_attention_and_back(api, flags, T, H, W, n_text, heads, d):
    """Fused projection -> norm, grid positions, token order -> attention of the clip as one packed sequence (whose keys may be in
    any order) -> gradients of the projection and the norm's weights, against differentiation of the definition in fp64."""
    if flags and n_text:
        n_text = 32                                      # whole rows of sixteen
    dt = torch.float16
    plan = api.Plan(T, H, W, d, 128, 8, 16, flags=getattr(api, flags) if flags else 0, n_text=n_text)
    rot = api.Rotary(d, AXES[d], norm="rms")
    attn = api.PackedAttn(heads, heads, d, dtype=dt, causal=False)
    N = plan.N
    qkv = make(api, (1, N, heads, heads, d), dt, 45)
    w = params(d, dt, "rms", 46)
    do = torch.randn(1, heads, N, d, device="cuda").to(dt)                        # of O, in Q's order
    Q, K, V = rot.forward(*qkv, plan=plan, **w)
    packed = lambda t: t[0].transpose(0, 1)                                      # [tokens, heads, d], a view
    cu, kw = i32([0, N]), dict(max_q=N, max_k=N)
    o, lse = attn.forward(packed(Q), packed(K), packed(V), cu, want_lse=True, **kw)
    dq, dk, dv = attn.backward(packed(do), packed(Q), packed(K), packed(V), o, lse, cu, **kw)
    lift = lambda t: t.transpose(0, 1)[None]
    dxs, grads = rot.backward(lift(dq), lift(dk), lift(dv), q=qkv[0], k=qkv[1], plan=plan, **w)
    attn.check_status()

    pos, tiles, raster = grid_pos(T, H, W, n_text), plan_order(plan), torch.arange(N)
    q_order = raster if flags else tiles
    leaves = [cpu64(x).requires_grad_() for x in qkv] + [cpu64(w[n]).requires_grad_() for n in ("q_weight", "k_weight")]
    q, k = (reference(leaves[i], pos, "rms", leaves[3 + i], None, False, 1e-6, plan.N_video)[0] for i in range(2))
    s = torch.einsum("bnhd,bmhd->bhnm", q, k) / math.sqrt(d)
    out = torch.einsum("bhnm,bmhd->bhnd", torch.softmax(s, -1), leaves[2])[:, :, q_order]
    want = torch.autograd.grad(out, leaves, cpu64(do))
    # every stage rounds to fp16 (2^-11): q, k (scores of up to about 5 move by their sum), P, dS, dq, dk, dx: below 32
    # roundings of the size of the result, in the relative norm
    got = [lift(o), *dxs, grads["q_weight"], grads["k_weight"]]
    for name, a, b in zip(("o", "dq", "dk", "dv", "q_weight", "k_weight"), got, [out.detach(), *want]):
        rel = float((cpu64(a) - b).norm() / b.norm())
        assert rel <= 32 * 2.0 ** -11, (name, rel)
    plan.close()
