"""Head norm, rotary positions with several axes and token order (``tra_rotary_forward`` / ``_backward``) against a
plain fp64 implementation.

Tolerances, per element, from the arithmetic.  One rounding to the output type: eps / 2 of the value.  fp32 steps, in
units of 2^-24: the half-turn count is rounded once (pi / 2 units of angle) and sincospif is off by 2 ulp, 6 together;
sums over d <= 256 channels are 16 terms per thread and at most four shuffles, 20 units of the sum of magnitudes, half
of that through the reciprocal root, whose own error is 2 ulp; products and sums of the rotation and the weight 6.
64 units of (|z1| + |z2| + |w|) cover the forward pass (|w| stands for the mean, whose 20 units of mean |x| r <= 1 are
scaled by the weight).  The gradient repeats the norm (n off by 40 units) and takes two more means of up to
G = max over the row of |u1| + |u2| times |w|: 128 units of r G (2 + |n|).  A weight's gradient adds R terms u n, each
off by 64 units of |u| (|n| + 1), through chains of at most 300 additions."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -24
AXES = {16: (8, 4, 4), 32: (12, 10, 10), 48: (16, 16, 16), 64: (24, 20, 20), 96: (32, 32, 32), 128: (44, 42, 42),
        256: (88, 84, 84)}


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def frequencies(d, theta=10000.0):
    axis, freq = [], []
    for a, c in enumerate(AXES[d]):
        axis += [a] * (c // 2)
        freq += [theta ** (-2.0 * k / c) for k in range(c // 2)]
    return torch.tensor(axis), torch.tensor(freq, dtype=torch.float64)


def reference(x, pos, norm, weight, bias, halves, eps, turned):
    """x fp64 [B, N, h, d] on the CPU, pos int [N, 3]; tokens >= turned keep their angle at zero.
    Returns y, and what the tolerances need: z, n, r."""
    d = x.shape[-1]
    n, r = x, torch.ones_like(x[..., :1])
    if norm == "layer":
        n = x - x.mean(-1, keepdim=True)
    if norm:
        r = 1.0 / torch.sqrt((n * n).mean(-1, keepdim=True) + eps)
        n = n * r
    z = n
    if weight is not None:
        z = z * weight
    if bias is not None:
        z = z + bias
    axis, freq = frequencies(d)
    ang = pos.double()[:, axis] * freq
    ang[turned:] = 0
    c, s = torch.cos(ang)[None, :, None], torch.sin(ang)[None, :, None]
    return rotate(z, c, s, halves), z, n, r, (c, s)


def rotate(z, c, s, halves):
    d = z.shape[-1]
    a, b = (z[..., : d // 2], z[..., d // 2:]) if halves else (z[..., 0::2], z[..., 1::2])
    ya, yb = a * c - b * s, a * s + b * c
    return torch.cat([ya, yb], -1) if halves else torch.stack([ya, yb], -1).flatten(-2)


def pair_size(z, halves):
    """|z1| + |z2| of every channel's pair."""
    a = z.abs()
    d = a.shape[-1]
    if halves:
        s = a[..., : d // 2] + a[..., d // 2:]
        return torch.cat([s, s], -1)
    return (a[..., 0::2] + a[..., 1::2]).repeat_interleave(2, -1)


def check(got, want, tol, what):
    got = got.detach().double().cpu()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst " \
                          f"{float(((got - want).abs() / tol.clamp_min(1e-300))[bad].max())} times the tolerance"


def half_eps(dtype):
    return torch.finfo(dtype).eps / 2


def make(api, shape, dtype, seed):
    """q, k, v as slices of one fused projection [B, N, hq + 2 hk, d]"""
    B, N, hq, hk, d = shape
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(B, N, hq + 2 * hk, d, generator=g, device="cuda").mul_(1.5).add_(0.2).to(dtype)
    return x[:, :, :hq], x[:, :, hq:hq + hk], x[:, :, hq + hk:]


def params(d, dtype, norm, seed):
    if norm is None:
        return {}
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = {}
    for n in "qk":
        out[n + "_weight"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype)
        if norm == "layer":
            out[n + "_bias"] = (0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    return out


def cpu64(t):
    return None if t is None else t.detach().double().cpu()


def check_forward(outs, qkv, pos, norm, w, halves, dtype, turned, order=None, eps=1e-6):
    for out, x, name in zip(outs, qkv, "qkv"):
        x = cpu64(x)
        if name == "v":
            want, tol = x, torch.zeros_like(x)
        else:
            weight, bias = cpu64(w.get(name + "_weight")), cpu64(w.get(name + "_bias"))
            want, z, *_ = reference(x, pos, norm, weight, bias, halves, eps, turned)
            top = 1.0 if weight is None else float(weight.abs().max())
            tol = half_eps(dtype) * want.abs() * (1 + 2 * half_eps(dtype)) + \
                64 * UNIT * (pair_size(z, halves) + (top if norm else 0.0)) + torch.finfo(dtype).tiny
        if order is not None:
            want, tol = (t[:, order].transpose(1, 2) for t in (want, tol))
        check(out, want, tol, name)


def check_backward(dxs, grads, dys, qkv, pos, norm, w, halves, dtype, turned, order=None, eps=1e-6):
    for dx, dy, x, name in zip(dxs, dys, qkv, "qkv"):
        x, dy = cpu64(x), cpu64(dy)
        if order is not None:
            back = torch.empty_like(order)
            back[order] = torch.arange(order.numel())
            dy = dy.transpose(1, 2)[:, back]
        if name == "v":
            check(dx, dy, torch.zeros_like(dy), "dv")
            continue
        weight = cpu64(w.get(name + "_weight"))
        _, z, n, r, (c, s) = reference(x, pos, norm, weight, None, halves, eps, turned)
        u = rotate(dy, c, -s, halves)
        if norm is None:
            check(dx, u, half_eps(dtype) * u.abs() * (1 + 2 * half_eps(dtype)) + 64 * UNIT * pair_size(dy, halves)
                  + torch.finfo(dtype).tiny, "d" + name)
            continue
        wt = torch.ones(x.shape[-1], dtype=torch.float64) if weight is None else weight
        gr = u * wt
        want = gr - n * (gr * n).mean(-1, keepdim=True)
        if norm == "layer":
            want = want - gr.mean(-1, keepdim=True)
        want = want * r
        G = (pair_size(dy, halves) * wt.abs()).amax(-1, keepdim=True)
        tol = half_eps(dtype) * want.abs() * (1 + 2 * half_eps(dtype)) + 128 * UNIT * r * G * (2 + n.abs()) \
            + torch.finfo(dtype).tiny
        check(dx, want, tol, "d" + name)
        if not grads:
            continue
        size = (pair_size(dy, halves) * (n.abs() + 1)).sum((0, 1, 2))
        check(grads[name + "_weight"], (u * n).sum((0, 1, 2)), 364 * UNIT * size, name + "_weight")
        if norm == "layer":
            check(grads[name + "_bias"], u.sum((0, 1, 2)), 364 * UNIT * size, name + "_bias")


def grid_pos(T, H, W, n_text=0):
    n = torch.arange(T * H * W)
    p = torch.stack([n // (H * W), (n // W) % H, n % W], 1)
    return torch.cat([p, torch.zeros(n_text, 3, dtype=p.dtype)])


def plan_order(plan):
    _, _, coord = plan.tables()
    c = torch.from_numpy(coord).long()
    order = (c[:, 0] * plan.H + c[:, 1]) * plan.W + c[:, 2]
    return torch.cat([order, torch.arange(plan.N_video, plan.N)])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("norm", [None, "rms", "layer"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 16), (2, 37, 3, 1, 32), (1, 130, 5, 5, 64), (1, 19, 2, 2, 96),
                                   (3, 65, 8, 2, 128), (1, 33, 12, 4, 256), (1, 700, 40, 8, 128), (1, 5, 7, 7, 48)])
def test_positions(api, dtype, norm, halves, shape):
    B, N, hq, hk, d = shape
    rot = api.Rotary(d, AXES[d], halves=halves, norm=norm)
    qkv = make(api, shape, dtype, 5)
    w = params(d, dtype, norm, 6)
    g = torch.Generator().manual_seed(7)
    pos = torch.randint(-50000, 2000000, (N, 3), generator=g)
    pos[0] = torch.tensor([2 ** 31 - 1, -2 ** 31, 0])
    dev_pos = pos.to(torch.int32).cuda()
    outs = rot.forward(*qkv, pos=dev_pos, **w)
    check_forward(outs, qkv, pos, norm, w, halves, dtype, N)
    dys = tuple(torch.randn(o.shape, device="cuda").to(dtype) for o in outs)
    weights = {k: t for k, t in w.items() if k.endswith("weight")}
    x = dict(q=qkv[0], k=qkv[1]) if norm else {}
    dxs, grads = rot.backward(*dys, **x, pos=dev_pos, **weights)
    check_backward(dxs, grads, dys, qkv, pos, norm, w, halves, dtype, N)
    assert set(grads) == (set() if norm is None else {"q_weight", "k_weight"} if norm == "rms"
                          else {"q_weight", "k_weight", "q_bias", "k_bias"})
    again, grads2 = rot.backward(*dys, **x, pos=dev_pos, **weights)
    assert all(torch.equal(a, b) for a, b in zip(dxs, again)) and all(torch.equal(grads[n], grads2[n]) for n in grads)


@pytest.mark.parametrize("grid", [(4, 8, 8, 0, 4, 4, 64), (3, 7, 9, 5, 8, 16, 128), (2, 16, 32, 77, 8, 16, 128),
                                  (1, 1, 1, 0, 8, 16, 128)])
@pytest.mark.parametrize("dtype,norm,heads", [(torch.bfloat16, "rms", 2), (torch.float16, None, 5),
                                              (torch.float32, "layer", 12)])
def test_plan(api, grid, dtype, norm, heads):
    T, H, W, n_text, th, tw, block = grid
    for d in (64, 128):
        plan = api.Plan(T, H, W, d, block, th, tw, n_text=n_text)
        rot = api.Rotary(d, AXES[d], norm=norm)
        N = plan.N
        qkv = make(api, (2, N, heads, heads, d), dtype, 15)
        w = params(d, dtype, norm, 16)
        order, pos, turned = plan_order(plan), grid_pos(T, H, W, n_text), plan.N_video
        outs = rot.forward(*qkv, plan=plan, **w)
        assert all(o.is_contiguous() and tuple(o.shape) == (2, heads, N, d) for o in outs)
        check_forward(outs, qkv, pos, norm, w, False, dtype, turned, order)
        if dtype == torch.bfloat16:          # V is what the gather makes of it, bit for bit
            assert torch.equal(outs[2], plan.tile_major_gather(qkv[2].transpose(1, 2).contiguous()))
        dys = tuple(torch.randn(o.shape, device="cuda").to(dtype) for o in outs)
        fused = torch.full((2, N, 3 * heads, d), 7.0, dtype=dtype, device="cuda")
        views = tuple(fused[:, :, i * heads:(i + 1) * heads] for i in range(3))
        weights = {k: t for k, t in w.items() if k.endswith("weight")}
        dxs, grads = rot.backward(*dys, q=qkv[0] if norm else None, k=qkv[1] if norm else None, plan=plan, out=views, **weights)
        check_backward(views, grads, dys, qkv, pos, norm, w, False, dtype, turned, order)
        plan.close()


def test_plan_flags_and_explicit_positions(api):
    """Raster-order plans take Q (and O), or everything, in raster order; explicit positions override the grid's."""
    T, H, W, d, heads = 2, 16, 32, 64, 3
    pos = grid_pos(T, H, W) * 3 + 1
    for flags, raster in ((0, ""), (api.TRA_ORDER_RASTER, "qkv"), (api.TRA_ORDER_RASTER_QO, "q")):
        plan = api.Plan(T, H, W, d, 64, 8, 16, flags=flags)
        rot = api.Rotary(d, AXES[d], norm="rms")
        qkv = make(api, (1, plan.N, heads, heads, d), torch.bfloat16, 25)
        outs = rot.forward(*qkv, plan=plan, pos=pos.to(torch.int32).cuda())
        for i, name in enumerate("qkv"):
            x = cpu64(qkv[i])
            want = x if name == "v" else reference(x, pos, "rms", None, None, False, 1e-6, plan.N)[0]
            want = want.transpose(1, 2) if name in raster else want[:, plan_order(plan)].transpose(1, 2)
            assert (cpu64(outs[i]) - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 1e-4
        plan.close()


def test_gradient_against_differences(api):
    """<dx, e> and <dw, e> against central differences of the fp64 definition along a direction e."""
    d, N, h = 64, 23, 3
    for norm in ("rms", "layer"):
        rot = api.Rotary(d, AXES[d], norm=norm)
        qkv = make(api, (1, N, h, h, d), torch.float32, 31)
        w = params(d, torch.float32, norm, 32)
        pos = torch.randint(0, 1000, (N, 3), generator=torch.Generator().manual_seed(33))
        dy = torch.randn(1, N, h, d, device="cuda")
        (dx, _, _), grads = rot.backward(dy, q=qkv[0], pos=pos.to(torch.int32).cuda(), q_weight=w["q_weight"])
        x, wt, dy64 = cpu64(qkv[0]), cpu64(w["q_weight"]), cpu64(dy)
        b = cpu64(w.get("q_bias"))
        f = lambda x_, w_, b_: float((reference(x_, pos, norm, w_, b_, False, 1e-6, N)[0] * dy64).sum())
        step = 1e-5
        gen = torch.Generator().manual_seed(34)
        for what, got, at in (("x", dx, 0), ("w", grads["q_weight"], 1)) + \
                ((("b", grads["q_bias"], 2),) if norm == "layer" else ()):
            base = [x, wt, b]
            e = torch.randn(base[at].shape, generator=gen, dtype=torch.float64)
            up, down = list(base), list(base)
            up[at], down[at] = base[at] + step * e, base[at] - step * e
            diff = (f(*up) - f(*down)) / (2 * step)
            inner = float((cpu64(got) * e).sum())
            # the differences are off by step^2 and by 2^-52 / step of sums of size sum |dy y|, far below; the kernel's
            # elements by at most 1000 units of the sizes of their terms, which add up like the terms do
            size = float((cpu64(got).abs() * e.abs()).sum()) + float(dy64.abs().sum())
            assert abs(diff - inner) <= 1000 * UNIT * size, (norm, what, diff, inner)


def test_in_place_none_and_side_stream(api):
    d, N = 128, 301
    rot = api.Rotary(d, AXES[d], norm="rms")
    q, k, v = make(api, (1, N, 4, 2, d), torch.bfloat16, 41)
    pos = torch.randint(0, 5000, (N, 3), device="cuda", dtype=torch.int32)
    want = rot.forward(q, k, None, pos=pos)
    assert want[2] is None
    only_q = rot.forward(q, pos=pos)
    assert torch.equal(only_q[0], want[0]) and only_q[1] is None
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = rot.forward(q, k, None, pos=pos)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(on_side[0], want[0]) and torch.equal(on_side[1], want[1])
    q2, k2 = q.clone(memory_format=torch.contiguous_format), k.clone(memory_format=torch.contiguous_format)
    rot.forward(q2, k2, pos=pos, out=(q2, k2, None))
    assert torch.equal(q2, want[0]) and torch.equal(k2, want[1])


def test_captured_and_replayed(api):
    d, N, h = 64, 57, 3
    rot = api.Rotary(d, AXES[d], norm="layer")
    q, k, v = (t.clone() for t in make(api, (1, N, h, h, d), torch.float32, 51))
    pos = torch.randint(0, 5000, (N, 3), device="cuda", dtype=torch.int32)
    dy = torch.randn(1, N, h, d, device="cuda")
    rot.backward(dy, q=q, pos=pos)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = rot.forward(q, k, v, pos=pos)
        dx, grads = rot.backward(dy, q=q, pos=pos)
    for seed in (1, 2):
        torch.manual_seed(seed)
        q.normal_()
        dy.normal_()
        pos.random_(0, 9000)
        graph.replay()
        want = rot.forward(q, k, v, pos=pos)
        want_dx, want_g = rot.backward(dy, q=q, pos=pos)
        assert all(torch.equal(a, b) for a, b in zip(y, want))
        assert torch.equal(dx[0], want_dx[0]) and all(torch.equal(grads[n], want_g[n]) for n in grads)


def test_nothing_leaks_between_rows(api):
    """A row of NaN or infinity spoils itself (and the weights' gradients), no other row."""
    d, N, h = 128, 41, 5
    rot = api.Rotary(d, AXES[d], norm="layer")
    q, _, _ = make(api, (1, N, h, h, d), torch.bfloat16, 61)
    q = q.clone()
    pos = torch.randint(0, 5000, (N, 3), device="cuda", dtype=torch.int32)
    dy = torch.randn_like(q)
    y, (dx, _, _) = rot.forward(q, pos=pos)[0], rot.backward(dy, q=q, pos=pos)[0]
    q[0, 7, 2], q[0, 8, 0, 5] = float("nan"), float("inf")
    y2, (dx2, _, _) = rot.forward(q, pos=pos)[0], rot.backward(dy, q=q, pos=pos)[0]
    keep = torch.ones(N, h, dtype=torch.bool, device="cuda")
    keep[7, 2] = keep[8, 0] = False
    assert torch.equal(y[0][keep], y2[0][keep]) and torch.equal(dx[0][keep], dx2[0][keep])
    assert torch.isnan(y2[0, 7, 2]).all()


@pytest.mark.parametrize("T,H,W,heads,d,block,th,tw,n_text", [(4, 8, 8, 2, 64, 64, 4, 4, 0), (2, 16, 32, 3, 128, 128, 8, 16, 19)])
def test_with_the_attention_that_follows(api, T, H, W, heads, d, block, th, tw, n_text):
    """Fused projection -> norm, positions, tile-major order -> dense attention -> scatter, against fp64."""
    plan = api.Plan(T, H, W, d, block, th, tw, n_text=n_text)
    rot = api.Rotary(d, AXES[d], norm="rms")
    qkv = make(api, (1, plan.N, heads, heads, d), torch.bfloat16, 71)
    w = params(d, torch.bfloat16, "rms", 72)
    Q, K, V = rot.forward(*qkv, plan=plan, **w)
    O, _, _ = plan.entropy_attn(Q, K, V, want_entropy=False)
    O = plan.tile_major_scatter(O)
    plan.check_status()
    pos = grid_pos(T, H, W, n_text)
    q, k = (reference(cpu64(x), pos, "rms", cpu64(w[n + "_weight"]), None, False, 1e-6, plan.N_video)[0]
            for x, n in zip(qkv, "qk"))
    # the attention works on the rounded q and k
    q, k = (t.to(torch.bfloat16).double() for t in (q, k))
    p = torch.softmax(torch.einsum("bnhd,bmhd->bhnm", q, k) / math.sqrt(d), -1)
    want = torch.einsum("bhnm,bmhd->bhnd", p, cpu64(qkv[2]))
    err = (cpu64(O) - want).abs()
    # a q or k on the border of two bf16 values may round the other way: its scores move by 2^-8 of a term; else the bar
    # of the attention calls, 1e-2 and 5e-3 in relative L2
    assert float(err.max()) <= 2e-2 and float(err.norm() / want.norm()) <= 5e-3
    plan.close()
