"""Gradients of attention over packed sequences (``tra_packed_attn_backward``) against fp64 formulas and differences; the
tolerances are derived in packed_reference.py."""
import math

import pytest
import torch

from tests.packed_reference import check, i32, packed, randn, reference

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def run(api, dtype, d, hq, hk, causal, lens_q, lens_k=None, seed=1, sm_scale=None):
    """Rows outside the sequences hold NaN in the inputs and a mark in the outputs."""
    same = lens_k is None
    lens_k = lens_q if same else lens_k
    pad = 3
    cu, ck = [pad + c for c in packed(lens_q)], [pad + c for c in packed(lens_k)]
    tq, tk = cu[-1] + pad, ck[-1] + pad
    q, do = randn((tq, hq, d), dtype, seed, 1.5), randn((tq, hq, d), dtype, seed + 3)
    k, v = randn((tk, hk, d), dtype, seed + 1), randn((tk, hk, d), dtype, seed + 2)
    for t, c in ((q, cu), (do, cu), (k, ck), (v, ck)):
        t[:c[0]] = t[c[-1]:] = float("nan")
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, causal=causal)
    kw = dict(max_q=max(lens_q), max_k=max(lens_k), sm_scale=sm_scale)
    cu_q, cu_k = i32(cu), None if same else i32(ck)
    o, lse = torch.full_like(q, float("nan")), torch.full((tq, hq), float("nan"), device="cuda")
    attn.forward(q, k, v, cu_q, cu_k, o=o, lse=lse, **kw)
    outs = [torch.full_like(t, 77.0) for t in (q, k, v)]
    got = attn.backward(do, q, k, v, o, lse, cu_q, cu_k, dq=outs[0], dk=outs[1], dv=outs[2], **kw)
    attn.check_status()
    scale = 1 / math.sqrt(d) if sm_scale is None else sm_scale
    want = reference(q, k, v, cu, ck[:-1], ck[1:], causal, scale, do=do)
    for name, t, c in (("dq", got[0], cu), ("dk", got[1], ck), ("dv", got[2], ck)):
        rows = slice(c[0], c[-1])
        check(t[rows], want[name][rows], want[name + "_tol"][rows], name)
        assert (t[:c[0]] == 77).all() and (t[c[-1]:] == 77).all(), name
    again = attn.backward(do, q, k, v, o, lse, cu_q, cu_k, **kw)
    for t, t2, c in zip(got, again, (cu, ck, ck)):
        assert torch.equal(t[c[0]:c[-1]], t2[c[0]:c[-1]])
    attn.close()


LENS = [[1], [128], [129, 127], [1, 300, 2, 77, 513], [0, 5, 0, 130, 0], [3] * 40, [255, 256, 257], [1000]]


@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d,hq,hk", [(BF, 128, 2, 2), (HALF, 64, 3, 1), (BF, 64, 10, 2), (HALF, 128, 8, 1)])
def test_prompts(api, lens, causal, dtype, d, hq, hk):
    run(api, dtype, d, hq, hk, causal, lens)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 6, 7, 16, 43, 64, 100, 128])
def test_groups(api, group):
    run(api, BF, 64, group, 1, True, [70, 9, 201])
    run(api, HALF, 128, 2 * group, 2, False, [33, 140])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("group", [1, 4, 12, 13, 20, 22, 32, 33])
def test_streamed_tiles(api, causal, group):
    """Lengths about the tiles that the blocks stream: 64 keys or 64 rows (64 / group tokens) at head_dim 64, 128 where that
    would leave rows empty."""
    t = 64 // group
    run(api, BF, 64, group, 1, causal, [63, 64, 65, 1, 127, 128, 129, 191, 193])
    run(api, HALF, 64, 2 * group, 2, causal, [t, 2 * t + 1, 3 * t, 1], [65, 64 + t, 320, 63])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_more_or_fewer_keys_than_queries(api, causal, dtype, d):
    run(api, dtype, d, 4, 2, causal, [100, 40, 60, 300, 20], [1000, 40, 25, 7, 0])
    run(api, dtype, d, 4, 4, causal, [200], [0])
    run(api, dtype, d, 4, 4, causal, [0, 3], [150, 300])
    run(api, dtype, d, 2, 2, causal, [0], [150])


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("lens", [[2], [2, 3, 1, 2], [17, 5], [40, 130], [300]], ids=str)
@pytest.mark.parametrize("d,hq,hk", [(128, 4, 2), (64, 3, 3), (64, 16, 1)])
def test_rows_that_cancel(api, dtype, lens, d, hq, hk):
    """Short sequences and peaked rows, where P (dP - delta) cancels: the remainder of o that ``want_lse`` keeps takes the
    rounding of o out of the gradients."""
    cu = packed(lens)
    n = cu[-1]
    q, k, v, do = (randn((n, h, d), dtype, i, 2.5 if i == 0 else 1.0) for i, h in enumerate((hq, hk, hk, hq)))
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, causal=True)
    kw = dict(max_q=max(lens), max_k=max(lens))
    o, lse = attn.forward(q, k, v, i32(cu), want_lse=True, **kw)
    want = reference(q, k, v, cu, cu[:-1], cu[1:], True, d ** -0.5, do=do, o_rest=True)
    u = torch.finfo(dtype).eps / 2
    # O and its remainder together: the rounding of the remainder, u^2 |o|, and the errors that come before
    both = o.double() + lse.o_rest.double()
    check(both, want["o"], want["o_tol"] - u * want["o"].abs() * (1 + u) + 2.0 ** -24, "o + rest")
    for name, t in zip(("dq", "dk", "dv"), attn.backward(do, q, k, v, o, lse, i32(cu), **kw)):
        check(t, want[name], want[name + "_tol"], name)
    o2 = torch.empty_like(o)
    attn.forward(q * 0.5, k, v, i32(cu), o=o2, lse=lse, **kw)            # an lse used again keeps its remainder up to date
    alone = attn.forward(q * 0.5, k, v, i32(cu), want_lse=True, **kw)
    assert torch.equal(o2, alone[0]) and torch.equal(lse.o_rest, alone[1].o_rest)
    with pytest.raises(ValueError):
        attn.backward(do[1:], q[1:], k, v, o[1:], lse, i32(cu), **kw)


def test_many_sequences(api):
    lens = [(7 * i) % 4 for i in range(1050)]
    lens[2], lens[700] = 400, 130
    run(api, BF, 64, 2, 1, True, lens)


def test_scales(api):
    run(api, BF, 128, 2, 2, True, [200], sm_scale=0.5)
    run(api, HALF, 64, 2, 2, False, [300], sm_scale=1e-4)


def test_against_differences(api):
    """<gradient, e> against central differences of the fp64 definition along a direction e."""
    d, hq, hk, lens = 64, 4, 2, [37, 150]
    cu = packed(lens)
    n = cu[-1]
    for causal in (True, False):
        q, do = randn((n, hq, d), HALF, 1, 1.5), randn((n, hq, d), HALF, 4)
        k, v = randn((n, hk, d), HALF, 2), randn((n, hk, d), HALF, 3)
        attn = api.PackedAttn(hq, hk, d, dtype=HALF, causal=causal)
        kw = dict(max_q=max(lens), max_k=max(lens))
        o, lse = attn.forward(q, k, v, i32(cu), want_lse=True, **kw)
        grads = attn.backward(do, q, k, v, o, lse, i32(cu), **kw)
        want = reference(q, k, v, cu, cu[:-1], cu[1:], causal, d ** -0.5, do=do)

        def f(q, k, v):
            total = 0.0
            for a, b in zip(cu[:-1], cu[1:]):
                s = torch.einsum("nhd,mhd->hnm", q[a:b], k[a:b].repeat_interleave(hq // hk, 1)) * d ** -0.5
                if causal:
                    s = s.masked_fill(torch.ones(b - a, b - a, device="cuda").triu(1).bool(), -math.inf)
                out = torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), v[a:b].repeat_interleave(hq // hk, 1))
                total += float((out * do[a:b].double()).sum())
            return total

        base = [t.double() for t in (q, k, v)]
        step = 1e-5
        for i, name in enumerate(("dq", "dk", "dv")):
            e = randn(base[i].shape, torch.float32, 20 + i).double()
            up, down = list(base), list(base)
            up[i], down[i] = base[i] + step * e, base[i] - step * e
            diff = (f(*up) - f(*down)) / (2 * step)
            inner = float((grads[i].double() * e).sum())
            # the elements' tolerances at their worst together; the differences' own error is of the order step^2 and
            # 2^-52 / step of the sum's terms, far below
            tol = float((want[name + "_tol"] * e.abs()).sum())
            assert abs(diff - inner) <= tol, (name, diff, inner, tol)
            # and far closer than the worst case: the errors are independent, their root sum of squares times eight
            rss = float(((want[name + "_tol"] * e) ** 2).sum().sqrt())
            assert abs(diff - inner) <= 8 * rss + 1e-6 * abs(diff), (name, diff, inner, rss)


def test_strides(api):
    """Slices of fused projections in, slices of a fused gradient out."""
    d, hq, hk, lens = 128, 6, 2, [200, 77]
    cu, n = packed(lens), sum(lens)
    fused = randn((n, hq + 2 * hk, d), BF, 3)
    q, k, v = fused[:, :hq], fused[:, hq:hq + hk], fused[:, hq + hk:]
    do = randn((hq, n, d), BF, 4).transpose(0, 1)
    attn = api.PackedAttn(hq, hk, d)
    kw = dict(max_q=200, max_k=200)
    o, lse = attn.forward(q, k, v, i32(cu), want_lse=True, **kw)
    want = attn.backward(do.contiguous(), q.contiguous(), k.contiguous(), v.contiguous(), o, lse, i32(cu), **kw)
    g = torch.full_like(fused, 5.0)
    attn.backward(do, q, k, v, o, lse, i32(cu), dq=g[:, :hq], dk=g[:, hq:hq + hk], dv=g[:, hq + hk:], **kw)
    assert torch.equal(g, torch.cat(want, 1))


def test_capture_and_streams(api):
    d, hq, hk, n = 64, 4, 2, 333
    attn = api.PackedAttn(hq, hk, d)
    q, k, v, do = (randn((n, h, d), BF, i) for i, h in enumerate((hq, hk, hk, hq)))
    cu = i32([0, 100, n])

    def step():
        o, lse = attn.forward(q, k, v, cu, max_q=n, max_k=n, want_lse=True)
        return (o, *attn.backward(do, q, k, v, o, lse, cu, max_q=n, max_k=n))

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = step()
    b = step()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for cut in (100, 1, n):
        cu[1] = cut
        q.normal_()
        do.normal_()
        graph.replay()
        want = step()
        assert all(torch.equal(x, y) for x, y in zip(out, want))
    attn.check_status()


def test_layer_around_it(api):
    """Fused projection -> head norm and rotary positions -> packed attention, and all the way back to the projection's
    and the norm weights' gradients, against differentiation of the definition in fp64."""
    d, hq, hk, lens = 64, 4, 2, [61, 130, 1]
    cu, n = packed(lens), sum(lens)
    rot = api.Rotary(d, (24, 20, 20), norm="rms")
    attn = api.PackedAttn(hq, hk, d, dtype=HALF, causal=True)
    fused = randn((1, n, hq + 2 * hk, d), HALF, 7)
    wq, wk = (1 + 0.1 * randn((d,), torch.float32, 8)).to(HALF), (1 + 0.1 * randn((d,), torch.float32, 9)).to(HALF)
    pos = torch.randint(0, 300, (n, 3), device="cuda", dtype=torch.int32)
    do = randn((n, hq, d), HALF, 10)
    split = lambda t: (t[:, :, :hq], t[:, :, hq:hq + hk], t[:, :, hq + hk:])
    q, k, v = rot.forward(*split(fused), pos=pos, q_weight=wq, k_weight=wk)
    kw = dict(max_q=max(lens), max_k=max(lens))
    o, lse = attn.forward(q[0], k[0], v[0], i32(cu), want_lse=True, **kw)
    dq, dk, dv = attn.backward(do, q[0], k[0], v[0], o, lse, i32(cu), **kw)
    dfused = torch.empty_like(fused)
    _, wg = rot.backward(dq[None], dk[None], dv[None], q=split(fused)[0], k=split(fused)[1], pos=pos, q_weight=wq, k_weight=wk,
                         out=split(dfused))
    attn.check_status()

    x = fused.double().requires_grad_()
    weights = [w.double().requires_grad_() for w in (wq, wk)]
    axis = torch.tensor([0] * 12 + [1] * 10 + [2] * 10, device="cuda")
    freq = torch.tensor([1e4 ** (-2 * i / c) for c in (24, 20, 20) for i in range(c // 2)], device="cuda", dtype=torch.float64)
    ang = pos.double()[:, axis] * freq
    qkv = []
    for t, w in zip(split(x), weights + [None]):
        if w is not None:
            t = w * t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6)
            z = torch.view_as_complex(t.reshape(1, n, -1, d // 2, 2)) * torch.polar(torch.ones_like(ang), ang)[:, None]
            t = torch.view_as_real(z).flatten(-2)
        qkv.append(t[0])
    outs = []
    for a, b in zip(cu[:-1], cu[1:]):
        qs, ks, vs = (t[a:b] for t in qkv)
        s = torch.einsum("nhd,mhd->hnm", qs, ks.repeat_interleave(hq // hk, 1)) * d ** -0.5
        s = s.masked_fill(torch.ones(b - a, b - a, device="cuda").triu(1).bool(), -math.inf)
        outs.append(torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), vs.repeat_interleave(hq // hk, 1)))
    out = torch.cat(outs)
    gx, gq, gk = torch.autograd.grad(out, [x] + weights, do.double())
    # every stage rounds to fp16 (2^-11): q, k (scores of up to about 5 move by their sum), P, dS, dq, dk, dx: below 32
    # roundings of the size of the result, in the relative norm
    for name, got, want in (("o", o, out), ("dx", dfused, gx), ("wq", wg["q_weight"], gq), ("wk", wg["k_weight"], gk)):
        rel = float(((got.double() - want).norm() / want.norm()).detach())
        assert rel <= 32 * 2.0 ** -11, (name, rel)
