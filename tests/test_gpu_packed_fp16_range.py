"""fp16 gradients of packed attention follow the size of what they are made of: a small upstream gradient over many keys does not
sink into fp16's subnormal numbers, a large one does not overflow on the way.

The gradients are linear in dO.  Scaled by a power of two, every fp32 and fp16 number between dO and the results scales
with it exactly, as long as none of them leaves its type's normal range; the results are rounded to fp16, whose spacing stops
shrinking below 2^-14.  So the results have to be the scaled ones bit by bit where both are normal numbers, and within the half
spacing 2^-25 (and the scaled result's own rounding, 2^-11 of it) where they are not."""
import pytest
import torch

from tests.packed_reference import i32, packed, randn, reference

pytestmark = pytest.mark.gpu
HALF = torch.float16
NORMAL = 2.0 ** -14


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def unit_do(shape, seed):
    """+-(1 + i / 1024) 2^e, e = -2 .. 1: normal numbers of fp16 for scales of 2^-12 .. 2^13."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda lo, hi: torch.randint(lo, hi, shape, generator=g, device="cuda").double()
    return ((2 * r(0, 2) - 1) * (1 + r(0, 1024) / 1024) * 2.0 ** r(-2, 2)).to(HALF)


def gradients(attn, q, k, v, do, cu, ck, max_q, max_k, sm_scale):
    o, lse = attn.forward(q, k, v, cu, ck, max_q=max_q, max_k=max_k, want_lse=True, sm_scale=sm_scale)
    out = attn.backward(do, q, k, v, o, lse, cu, ck, max_q=max_q, max_k=max_k, sm_scale=sm_scale)
    attn.check_status()
    return [t.double() for t in out]


@pytest.mark.parametrize("power", [-12, -7, 7, 12])
@pytest.mark.parametrize("d,hq,hk,causal,lens,v_mul", [
    (128, 2, 2, False, [1500], 1.0), (64, 6, 2, True, [700, 3, 130], 1.0), (128, 4, 1, True, [2, 90], 8.0), (64, 2, 2, False, [60], 8.0)])
def test_gradients_scale_with_do(api, power, d, hq, hk, causal, lens, v_mul):
    cu, n = packed(lens), sum(lens)
    q, k = randn((n, hq, d), HALF, 1, 0.3), randn((n, hk, d), HALF, 2)
    v, do = randn((n, hk, d), HALF, 3, v_mul), unit_do((n, hq, d), 4)
    attn = api.PackedAttn(hq, hk, d, dtype=HALF, causal=causal)
    args = (i32(cu), None, max(lens), max(lens), 1 / 256 if v_mul > 1 else None)     # (results inside fp16's range)
    one = gradients(attn, q, k, v, do, *args)
    scaled = gradients(attn, q, k, v, do * 2.0 ** power, *args)
    compared = 0
    for name, a, b in zip(("dq", "dk", "dv"), one, scaled):
        assert a.isfinite().all()
        want = a * 2.0 ** power
        if float(want.abs().max()) > 65504:              # dv's sums
            assert name == "dv"
            want = want.clamp(-65504, 65504)
            b = b.clamp(-65504, 65504)
        normal = (a.abs() >= NORMAL) & (want.abs() >= NORMAL)
        assert torch.equal(b[normal], want[normal]), name
        compared += int(normal.sum())                    # (one of the three may lie below as a whole)
        off = (b - want).abs()[~normal]
        tol = (2.0 ** -25 + 2.0 ** -11 * want.abs()[~normal]) * max(1.0, 2.0 ** power)
        assert (off <= tol).all(), name
    assert compared


@pytest.mark.parametrize("d", [64, 128])
def test_small_upstream_gradient_over_long_rows(api, d):
    """4,096 keys seen about evenly, |dO| about 4e-4: dS about 1e-6, which fp16 as it stands holds with four bits.  dq is a normal
    number of fp16 (K is large)."""
    n = 4096
    q, k = randn((n, 1, d), HALF, 1, 1e-3), randn((n, 1, d), HALF, 2)
    v, do = randn((n, 1, d), HALF, 3), unit_do((n, 1, d), 4) * 2.0 ** -12
    attn = api.PackedAttn(1, 1, d, dtype=HALF, causal=False)
    dq, dk, dv = gradients(attn, q, k * 64, v, do, i32([0, n]), None, n, n, 1.0)
    want = reference(q, k * 64, v, [0, n], [0], [n], False, 1.0, do=do)
    # two roundings of 2^-11 at most, dS and the result; the fp32 steps lie far below
    assert float(want["dq"].abs().median()) > NORMAL
    err = float(((dq - want["dq"]).norm() / want["dq"].norm()))
    assert err <= 2 * 2.0 ** -11, err


@pytest.mark.parametrize("d", [64, 128])
def test_probabilities_of_long_rows(api, d):
    """One query over 70,000 keys: dv_j = P_j dO with P about 2^-16, a subnormal number of fp16.  P's rounding and the result's,
    2^-11 each, and the error of the exponent S - lse, of the scores' products and of 2^x; lse is the forward call's."""
    m = 70000
    q, k = randn((1, 1, d), HALF, 1), randn((m, 1, d), HALF, 2, 0.3)
    v, do = randn((m, 1, d), HALF, 3), unit_do((1, 1, d), 4) * 64
    attn = api.PackedAttn(1, 1, d, dtype=HALF, causal=False)
    cu, ck = i32([0, 1]), i32([0, m])
    o, lse = attn.forward(q, k, v, cu, ck, max_q=1, max_k=m, want_lse=True)
    _, _, dv = attn.backward(do, q, k, v, o, lse, cu, ck, max_q=1, max_k=m)
    s = d ** -0.5 * (k[:, 0].double() @ q[0, 0].double())
    want = torch.exp(s - lse.double()[0, 0])[:, None] * do[0].double()
    size = d ** -0.5 * float(q[0, 0].double().norm() * k[:, 0].double().norm(dim=-1).max())
    e = size * (d + 8) * 2.0 ** -23 + (float(lse[0, 0].abs()) + 12 + 8) * 2.0 ** -22
    u = 2.0 ** -11
    tol = want.abs() * ((1 + u) ** 2 * (1 + 2 * e) - 1) + 2.0 ** -25
    assert ((dv[:, 0].double() - want).abs() <= tol).all()


def test_scale_ignores_what_lies_outside(api):
    """Huge numbers and NaN in dO and V outside the sequences do not touch the gradients inside; sequences without
    gradient give zeros."""
    d, n, pad = 64, 200, 5
    q, k, v = (randn((n + 2 * pad, 2, d), HALF, i) for i in range(3))
    do = unit_do((n + 2 * pad, 2, d), 4) * 2.0 ** -12
    attn = api.PackedAttn(2, 2, d, dtype=HALF, causal=True)
    cu = i32([pad, pad + 50, pad + n])
    inside = slice(pad, pad + n)
    base = [t[inside] for t in gradients(attn, q, k, v, do, cu, None, 150, 150, None)]
    for bad in (65504.0, float("inf"), float("nan")):
        for t in (do, v):
            t[:pad], t[pad + n:] = bad, bad
        got = gradients(attn, q, k, v, do, cu, None, 150, 150, None)
        assert all(torch.equal(a, b[inside]) for a, b in zip(base, got))
    do.zero_()
    assert all((t[inside] == 0).all() for t in gradients(attn, q, k, v, do, cu, None, 150, 150, None))


def test_replays_follow_the_size_of_do(api):
    """The scale belongs to a call: replays of a captured one with a large dO, then a small one, give what calls of their own give."""
    d, n = 64, 300
    q, k, v = (randn((n, h, d), HALF, i) for i, h in enumerate((4, 2, 2)))
    do, unit = torch.empty(n, 4, d, dtype=HALF, device="cuda"), unit_do((n, 4, d), 4)
    attn = api.PackedAttn(4, 2, d, dtype=HALF, causal=True)
    cu = i32([0, 100, n])
    o, lse = attn.forward(q, k, v, cu, max_q=200, max_k=200, want_lse=True)
    step = lambda: attn.backward(do, q, k, v, o, lse, cu, max_q=200, max_k=200)
    do.copy_(unit)
    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    first = None
    for power in (12, -12, 0, 12):
        do.copy_(unit * 2.0 ** power)
        for graph, _ in graphs:
            graph.replay()
        want = step()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            there = step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(there, want))
        first = [t.clone() for t in want] if first is None else first
    assert all(torch.equal(a, b) for a, b in zip(first, want))
    attn.check_status()


@pytest.mark.parametrize("d,group,hk", [(64, 1, 5), (64, 3, 2), (128, 5, 3), (128, 1, 2), (64, 22, 2)])
def test_heads_of_different_sizes(api, d, group, hk):
    """Every key/value head has a scale of its own: the gradients are those of calls with one such head, bit by bit, whatever the other
    heads hold; slices of fused tensors among them."""
    lens = [70, 1, 333]
    cu, n = packed(lens), sum(lens)
    sizes = torch.tensor([2.0 ** (-8 + 7 * (i % 3)) for i in range(hk)], device="cuda", dtype=HALF)
    fused = randn((n, (group + 2) * hk, d), HALF, 1)
    q, k, v = fused[:, :group * hk], fused[:, group * hk:-hk], fused[:, -hk:]
    v *= sizes[:, None]
    do = unit_do((group * hk, n, d), 4).transpose(0, 1) * sizes.flip(0).repeat_interleave(group)[:, None]
    attn, one = api.PackedAttn(group * hk, hk, d, dtype=HALF), api.PackedAttn(group, 1, d, dtype=HALF)
    kw = dict(max_q=max(lens), max_k=max(lens))
    o, lse = attn.forward(q, k, v, i32(cu), want_lse=True, **kw)
    dq, dk, dv = attn.backward(do, q, k, v, o, lse, i32(cu), **kw)
    for h in range(hk):
        mine, kv = slice(h * group, (h + 1) * group), slice(h, h + 1)
        got = one.backward(do[:, mine], q[:, mine], k[:, kv], v[:, kv], o[:, mine], lse[:, mine].contiguous(), i32(cu),
                           o_rest=lse.o_rest[:, mine].contiguous(), **kw)
        assert torch.equal(got[0], dq[:, mine]) and torch.equal(got[1], dk[:, kv]) and torch.equal(got[2], dv[:, kv]), h
    attn.check_status()
