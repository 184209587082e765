"""Attention over packed sequences with a window and first tokens, forward and gradients, against a plain fp64 implementation; the
tolerances are derived in packed_reference.py."""
import math

import pytest
import torch

from tests.packed_reference import check, i32, packed, randn
from tests.window_reference import reference, seen

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def forward(api, dtype, d, hq, hk, window, sinks, lens_q, lens_k=None, slots=None, seed=1, mul=1.5):
    """Rows outside the sequences: queries and keys hold NaN, O and lse a mark that has to stay."""
    lens_k = lens_q if lens_k is None else lens_k
    pad = 3
    cu = [pad + c for c in packed(lens_q)]
    total_q = cu[-1] + pad
    if slots is None:
        kb = [pad + c for c in packed(lens_k)[:-1]]
        total_k = pad + sum(lens_k) + pad
    else:
        kb = [s * slots for s in range(len(lens_k))]
        total_k = slots * len(lens_k)
    ke = [b + n for b, n in zip(kb, lens_k)]
    q, k, v = (randn((n, h, d), dtype, seed + i, mul if i == 0 else 1.0)
               for i, (n, h) in enumerate(((total_q, hq), (total_k, hk), (total_k, hk))))
    q[:cu[0]], q[cu[-1]:] = float("nan"), float("nan")
    own = torch.zeros(total_k, dtype=torch.bool, device="cuda")
    for b, e in zip(kb, ke):
        own[b:e] = True
    k[~own], v[~own] = float("nan"), float("inf")
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, window=window, sinks=sinks)
    want = reference(q, k, v, cu, kb, ke, window, sinks, d ** -0.5)
    kw = dict(k_range=(i32(kb), i32(ke)), max_q=max(lens_q), max_k=max(lens_k))
    o = torch.full((total_q, hq, d), 77.0, dtype=dtype, device="cuda")
    lse = torch.full((total_q, hq), 55.0, device="cuda")
    attn.forward(q, k, v, i32(cu), o=o, lse=lse, **kw)
    attn.check_status()
    rows = slice(cu[0], cu[-1])
    check(o[rows], want["o"][rows], want["o_tol"][rows], "o")
    check(lse[rows], want["lse"][rows], want["lse_tol"][rows], "lse")
    for t, mark in ((o, 77.0), (lse, 55.0)):
        assert (t[:cu[0]] == mark).all() and (t[cu[-1]:] == mark).all()
    o2 = torch.full_like(o, 77.0)
    attn.forward(q, k, v, i32(cu), o=o2, **kw)
    assert torch.equal(o, o2)


def backward(api, dtype, d, hq, hk, window, sinks, lens_q, lens_k=None, seed=1):
    same = lens_k is None
    lens_k = lens_q if same else lens_k
    pad = 3
    cu, ck = [pad + c for c in packed(lens_q)], [pad + c for c in packed(lens_k)]
    tq, tk = cu[-1] + pad, ck[-1] + pad
    q, do = randn((tq, hq, d), dtype, seed, 1.5), randn((tq, hq, d), dtype, seed + 3)
    k, v = randn((tk, hk, d), dtype, seed + 1), randn((tk, hk, d), dtype, seed + 2)
    for t, c in ((q, cu), (do, cu), (k, ck), (v, ck)):
        t[:c[0]] = t[c[-1]:] = float("nan")
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, window=window, sinks=sinks)
    kw = dict(max_q=max(lens_q), max_k=max(lens_k))
    cu_q, cu_k = i32(cu), None if same else i32(ck)
    o, lse = torch.full_like(q, float("nan")), torch.full((tq, hq), float("nan"), device="cuda")
    attn.forward(q, k, v, cu_q, cu_k, o=o, lse=lse, **kw)
    outs = [torch.full_like(t, 77.0) for t in (q, k, v)]
    got = attn.backward(do, q, k, v, o, lse, cu_q, cu_k, dq=outs[0], dk=outs[1], dv=outs[2], **kw)
    attn.check_status()
    want = reference(q, k, v, cu, ck[:-1], ck[1:], window, sinks, d ** -0.5, do=do)
    for name, t, c in (("dq", got[0], cu), ("dk", got[1], ck), ("dv", got[2], ck)):
        rows = slice(c[0], c[-1])
        check(t[rows], want[name][rows], want[name + "_tol"][rows], name)
        assert (t[:c[0]] == 77).all() and (t[c[-1]:] == 77).all(), name
    again = attn.backward(do, q, k, v, o, lse, cu_q, cu_k, **kw)
    for t, t2, c in zip(got, again, (cu, ck, ck)):
        assert torch.equal(t[c[0]:c[-1]], t2[c[0]:c[-1]])


WINDOWS = [(1, 0), (1, 1), (7, 3), (64, 8), (100, 0), (128, 128), (200, 130), (129, 4), (500, 1), (300, 256)]
LENS = [1, 300, 2, 77, 0, 513, 700]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("dtype,d,hq,hk", [(BF, 128, 2, 2), (HALF, 64, 3, 1), (BF, 64, 10, 2), (HALF, 128, 8, 1)])
def test_prompts(api, dtype, d, hq, hk, window, sinks):
    forward(api, dtype, d, hq, hk, window, sinks, LENS)


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("dtype,d,hq,hk", [(BF, 128, 2, 2), (HALF, 64, 3, 1), (BF, 64, 10, 2), (HALF, 128, 8, 1), (BF, 64, 33, 1)])
def test_gradients(api, dtype, d, hq, hk, window, sinks):
    backward(api, dtype, d, hq, hk, window, sinks, LENS)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 16, 43, 64, 100, 128])
def test_groups(api, group):
    for call in (forward, backward):
        call(api, BF, 64, group, 1, 20, 5, [70, 9, 201])
        call(api, HALF, 128, 2 * group, 2, 40, 0, [33, 140])


@pytest.mark.parametrize("window,sinks", [(1, 0), (30, 2), (256, 64), (1000, 200)])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_more_or_fewer_keys_than_queries(api, dtype, d, window, sinks):
    """Chunks behind a cache; sequences with fewer keys than queries, whose first queries see nothing; none at all."""
    for call in (forward, backward):
        call(api, dtype, d, 4, 2, window, sinks, [100, 40, 60, 300, 20], [1000, 40, 25, 7, 0])
        call(api, dtype, d, 4, 4, window, sinks, [200, 0, 3], [1200, 150, 300])
    forward(api, dtype, d, 4, 4, window, sinks, [17, 130], [2000, 131], slots=2048)


@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 64), (65, 3), (500, 7), (3000, 100)])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64), (BF, 64), (HALF, 128)])
@pytest.mark.parametrize("hq,hk", [(1, 1), (10, 2), (16, 1)])
def test_one_token(api, dtype, d, hq, hk, window, sinks):
    forward(api, dtype, d, hq, hk, window, sinks, [1] * 7, [1, 64, 65, 0, 777, 3000, 16])
    forward(api, dtype, d, hq, hk, window, sinks, [1, 0, 1], [2000, 100, 1], slots=2048)
    forward(api, dtype, d, hq, hk, window, sinks, [1], [40000])


@pytest.mark.parametrize("window,sinks", [(1, 1), (5, 0), (70, 66), (600, 2)])
def test_few_tokens(api, window, sinks):
    forward(api, BF, 128, 4, 2, window, sinks, [8, 3, 1, 0, 8, 5], [8, 700, 33, 20, 1900, 2])
    forward(api, HALF, 64, 5, 1, window, sinks, [3, 2, 3], [70, 2, 641], slots=700)
    forward(api, BF, 64, 1, 1, window, sinks, [16, 15], [16, 4000])


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_few_tiles_long_keys(api, dtype, d):
    """Tiles split over the parts of their key axis."""
    forward(api, dtype, d, 4, 4, 3000, 300, [97], [9000])
    forward(api, dtype, d, 4, 4, 2500, 0, [20, 1, 0, 33], [4001, 4097, 12, 0], slots=4100)


def test_many_sequences(api):
    lens = [(7 * i) % 5 for i in range(1100)]
    lens[3], lens[600], lens[1099] = 700, 301, 260
    for call in (forward, backward):
        call(api, BF, 64, 2, 1, 50, 3, lens)


def test_a_window_that_hides_nothing_is_causal_order(api):
    d, n = 128, 400
    q, k, v = randn((n, 4, d), BF, 1), randn((n, 2, d), BF, 2), randn((n, 2, d), BF, 3)
    kw = dict(max_q=n, max_k=n, want_lse=True)
    a, b = api.PackedAttn(4, 2, d), api.PackedAttn(4, 2, d, window=300, sinks=100)
    x, y = a.forward(q, k, v, i32([0, n]), **kw), b.forward(q, k, v, i32([0, n]), **kw)
    assert all(torch.equal(s, t) for s, t in zip(x, y))
    c = api.PackedAttn(4, 2, d, window=1 << 30, sinks=1 << 30)
    assert torch.equal(c.forward(q, k, v, i32([0, n]), **kw)[0], x[0])


def test_tokens_one_by_one_match_the_whole_prompt(api):
    d, hq, hk, n, window, sinks = 128, 6, 2, 400, 90, 5
    attn = api.PackedAttn(hq, hk, d, window=window, sinks=sinks)
    q, k, v = randn((n, hq, d), BF, 1), randn((n, hk, d), BF, 2), randn((n, hk, d), BF, 3)
    want = reference(q, k, v, [0, n], [0], [n], window, sinks, d ** -0.5)
    cache_k, cache_v = (torch.full((512, hk, d), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    at = 0
    for step in (150, 200, 30) + (1,) * 20:
        cache_k[at:at + step], cache_v[at:at + step] = k[at:at + step], v[at:at + step]
        o, l = attn.forward(q[at:at + step], cache_k, cache_v, i32([0, step]), k_range=(i32([0]), i32([at + step])),
                            max_q=step, max_k=512, want_lse=True)
        check(o, want["o"][at:at + step], want["o_tol"][at:at + step], f"o at {at}")
        check(l, want["lse"][at:at + step], want["lse_tol"][at:at + step], f"lse at {at}")
        at += step
    attn.check_status()


@pytest.mark.parametrize("nq", [1, 300])
def test_keys_that_nobody_sees_are_not_read(api, nq):
    """Keys in front of every window may hold anything (whole 8-key pieces behind the first tokens, which are loaded with them,
    aside)."""
    d, m, window, sinks = 64, 3000, 100, 6
    attn = api.PackedAttn(2, 2, d, window=window, sinks=sinks)
    q, k, v = randn((nq, 2, d), BF, 1), randn((m, 2, d), BF, 2), randn((m, 2, d), BF, 3)
    kw = dict(k_range=(i32([0]), i32([m])), max_q=nq, max_k=m, want_lse=True)
    want = attn.forward(q, k, v, i32([0, nq]), **kw)
    k[8:m - nq - window + 1], v[8:m - nq - window + 1] = float("nan"), float("inf")
    got = attn.forward(q, k, v, i32([0, nq]), **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    k[:] = 1
    v[:] = 0.5
    assert (attn.forward(q, k, v, i32([0, nq]), **kw)[0] == 0.5).all()


def test_against_differences(api):
    """<gradient, e> against central differences of the fp64 definition along a direction e."""
    d, hq, hk, lens, window, sinks = 64, 4, 2, [37, 250], 40, 6
    cu = packed(lens)
    n = cu[-1]
    q, do = randn((n, hq, d), HALF, 1, 1.5), randn((n, hq, d), HALF, 4)
    k, v = randn((n, hk, d), HALF, 2), randn((n, hk, d), HALF, 3)
    attn = api.PackedAttn(hq, hk, d, dtype=HALF, window=window, sinks=sinks)
    kw = dict(max_q=max(lens), max_k=max(lens))
    o, lse = attn.forward(q, k, v, i32(cu), want_lse=True, **kw)
    grads = attn.backward(do, q, k, v, o, lse, i32(cu), **kw)
    want = reference(q, k, v, cu, cu[:-1], cu[1:], window, sinks, d ** -0.5, do=do)

    def f(q, k, v):
        total = 0.0
        for a, b in zip(cu[:-1], cu[1:]):
            kk, vv = (t[a:b].repeat_interleave(hq // hk, 1) for t in (k, v))
            s = torch.einsum("nhd,mhd->hnm", q[a:b], kk) * d ** -0.5
            s = s.masked_fill(~seen(b - a, b - a, window, sinks, "cuda"), -math.inf)
            total += (torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), vv) * do[a:b].double()).sum()
        return total

    base = [t.double() for t in (q, k, v)]
    for i, name in enumerate(("dq", "dk", "dv")):
        e = torch.randn(base[i].shape, generator=torch.Generator(device="cuda").manual_seed(9 + i), device="cuda", dtype=torch.float64)
        step = 1e-4
        moved = [[t + sign * step * e if j == i else t for j, t in enumerate(base)] for sign in (1, -1)]
        slope = (f(*moved[0]) - f(*moved[1])) / (2 * step)
        got = (grads[i].double() * e).sum()
        # the gradient's own tolerance along e; the differences' third-order term is below 1e-8 of the values here
        allowed = (want[name + "_tol"] * e.abs()).sum() + 1e-6 * slope.abs() + 1e-6
        assert abs(float(got - slope)) <= float(allowed), name


def test_graphs_and_streams(api):
    """Captured calls of one handle, replayed side by side with eager ones; lengths live on the device."""
    d, hq, hk, n = 64, 4, 2, 600
    attn = api.PackedAttn(hq, hk, d, window=70, sinks=9)
    q, k, v, do = (randn((n, h, d), BF, i) for i, h in enumerate((hq, hk, hk, hq)))
    cu = i32([0, 250, n])

    def call():
        o, lse = attn.forward(q, k, v, cu, max_q=n, max_k=n, want_lse=True)
        return (o, lse) + attn.backward(do, q, k, v, o, lse, cu, max_q=n, max_k=n)
    call()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for mid in (250, 1, 599):
        cu[1] = mid
        q.normal_()
        for graph, _ in graphs:
            graph.replay()
        want = call()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))
    side, main = torch.cuda.Stream(), torch.cuda.current_stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        there = call()
    here = call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(there, here))
    attn.check_status()


def test_refusals(api):
    for kw, code in ((dict(window=-1), api.TRA_ERR_INVALID_ARG), (dict(window=4, sinks=-1), api.TRA_ERR_INVALID_ARG),
                     (dict(sinks=4), api.TRA_ERR_INVALID_ARG), (dict(window=4, causal=False), api.TRA_ERR_UNSUPPORTED),
                     (dict(window=(1 << 30) + 1), api.TRA_ERR_UNSUPPORTED)):
        with pytest.raises(api.TraError) as e:
            api.PackedAttn(4, 2, 64, **kw)
        assert e.value.code == code


@pytest.mark.parametrize("dtype,d,hq,hk", [(BF, 128, 4, 1), (HALF, 64, 5, 1), (HALF, 128, 12, 2)])
@pytest.mark.parametrize("window,sinks", [(40, 3), (200, 140)])
def test_first_keys_of_long_sequences(api, dtype, d, hq, hk, window, sinks):
    """Sequences whose queries are cut into units for the first keys' gradients, among others that are not; more keys than queries."""
    backward(api, dtype, d, hq, hk, window, sinks, [3, 2500, 0, 130, 1, 1200, 511])
    backward(api, dtype, d, hq, hk, window, sinks, [900, 0, 1500, 20], [1900, 10, 1400, 20])


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("d,hq,hk,window,sinks,lens", [(64, 2, 2, 16, 2, [64, 37]), (128, 4, 4, 200, 0, [100]), (128, 3, 1, 90, 3, [37, 20, 9]), (64, 5, 1, 10, 0, [25, 50]),
                                                       (64, 2, 1, 4000, 0, [150, 33])])
def test_gradients_of_few_rows_are_near_their_rounding(api, dtype, d, hq, hk, window, sinks, lens):
    """Of squared errors, with that of rounding a gradient as 1: rounding dS once would add 1 (it is as large relative to its terms), and the P rounded for
    the O that delta is made of a third.  In two pieces dS adds 2^-16 of that for dk, and a half at most for dq, whose every second 32 keys have one piece: sqrt(1.34) =
    1.16 and sqrt(1.84) = 1.36, and 5 % for sums of few terms."""
    n = sum(lens)
    q, do = randn((n, hq, d), dtype, 1), randn((n, hq, d), dtype, 4)
    k, v = randn((n, hk, d), dtype, 2), randn((n, hk, d), dtype, 3)
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, window=window, sinks=sinks)
    cu = packed(lens)
    kw = dict(max_q=max(lens), max_k=max(lens))
    o, lse = attn.forward(q, k, v, i32(cu), want_lse=True, **kw)
    dq, dk, _ = attn.backward(do, q, k, v, o, lse, i32(cu), **kw)
    want = reference(q, k, v, cu, cu[:-1], cu[1:], window, sinks, d ** -0.5, do=do)
    for got, name, most in ((dq, "dq", 1.36), (dk, "dk", 1.16)):
        x = want[name]
        assert (got.double() - x).norm() <= 1.05 * most * (x.to(dtype).double() - x).norm(), name
