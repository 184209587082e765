"""Attention over packed sequences (``tra_packed_attn``) against a plain fp64 implementation; the tolerances are derived in
packed_reference.py."""
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


def run(api, dtype, d, hq, hk, causal, lens_q, lens_k=None, slots=None, seed=1, mul=1.5, sm_scale=None):
    """Forward with and without lse against the reference.  Rows outside the sequences: queries and keys hold NaN, O and lse
    a mark that has to stay."""
    lens_k = lens_q if lens_k is None else lens_k
    pad = 3                                               # rows in front of and behind the sequences
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
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, causal=causal)
    scale = 1 / math.sqrt(d) if sm_scale is None else sm_scale
    want = reference(q, k, v, cu, kb, ke, causal, scale)
    kw = dict(k_range=(i32(kb), i32(ke)), max_q=max(lens_q), max_k=max(lens_k), sm_scale=sm_scale)
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
    _, none = attn.forward(q, k, v, i32(cu), o=o2, **kw)
    assert none is None and torch.equal(o, o2)
    attn.close()


LENS = [[1], [128], [129, 127], [1, 300, 2, 77, 513], [1000], [0, 5, 0, 130, 0], [3] * 40, [255, 256, 257], [640, 1]]


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
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_more_or_fewer_keys_than_queries(api, causal, dtype, d):
    """Chunks behind a cache; sequences with fewer keys than queries, whose first queries see nothing (causal); none at all."""
    run(api, dtype, d, 4, 2, causal, [100, 40, 60, 300, 20], [1000, 40, 25, 7, 0])
    run(api, dtype, d, 4, 4, causal, [200], [0])
    run(api, dtype, d, 4, 4, causal, [17, 130], [2000, 131], slots=2048)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d,hq,hk", [(BF, 128, 12, 2), (HALF, 64, 4, 4)])
def test_few_tiles_long_keys(api, causal, dtype, d, hq, hk):
    """More than 16 rows per key/value head, too few tiles for the GPU: tiles split over the keys."""
    run(api, dtype, d, hq, hk, causal, [97], [5000])
    run(api, dtype, d, hq, hk, causal, [20, 1, 0, 33], [3001, 4097, 12, 0], slots=4100)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64), (BF, 64), (HALF, 128)])
@pytest.mark.parametrize("hq,hk", [(1, 1), (12, 12), (10, 2), (16, 1), (5, 1)])
def test_one_token(api, dtype, d, hq, hk):
    run(api, dtype, d, hq, hk, True, [1] * 7, [1, 64, 65, 0, 777, 3000, 16])
    run(api, dtype, d, hq, hk, True, [1, 0, 1], [2000, 100, 1], slots=2048)
    run(api, dtype, d, hq, hk, True, [1], [1])


@pytest.mark.parametrize("causal", [True, False])
def test_few_tokens(api, causal):
    """Several new tokens whose rows still fit sixteen; fewer keys than tokens among them."""
    run(api, BF, 128, 4, 2, causal, [8, 3, 1, 0, 8, 5], [8, 700, 33, 20, 1900, 2])
    run(api, HALF, 64, 5, 1, causal, [3, 2, 3], [70, 2, 641], slots=700)
    run(api, BF, 64, 1, 1, causal, [16, 15], [16, 4000])


def test_many_splits(api):
    run(api, BF, 128, 2, 2, True, [1], [40000])
    run(api, HALF, 128, 12, 2, True, [40], [30000])


def test_scales_and_extreme_scores(api):
    run(api, BF, 128, 2, 2, True, [200], sm_scale=3.0)            # peaked rows: one probability near 1, the rest far below
    run(api, HALF, 64, 2, 2, False, [300], sm_scale=1e-6)         # flat rows
    run(api, HALF, 128, 2, 1, True, [1, 1], [900, 3], sm_scale=2.0)
    run(api, BF, 128, 2, 2, True, [257], mul=40.0)


@pytest.mark.parametrize("rows", [1, 300])
def test_strides(api, rows):
    """Slices of a fused projection, heads-first storage, outputs inside a larger tensor."""
    d, hq, hk, n = 128, 6, 2, rows
    m = max(n, 500)
    fused = randn((m, hq + 2 * hk, d), BF, 3)
    q, k, v = fused[:n, :hq], fused[:, hq:hq + hk], fused[:, hq + hk:]
    attn = api.PackedAttn(hq, hk, d, causal=True)
    cu, kr = i32([0, n]), (i32([0]), i32([m]))
    want, wl = attn.forward(q.contiguous(), k.contiguous(), v.contiguous(), cu, k_range=kr, max_q=n, max_k=m, want_lse=True)
    big = torch.full((n, 2 * hq + 1, d), 9.0, dtype=BF, device="cuda")
    got, gl = attn.forward(q, k, v, cu, k_range=kr, max_q=n, max_k=m, want_lse=True, o=big[:, ::2][:, :hq])
    assert torch.equal(got, want) and torch.equal(gl, wl) and (big[:, 1::2] == 9).all()
    heads_first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    got, _ = attn.forward(*heads_first, cu, k_range=kr, max_q=n, max_k=m)
    assert torch.equal(got, want)


@pytest.mark.parametrize("n", [1, 64])
def test_streams_capture_and_shared_handle(api, n):
    d, hq, hk, m = 64, 4, 2, 3000
    attn = api.PackedAttn(hq, hk, d, causal=True)
    q, k, v = randn((n, hq, d), BF, 1), randn((m, hk, d), BF, 2), randn((m, hk, d), BF, 3)
    cu, kb, ke = i32([0, n]), i32([0]), i32([m])
    call = lambda: attn.forward(q, k, v, cu, k_range=(kb, ke), max_q=n, max_k=m, want_lse=True)
    call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = call()
    here = call()                                        # both in flight: each call has a workspace of its own
    torch.cuda.synchronize()
    assert torch.equal(on_side[0], here[0]) and torch.equal(on_side[1], here[1])
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for length in (m, 1700, n):                          # lengths live on the device: a replay follows them
        ke.fill_(length)
        q.normal_()
        k.normal_()
        for graph, _ in graphs:
            graph.replay()
        want = call()
        for _, out in graphs:
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    attn.check_status()


def test_offsets_past_32_bits(api):
    """A cache whose last slots lie more than 2^32 bytes (and 2^31 elements) behind its first."""
    d, hk, n = 128, 8, 700
    total = (1 << 31) // (hk * d) + 5000
    k, v = (torch.empty(total, hk, d, dtype=BF, device="cuda") for _ in range(2))
    b = total - n
    for t, seed in ((k, 1), (v, 2)):
        t[b:] = randn((n, hk, d), BF, seed)
    for nq in (1, 150):
        q = randn((nq, 2 * hk, d), BF, 3)
        attn = api.PackedAttn(2 * hk, hk, d, causal=True)
        o, lse = attn.forward(q, k, v, i32([0, nq]), k_range=(i32([b]), i32([total])), max_q=nq, max_k=n, want_lse=True)
        want = reference(q, k[b:].contiguous(), v[b:].contiguous(), [0, nq], [0], [n], True, d ** -0.5)
        check(o, want["o"], want["o_tol"], "o")
        check(lse, want["lse"], want["lse_tol"], "lse")


@pytest.mark.parametrize("nq", [1, 200])
def test_ranges_outside_the_tensors_are_cut_and_reported(api, nq):
    d, h, m = 64, 2, 400
    attn = api.PackedAttn(h, h, d, causal=False)
    q, k, v = randn((nq, h, d), BF, 1), randn((m, h, d), BF, 2), randn((m, h, d), BF, 3)
    kw = dict(max_q=nq, max_k=m)
    good, _ = attn.forward(q, k, v, i32([0, nq]), k_range=(i32([0]), i32([m])), **kw)
    attn.check_status()
    for cu, b, e in (([0, nq], [0], [m + 50]), ([0, nq], [-9], [m]), ([0, nq], [300], [200]), ([0, nq + 3], [0], [m]),
                     ([0, -1], [0], [m]), ([-5, nq], [0], [m])):
        o, _ = attn.forward(q, k, v, i32(cu), k_range=(i32(b), i32(e)), **kw)
        assert attn.status() == api.TRA_ERR_INVALID_ARG
        assert attn.status() == api.TRA_OK
        if cu == [0, nq] and b[0] <= 0:
            assert torch.equal(o, good)
    attn.forward(q, k, v, i32([0, nq]), k_range=(i32([0]), i32([m])), max_q=nq, max_k=100)
    assert attn.status() == api.TRA_ERR_INVALID_ARG


def test_prefill_then_tokens_match_the_whole_prompt(api):
    """A prompt in chunks and then token by token over a growing cache gives the rows of the whole prompt."""
    d, hq, hk, n = 128, 6, 2, 300
    attn = api.PackedAttn(hq, hk, d, causal=True)
    q, k, v = randn((n, hq, d), BF, 1), randn((n, hk, d), BF, 2), randn((n, hk, d), BF, 3)
    whole, lse = attn.forward(q, k, v, i32([0, n]), max_q=n, max_k=n, want_lse=True)
    want = reference(q, k, v, [0, n], [0], [n], True, d ** -0.5)
    cache_k, cache_v = (torch.full((512, hk, d), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    at = 0
    for step in (100, 150, 30) + (1,) * 20:
        cache_k[at:at + step], cache_v[at:at + step] = k[at:at + step], v[at:at + step]
        o, l = attn.forward(q[at:at + step], cache_k, cache_v, i32([0, step]), k_range=(i32([0]), i32([at + step])),
                            max_q=step, max_k=512, want_lse=True)
        check(o, want["o"][at:at + step], want["o_tol"][at:at + step], f"o at {at}")
        check(l, want["lse"][at:at + step], want["lse_tol"][at:at + step], f"lse at {at}")
        at += step
    check(whole, want["o"], want["o_tol"], "o")
    attn.check_status()


def test_binding_refusals(api):
    d, n = 64, 40
    attn = api.PackedAttn(4, 2, d, causal=True)
    q, k, v = randn((n, 4, d), BF, 1), randn((n, 2, d), BF, 2), randn((n, 2, d), BF, 3)
    cu = i32([0, n])
    kw = dict(max_q=n, max_k=n)
    bad = [
        lambda: attn.forward(q.half(), k, v, cu, **kw), lambda: attn.forward(q.cpu(), k, v, cu, **kw),
        lambda: attn.forward(q, k, v[:-1], cu, **kw), lambda: attn.forward(k, k, v, cu, **kw),
        lambda: attn.forward(q[..., ::2], k, v, cu, **kw), lambda: attn.forward(q, k, v, cu.long(), **kw),
        lambda: attn.forward(q, k, v, cu[:1], **kw), lambda: attn.forward(q, k, v, cu, cu[:1], **kw),
        lambda: attn.forward(q, k, v, cu, cu, k_range=(cu[:1], cu[1:]), **kw),
        lambda: attn.forward(q, k, v, cu, lse=torch.empty(n, 4, device="cuda", dtype=torch.float64), **kw),
        lambda: attn.forward(q[0], k, v, cu, **kw), lambda: api.PackedAttn(4, 2, d, dtype=torch.float32),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: attn.forward(q, k, v, cu, max_q=n + 1, max_k=n), lambda: attn.forward(q, k, v, cu, max_q=n, max_k=n + 1),
                 lambda: attn.forward(q, k, v, cu, sm_scale=0.0, **kw), lambda: api.PackedAttn(4, 3, d), lambda: api.PackedAttn(4, 2, 80),
                 lambda: attn.forward(q, k[:, :1].expand(n, 2, d), v, cu, **kw)):      # a stride of zero
        with pytest.raises(api.TraError):
            call()
    o, lse = attn.forward(q, k, v, cu, want_lse=True, **kw)
    with pytest.raises(ValueError):
        attn.backward(q, q, k, v, o, None, cu, **kw)
    with pytest.raises(ValueError):
        attn.backward(q[:-1], q, k, v, o, lse, cu, **kw)
    attn.check_status()
    torch.cuda.synchronize()


def test_many_sequences(api):
    """More sequences than one search step reads, long ones among short and empty ones; keys shared by two sequences."""
    lens = [(7 * i) % 5 for i in range(1100)]
    lens[3], lens[600], lens[1099] = 700, 301, 260
    run(api, BF, 64, 2, 1, True, lens)
    lens = [0] * 40 + [300] + [0] * 33 + [1]
    run(api, HALF, 64, 1, 1, False, lens)
    d, n, m = 64, 90, 500
    attn = api.PackedAttn(2, 2, d, causal=True)
    q, k, v = randn((2 * n, 2, d), BF, 1), randn((m, 2, d), BF, 2), randn((m, 2, d), BF, 3)
    o, _ = attn.forward(q, k, v, i32([0, n, 2 * n]), k_range=(i32([0, 0]), i32([m, m - 77])), max_q=n, max_k=m)
    want = reference(q, k, v, [0, n, 2 * n], [0, 0], [m, m - 77], True, d ** -0.5)
    check(o, want["o"], want["o_tol"], "o")


@pytest.mark.parametrize("n", [1, 40])
def test_no_tokens(api, n):
    """No keys at all, no queries at all, neither."""
    d = 64
    attn = api.PackedAttn(2, 1, d, causal=True)
    q, none = randn((n, 2, d), BF, 1), torch.empty(0, 1, d, dtype=BF, device="cuda")
    o, lse = attn.forward(q, none, none, i32([0, n]), i32([0, 0]), max_q=n, max_k=0, want_lse=True)
    assert (o == 0).all() and (lse == -math.inf).all()
    dq, dk, dv = attn.backward(q, q, none, none, o, lse, i32([0, n]), i32([0, 0]), max_q=n, max_k=0)
    assert (dq == 0).all() and dk.shape == (0, 1, d)
    k, noq = randn((n, 1, d), BF, 2), torch.empty(0, 2, d, dtype=BF, device="cuda")
    o, lse = attn.forward(noq, k, k, i32([0, 0]), i32([0, n]), max_q=0, max_k=n, want_lse=True)
    assert o.shape == (0, 2, d)
    dq, dk, dv = attn.backward(noq, noq, k, k, o, lse, i32([0, 0]), i32([0, n]), max_q=0, max_k=n)
    assert (dk == 0).all() and (dv == 0).all()
    o, _ = attn.forward(noq, none, none, i32([0, 0]), max_q=0, max_k=0)
    attn.backward(noq, noq, none, none, o, lse, i32([0, 0]), max_q=0, max_k=0)
    attn.check_status()


def test_two_handles_and_streams_at_once(api):
    """Long launches of two handles on two streams, both taking over blocks: each gives what it gives alone."""
    d, n = 128, 3000
    a, b = api.PackedAttn(8, 2, d, causal=True), api.PackedAttn(4, 4, d, causal=False)
    qa, ka, va = randn((n, 8, d), BF, 1), randn((n, 2, d), BF, 2), randn((n, 2, d), BF, 3)
    qb, kb, vb = randn((n, 4, d), BF, 4), randn((n, 4, d), BF, 5), randn((n, 4, d), BF, 6)
    cu = i32([0, 1000, n])
    kw = dict(max_q=n, max_k=n, want_lse=True)
    wa, wb = a.forward(qa, ka, va, cu, **kw), b.forward(qb, kb, vb, cu, **kw)
    ga = a.backward(qa, qa, ka, va, *wa, cu, max_q=n, max_k=n)
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s):
            xa = a.forward(qa, ka, va, cu, **kw)
            ha = a.backward(qa, qa, ka, va, *xa, cu, max_q=n, max_k=n)
        with torch.cuda.stream(t):
            xb = b.forward(qb, kb, vb, cu, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(xa + xb + ha, wa + wb + ga))
