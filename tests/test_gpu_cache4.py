"""The cache of 4 bits (``tra_cache4_write``, ``_read``) and attention over it (``tra_packed_attn_cache4``) against plain fp64 forms; the
tolerances are derived in cache4_reference.py."""
import math

import pytest
import torch

from tests.cache4_reference import attention, values
from tests.packed_reference import check, i32, packed, randn

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def same(got, want_fp64):
    """Rounded once: exactly the type's nearest number (fp64 -> type in one step, by way of fp32 where that is exact enough: the
    values have 8 + 4 + 16 bits at most, so the conversion through fp32 may round twice only on ties)."""
    want = want_fp64.to(torch.float32).to(got.dtype)
    ulp = (want.view(torch.int16).int() - got.view(torch.int16).int()).abs()
    exact = torch.equal(torch.nan_to_num(got, nan=7.0), torch.nan_to_num(want, nan=7.0))
    return exact or bool(((got.double() - want_fp64).abs() <= torch.finfo(got.dtype).eps / 2 * want_fp64.abs() * (1 + 2 ** -10) + 2.0 ** -134).all()) and int(ulp.max()) <= 1


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("d,heads", [(128, 8), (64, 3), (128, 1), (64, 2)])
@pytest.mark.parametrize("n", [1, 7, 64, 333])
def test_write_and_read(api, dtype, d, heads, n):
    attn = api.PackedAttn(heads, heads, d, dtype=dtype)
    cache = api.Cache4(attn, 700)
    k, v = randn((n, heads, d), dtype, 1, 2.0), randn((n, heads, d), dtype, 2)
    k[:, :, 5] += 9.0                                         # a channel with an offset
    slots = torch.randperm(700, device="cuda")[:n].to(torch.int32)
    cache.write(k, v, slots)
    got = cache.read(slots)
    attn.check_status()
    for x, y in zip((k, v), got):
        assert same(y, values(x))
    back = torch.randperm(n, device="cuda")
    again = cache.read(slots[back])
    assert all(torch.equal(a[back], b) for a, b in zip(got, again))


def special(dtype, d, n=40):
    """Rows that are hard to quantise: constant groups, zeros, the type's largest and smallest numbers, exact halves of a step."""
    big, tiny = torch.finfo(dtype).max, float(torch.finfo(dtype).smallest_normal)
    x = torch.zeros(n, 1, d, dtype=dtype, device="cuda")
    x[1] = 3.0
    x[2] = -0.0
    x[3, 0, ::2], x[3, 0, 1::2] = big, -big
    x[4] = torch.linspace(-big, big, d, dtype=torch.float64, device="cuda").to(dtype)
    x[5] = torch.linspace(0, tiny, d, device="cuda").to(dtype)
    x[6, 0, 7] = tiny
    x[7] = (torch.arange(d, device="cuda") % 31 / 2).to(dtype)          # steps of 1, halves between
    x[8] = -(torch.arange(d, device="cuda") % 31 / 2).to(dtype)
    x[9] = (1000 + torch.arange(d, device="cuda") % 3).to(dtype)
    x[10, 0, :32], x[10, 0, 32:] = 1.0, 2.0 ** -20
    x[11:] = randn((n - 11, 1, d), dtype, 5, 1.0) * torch.exp(torch.linspace(-12, 8, n - 11, device="cuda"))[:, None, None].to(dtype)
    return x


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_hard_rows(api, dtype, d):
    x = special(dtype, d)
    n = x.shape[0]
    attn = api.PackedAttn(1, 1, d, dtype=dtype)
    cache = api.Cache4(attn, n)
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    cache.write(x, x.flip(0), slots)
    k, v = cache.read(slots)
    want = values(x)
    bound = float(torch.finfo(dtype).max)
    fits = want.abs() <= bound
    assert same(k[fits], want[fits]) and torch.equal(k, v.flip(0))
    assert (k[~fits].isinf() | (k[~fits].abs() == bound)).all()          # low + 15 step may pass the type's range


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_groups_that_are_not_finite_read_back_as_nan(api, dtype, d):
    attn = api.PackedAttn(1, 1, d, dtype=dtype)
    cache = api.Cache4(attn, 8)
    x = randn((4, 1, d), dtype, 3)
    y = x.clone()
    y[0, 0, 3], y[1, 0, d - 1], y[2, 0, 40] = float("nan"), float("inf"), float("-inf")
    slots = i32([0, 1, 2, 3])
    cache.write(y, y, slots)
    k, v = cache.read(slots)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[0, 0, :32] = bad[1, 0, d - 32:] = bad[2, 0, 32:64] = True
    assert k[bad].isnan().all() and v[bad].isnan().all()
    assert same(k[~bad], values(x)[~bad]) and same(v[~bad], values(x)[~bad])


@pytest.mark.parametrize("d", [64, 128])
def test_strides_and_slots_left_out(api, d):
    heads, n = 3, 50
    attn = api.PackedAttn(6, heads, d)
    cache = api.Cache4(attn, 101)
    assert cache.tokens == 102
    every = torch.arange(102, dtype=torch.int32, device="cuda")
    base = randn((102, heads, d), BF, 9)
    cache.write(base, base, every)
    fused = randn((n, 6 + 2 * heads, d), BF, 3)
    k, v = fused[:, 6:6 + heads], fused[:, 6 + heads:]
    slots = (torch.arange(n, device="cuda") * 2).to(torch.int32)
    slots[3] = slots[17] = -1
    cache.write(k, v, slots)
    want_k, want_v = base.clone(), base.clone()
    used = slots >= 0
    want_k[slots[used].long()], want_v[slots[used].long()] = k[used], v[used]
    out = torch.full((102, 2 * heads + 1, d), 9.0, dtype=BF, device="cuda")
    cache.read(every, out[:, 1:1 + heads], out[:, 1 + heads:])
    assert (out[:, 0] == 9).all() and same(out[:, 1:1 + heads], values(want_k)) and same(out[:, 1 + heads:], values(want_v))
    slots = i32([5, -3, 7])
    kk, vv = torch.full((3, heads, d), 4.0, dtype=BF, device="cuda"), torch.full((3, heads, d), 4.0, dtype=BF, device="cuda")
    cache.read(slots, kk, vv)
    assert (kk[1] == 4).all() and (vv[1] == 4).all() and torch.equal(kk[0], out[5, 1:1 + heads])
    attn.check_status()
    # past the cache: left out and reported, and nothing else is touched
    cache.write(k[:3], v[:3], i32([102, 1 << 30, 2]))
    assert attn.status() == api.TRA_ERR_INVALID_ARG and attn.status() == api.TRA_OK
    cache.read(i32([0, 102, 0]), kk, vv)
    assert attn.status() == api.TRA_ERR_INVALID_ARG and (kk[1] == 4).all()
    cache.write(k[:0], v[:0], slots[:0])
    attn.check_status()


def run(api, dtype, d, hq, hk, lens_q, lens_k, window=0, sinks=0, slots=None, seed=1, mul=1.5, causal=True):
    """Every row of the cache that belongs to no sequence holds NaN steps; O and lse hold a mark that has to stay around the sequences."""
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
    q = randn((total_q, hq, d), dtype, seed, mul)
    k, v = randn((total_k, hk, d), dtype, seed + 1), randn((total_k, hk, d), dtype, seed + 2)
    k[..., 3] += 4.0
    q[:cu[0]], q[cu[-1]:] = float("nan"), float("nan")
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, window=window, sinks=sinks, causal=causal)
    cache = api.Cache4(attn, total_k)
    cache.k_step.fill_(float("nan"))
    cache.v_step.fill_(float("nan"))
    for b, e in zip(kb, ke):
        cache.write(k[b:e], v[b:e], torch.arange(b, e, dtype=torch.int32, device="cuda"))
    want = attention(q, k, v, cu, kb, ke, window, sinks, d ** -0.5, max(lens_q) * hq // hk > 64, causal)
    kw = dict(k_range=(i32(kb), i32(ke)), max_q=max(lens_q), max_k=max(lens_k))
    o = torch.full((total_q, hq, d), 77.0, dtype=dtype, device="cuda")
    lse = torch.full((total_q, hq), 55.0, device="cuda")
    attn.forward_cache4(q, cache, i32(cu), o=o, lse=lse, **kw)
    attn.check_status()
    rows = slice(cu[0], cu[-1])
    check(lse[rows], want["lse"][rows], want["lse_tol"][rows], "lse")
    check(o[rows], want["o"][rows], want["o_tol"][rows], "o")
    for t, mark in ((o, 77.0), (lse, 55.0)):
        assert (t[:cu[0]] == mark).all() and (t[cu[-1]:] == mark).all()
    o2 = torch.full_like(o, 77.0)
    _, none = attn.forward_cache4(q, cache, i32(cu), o=o2, **kw)
    assert none is None and torch.equal(o, o2)
    return o[rows], want["o"][rows]


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64), (BF, 64), (HALF, 128)])
@pytest.mark.parametrize("hq,hk", [(1, 1), (12, 12), (10, 2), (16, 1), (5, 1)])
def test_one_token(api, dtype, d, hq, hk):
    run(api, dtype, d, hq, hk, [1] * 7, [1, 64, 65, 0, 777, 3000, 16])
    run(api, dtype, d, hq, hk, [1, 0, 1], [2000, 100, 1], slots=2048)
    run(api, dtype, d, hq, hk, [1], [1])


@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 64), (65, 3), (500, 7), (3000, 100), (200, 300)])
@pytest.mark.parametrize("dtype,d,hq,hk", [(BF, 128, 10, 2), (HALF, 64, 1, 1), (BF, 64, 16, 1), (HALF, 128, 4, 4)])
def test_one_token_with_a_window(api, dtype, d, hq, hk, window, sinks):
    run(api, dtype, d, hq, hk, [1] * 7, [1, 64, 65, 0, 777, 3000, 16], window, sinks)
    run(api, dtype, d, hq, hk, [1, 0, 1], [2000, 100, 1], window, sinks, slots=2048)
    run(api, dtype, d, hq, hk, [1], [9001], window, sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 1), (5, 0), (70, 66), (600, 2)])
def test_few_tokens(api, window, sinks):
    run(api, BF, 128, 4, 2, [8, 3, 1, 0, 8, 5], [8, 700, 33, 20, 1900, 2], window, sinks)
    run(api, HALF, 64, 5, 1, [3, 2, 3], [70, 2, 641], window, sinks, slots=700)
    run(api, BF, 64, 1, 1, [16, 15], [16, 4000], window, sinks)
    run(api, HALF, 128, 6, 2, [10, 3, 20], [400, 33, 1000], window, sinks)          # more than one tile of rows
    run(api, BF, 128, 2, 1, [32, 1], [130, 700], window, sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 5), (700, 130), (300, 256)])
@pytest.mark.parametrize("dtype,d,hq,hk", [(BF, 128, 10, 2), (HALF, 64, 3, 1), (BF, 64, 4, 4), (HALF, 128, 8, 1)])
def test_chunks(api, dtype, d, hq, hk, window, sinks):
    """More than 64 rows per key/value head: keys and values read back in two pieces."""
    run(api, dtype, d, hq, hk, [100, 40, 60, 300, 20, 0, 1], [1000, 40, 25, 301, 0, 50, 1300], window, sinks)
    run(api, dtype, d, hq, hk, [97], [5000], window, sinks)
    run(api, dtype, d, hq, hk, [130, 77], [2000, 131], window, sinks, slots=2048)


def test_chunks_that_are_not_causal(api):
    run(api, BF, 128, 4, 2, [100, 1, 70], [300, 1000, 12], causal=False)
    run(api, HALF, 64, 4, 2, [100, 1, 70], [300, 1000, 12], causal=False)
    run(api, BF, 64, 4, 2, [3, 1], [300, 1000], causal=False)


def test_groups(api):
    for group in (1, 3, 7, 16, 43, 100, 128):
        run(api, BF, 64, group, 1, [70, 9, 2], [90, 700, 1030], 200, 9)
        run(api, HALF, 128, 2 * group, 2, [1, 1], [700, 33])


@pytest.mark.parametrize("nq", [1, 3])
def test_many_sequences(api, nq):
    run(api, BF, 64, 4, 2, [nq * (i % 3 > 0) for i in range(1100)], [(7 * i) % 97 + 3 for i in range(1100)])
    run(api, HALF, 128, 2, 1, [nq] * 400, [(37 * i) % 700 for i in range(400)], 90, 5)


def test_many_splits(api):
    run(api, BF, 128, 2, 2, [1], [40000])
    run(api, HALF, 64, 12, 2, [8], [30001])


def test_extreme_scores(api):
    run(api, BF, 128, 2, 2, [1, 1], [900, 3], mul=40.0)
    run(api, HALF, 64, 2, 1, [4], [700], mul=1e-3)
    run(api, BF, 64, 2, 1, [4], [700], mul=1e-30)
"""A row's largest element may be anything: its power of two is taken out."""


@pytest.mark.parametrize("k_size,v_size", [(1e-6, 1e-5), (30.0, 1e4), (1e-3, 3e-2)])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
@pytest.mark.parametrize("nq", [1, 70])
def test_sizes_of_keys_and_values(api, dtype, d, k_size, v_size, nq):
    """Values far from 1, and rows of very different sizes in one cache: what is small is off by 2^-22 of what is large, per key."""
    n, hq, hk = 600, 4, 2
    q = randn((nq, hq, d), dtype, 1) * torch.exp2(-torch.arange(nq, device="cuda") % 9).to(dtype)[:, None, None]
    k, v = randn((n, hk, d), dtype, 2, k_size), randn((n, hk, d), dtype, 3, v_size)
    v[300:] *= 2.0 ** -6
    attn = api.PackedAttn(hq, hk, d, dtype=dtype)
    cache = api.Cache4(attn, n)
    cache.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
    o, lse = attn.forward_cache4(q, cache, i32([0, nq]), k_range=(i32([0]), i32([n])), max_q=nq, max_k=n, want_lse=True)
    want = attention(q, k, v, [0, nq], [0], [n], 0, 0, d ** -0.5, nq > 32)
    check(lse, want["lse"], want["lse_tol"], "lse")
    check(o, want["o"], want["o_tol"], "o")


def test_nan_reaches_the_rows_that_see_it(api):
    d, n = 64, 300
    attn = api.PackedAttn(2, 1, d)
    cache = api.Cache4(attn, n)
    k, v = randn((n, 1, d), BF, 1), randn((n, 1, d), BF, 2)
    v[100, 0, 40] = float("nan")
    cache.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
    q = randn((1, 2, d), BF, 3)
    o, _ = attn.forward_cache4(q, cache, i32([0, 1]), k_range=(i32([0]), i32([n])), max_q=1, max_k=n)
    assert o[..., 32:].isnan().all() and o[..., :32].isfinite().all()
    k[100, 0, 0] = float("nan")
    cache.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
    o, lse = attn.forward_cache4(q, cache, i32([0, 1]), k_range=(i32([0]), i32([n])), max_q=1, max_k=n, want_lse=True)
    assert o.isnan().all() and lse.isnan().all()
    o, lse = attn.forward_cache4(q, cache, i32([0, 1]), k_range=(i32([101]), i32([n])), max_q=1, max_k=n, want_lse=True)
    assert o.isfinite().all() and lse.isfinite().all()
    q[0, 0, 3] = float("nan")
    o, lse = attn.forward_cache4(q, cache, i32([0, 1]), k_range=(i32([101]), i32([n])), max_q=1, max_k=n, want_lse=True)
    assert o[0, 0].isnan().all() and lse[0, 0].isnan() and o[0, 1].isfinite().all()


def test_nan_in_chunks(api):
    """More rows than the kernel for few takes: a NaN reaches the rows that see it, and nobody where no range holds it."""
    d, n, nq = 64, 300, 100
    for dtype in (BF, HALF):
        attn = api.PackedAttn(2, 1, d, dtype=dtype)
        cache = api.Cache4(attn, n)
        k, v = randn((n, 1, d), dtype, 1), randn((n, 1, d), dtype, 2)
        good = attn.forward_cache4
        k[250, 0, 0] = float("nan")
        cache.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
        q = randn((nq, 2, d), dtype, 3)
        o, lse = good(q, cache, i32([0, nq]), k_range=(i32([0]), i32([n])), max_q=nq, max_k=n, want_lse=True)
        first = 250 - (n - nq)                                # the first query that sees key 250
        assert o[first:].isnan().all() and lse[first:].isnan().all() and o[:first].isfinite().all()
        o, lse = good(q, cache, i32([0, nq]), k_range=(i32([0]), i32([250])), max_q=nq, max_k=n, want_lse=True)
        assert o.isfinite().all() and lse.isfinite().all()
        q[5, 1, 3] = float("nan")
        o, lse = good(q, cache, i32([0, nq]), k_range=(i32([0]), i32([250])), max_q=nq, max_k=n, want_lse=True)
        assert o[5, 1].isnan().all() and o[5, 0].isfinite().all() and o[6:].isfinite().all()


def test_offsets_past_32_bits(api):
    """Heads whose rows lie more than 2^32 bytes behind the first's."""
    d, hk, n = 128, 8, 700
    total = (1 << 32) // (d // 2) // (hk - 1) + 2000
    total += total % 2
    attn = api.PackedAttn(2 * hk, hk, d)
    cache = api.Cache4(attn, total)
    k, v = randn((n, hk, d), BF, 1), randn((n, hk, d), BF, 2)
    b = total - n
    slots = torch.arange(b, total, dtype=torch.int32, device="cuda")
    cache.write(k, v, slots)
    got = cache.read(slots)
    assert same(got[0], values(k)) and same(got[1], values(v))
    q = randn((1, 2 * hk, d), BF, 3)
    o, _ = attn.forward_cache4(q, cache, i32([0, 1]), k_range=(i32([b]), i32([total])), max_q=1, max_k=n)
    want = attention(q, k, v, [0, 1], [0], [n], 0, 0, d ** -0.5)
    check(o, want["o"], want["o_tol"], "o")


@pytest.mark.parametrize("n", [1, 200])
def test_ranges_outside_the_cache_are_cut_and_reported(api, n):
    d, h, m = 64, 2, 400
    attn = api.PackedAttn(h, h, d, causal=False)
    cache = api.Cache4(attn, m)
    cache.write(randn((m, h, d), BF, 1), randn((m, h, d), BF, 2), torch.arange(m, dtype=torch.int32, device="cuda"))
    q = randn((n, h, d), BF, 3)
    kw = dict(max_q=n, max_k=m)
    good, _ = attn.forward_cache4(q, cache, i32([0, n]), k_range=(i32([0]), i32([m])), **kw)
    attn.check_status()
    for cu, b, e in (([0, n], [0], [m + 50]), ([0, n], [-9], [m]), ([0, n], [300], [200]), ([0, n + 3], [0], [m]), ([-5, n], [0], [m])):
        o, _ = attn.forward_cache4(q, cache, i32(cu), k_range=(i32(b), i32(e)), **kw)
        assert attn.status() == api.TRA_ERR_INVALID_ARG and attn.status() == api.TRA_OK
        if cu == [0, n] and b[0] <= 0:
            assert torch.equal(o, good)


def test_no_tokens(api):
    d = 64
    attn = api.PackedAttn(2, 1, d)
    for tokens in (0, 10):
        cache = api.Cache4(attn, tokens)
        for n in (1, 70):
            q = randn((n, 2, d), BF, 1)
            o, lse = attn.forward_cache4(q, cache, i32([0, n]), k_range=(i32([0]), i32([0])), max_q=n, max_k=0, want_lse=True)
            assert (o == 0).all() and (lse == -math.inf).all()
            o, lse = attn.forward_cache4(q[:0], cache, i32([0, 0]), k_range=(i32([0]), i32([tokens])), max_q=0, max_k=tokens, want_lse=True)
            assert o.shape == (0, 2, d)
    attn.check_status()


def test_refusals(api):
    d, n = 64, 40
    attn = api.PackedAttn(4, 2, d)
    cache = api.Cache4(attn, n)
    k, q = randn((n, 2, d), BF, 1), randn((n, 4, d), BF, 2)
    slots, cu = torch.arange(n, dtype=torch.int32, device="cuda"), i32([0, n])
    kr, kw = (i32([0]), i32([n])), dict(max_q=n, max_k=n)
    for call in (lambda: cache.write(k.half(), k, slots), lambda: cache.write(k, k[:-1], slots), lambda: cache.write(k, k, slots.long()),
                 lambda: cache.write(k.cpu(), k, slots), lambda: cache.write(k[..., ::2], k, slots), lambda: cache.write(k[0], k, slots),
                 lambda: cache.read(slots.cpu()), lambda: cache.read(slots, k=k[1:]), lambda: cache.read(slots, k=k[1:], v=k), lambda: api.Cache4(attn, -1),
                 lambda: attn.forward_cache4(q.half(), cache, cu, k_range=kr, **kw), lambda: attn.forward_cache4(q, cache, cu, k_range=None, **kw),
                 lambda: attn.forward_cache4(q, cache, cu, k_range=(kr[0].long(), kr[1]), **kw),
                 lambda: api.PackedAttn(4, 4, d).forward_cache4(q, cache, cu, k_range=kr, **kw),
                 lambda: api.PackedAttn(4, 2, d, dtype=HALF).forward_cache4(q.half(), cache, cu, k_range=kr, **kw)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: attn.forward_cache4(q, cache, cu, k_range=kr, max_q=n + 1, max_k=n),
                 lambda: attn.forward_cache4(q, cache, cu, k_range=kr, max_q=n, max_k=n + 1),
                 lambda: attn.forward_cache4(q, cache, cu, k_range=kr, sm_scale=-1.0, **kw),
                 lambda: cache.write(k[:, :1].expand(n, 2, d), k, slots)):
        with pytest.raises(api.TraError):
            call()
    torch.cuda.synchronize()
    attn.check_status()


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("nq", [1, 12, 100])
def test_strided_queries_and_outputs(api, dtype, nq):
    """Queries as a slice of a fused projection or stored heads first, outputs inside a larger tensor: the bits of the contiguous call."""
    d, hq, hk, m = 128, 6, 2, 700
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, window=300, sinks=5)
    cache = api.Cache4(attn, m)
    cache.write(randn((m, hk, d), dtype, 1), randn((m, hk, d), dtype, 2), torch.arange(m, dtype=torch.int32, device="cuda"))
    fused = randn((nq, hq + 2 * hk, d), dtype, 3)
    q, cu = fused[:, :hq], i32([0, nq])
    kw = dict(k_range=(i32([0]), i32([m])), max_q=nq, max_k=m, want_lse=True)
    want = attn.forward_cache4(q.contiguous(), cache, cu, **kw)
    big = torch.full((nq, 2 * hq + 1, d), 9.0, dtype=dtype, device="cuda")
    got = attn.forward_cache4(q, cache, cu, o=big[:, ::2][:, :hq], **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (big[:, 1::2] == 9).all()
    got = attn.forward_cache4(q.transpose(0, 1).contiguous().transpose(0, 1), cache, cu, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("nq", [1, 90])
def test_scales_and_shared_keys(api, nq):
    """Scales far from the usual one; two sequences that share their first keys, whose ranges overlap."""
    d, hq, hk, m = 64, 4, 2, 500
    for dtype, scale in ((BF, 3.0), (HALF, 1e-6), (HALF, 0.5)):
        attn = api.PackedAttn(hq, hk, d, dtype=dtype)
        cache = api.Cache4(attn, m)
        k, v = randn((m, hk, d), dtype, 1), randn((m, hk, d), dtype, 2)
        cache.write(k, v, torch.arange(m, dtype=torch.int32, device="cuda"))
        q = randn((2 * nq, hq, d), dtype, 3)
        kb, ke = [0, 0], [m, m - 77]
        o, lse = attn.forward_cache4(q, cache, i32([0, nq, 2 * nq]), k_range=(i32(kb), i32(ke)), max_q=nq, max_k=m, sm_scale=scale, want_lse=True)
        want = attention(q, k, v, [0, nq, 2 * nq], kb, ke, 0, 0, scale, nq > 32)
        check(o, want["o"], want["o_tol"], "o")
        check(lse, want["lse"], want["lse_tol"], "lse")
        attn.check_status()


@pytest.mark.parametrize("q_size,k_size,scale", [(0.0, 0.0, None), (0.0, 1e-8, None), (1e-30, 1e-12, None), (0.0, 1.0, 1e-30), (1e-25, 0.0, 1e-25)])
@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("nq,window", [(1, 0), (9, 0), (9, 40), (100, 0), (100, 40)])
def test_scores_of_zero_and_next_to_it(api, dtype, nq, window, q_size, k_size, scale):
    """Queries or keys of zeros (a padded row, a cache that is still empty) leave every row the mean of the values it sees."""
    n, d = 300, 64
    q = randn((nq, 2, d), dtype, 1) * q_size
    k, v = randn((n, 1, d), dtype, 2) * k_size, randn((n, 1, d), dtype, 3)
    attn = api.PackedAttn(2, 1, d, dtype=dtype, window=window)
    cache = api.Cache4(attn, n)
    cache.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"))
    o, lse = attn.forward_cache4(q, cache, i32([0, nq]), k_range=(i32([0]), i32([n])), max_q=nq, max_k=n, want_lse=True, sm_scale=scale)
    attn.check_status()
    want = attention(q, k, v, [0, nq], [0], [n], window, 0, d ** -0.5 if scale is None else scale, 2 * nq > 64, True)
    check(lse, want["lse"], want["lse_tol"], "lse")
    check(o, want["o"], want["o_tol"], "o")


@pytest.mark.parametrize("dtype", [BF, HALF])
def test_a_last_pass_of_fewer_sequences(api, dtype):
    """What is read back at a time holds some of the sequences; the ones that are left are fewer, and their launch takes more parts."""
    m, nq, d = 200000, 70, 64
    n_seq = 11 if dtype is BF else 6
    k, v = randn((m, 1, d), dtype, 1), randn((m, 1, d), dtype, 2)
    q = randn((n_seq * nq, 1, d), dtype, 3)
    attn = api.PackedAttn(1, 1, d, dtype=dtype)
    cache = api.Cache4(attn, m)
    cache.write(k, v, torch.arange(m, dtype=torch.int32, device="cuda"))
    begin, end = [7 * s for s in range(n_seq)], [m - 31 * s for s in range(n_seq)]
    cu = [nq * s for s in range(n_seq + 1)]
    o, lse = attn.forward_cache4(q, cache, i32(cu), k_range=(i32(begin), i32(end)), max_q=nq, max_k=m, want_lse=True)
    attn.check_status()
    for s in (0, n_seq - 2, n_seq - 1):
        rows = slice(cu[s], cu[s + 1])
        want = attention(q[rows], k, v, [0, nq], [begin[s]], [end[s]], 0, 0, d ** -0.5, True, True)
        check(lse[rows], want["lse"], want["lse_tol"], f"lse of {s}")
        check(o[rows], want["o"], want["o_tol"], f"o of {s}")
