"""A long stream through the operators that it uses together: rotary positions, the 4-bit cache, attention with a window over it, chunk by
chunk and token by token, eager and captured; and a training step of a layer with a window.  Against fp64."""
import math

import pytest
import torch

from tests.cache4_reference import attention, values
from tests.packed_reference import check, i32, packed, randn
from tests.window_reference import seen

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.mark.parametrize("dtype,d,hq,hk,window,sinks", [(BF, 128, 10, 2, 100, 4), (HALF, 64, 4, 4, 0, 0), (BF, 64, 6, 1, 64, 64), (HALF, 128, 8, 2, 37, 1)])
def test_two_streams_in_chunks_and_tokens(api, dtype, d, hq, hk, window, sinks):
    """Two sequences in slots of one cache, every step a chunk or a token of each (or of one of them)."""
    slots, steps = 512, [(200, 130), (0, 60), (33, 1), (7, 7)] + [(1, 1)] * 5 + [(1, 0), (0, 1), (90, 1)]
    lens = [sum(s[i] for s in steps) for i in range(2)]
    rot = api.Rotary(d, (d,), norm="rms")
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, window=window, sinks=sinks)
    cache = api.Cache4(attn, 2 * slots)
    cache.k_step.fill_(float("nan"))
    cache.v_step.fill_(float("nan"))
    raw = [[randn((n, h, d), dtype, 10 * s + i) for i, h in enumerate((hq, hk, hk))] for s, n in enumerate(lens)]
    weight = randn((d,), dtype, 7, 0.1) + 1
    whole = []                                               # what the cache was given and asked, sequence by sequence
    for s, n in enumerate(lens):
        pos = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous()
        q, k, v = rot.forward(*(t[None] for t in raw[s]), pos=pos, q_weight=weight, k_weight=weight)
        whole.append((q[0], k[0], v[0]))
    at = [0, 0]
    for step in steps:
        q, k, v, pos, where = [], [], [], [], []
        for s, n in enumerate(step):
            part = slice(at[s], at[s] + n)
            for t, x in zip((q, k, v), raw[s]):
                t.append(x[part])
            pos += list(range(at[s], at[s] + n))
            where += list(range(s * slots + at[s], s * slots + at[s] + n))
            at[s] += n
        q, k, v = (torch.cat(t)[None] for t in (q, k, v))
        q, k, v = rot.forward(q, k, v, pos=i32(pos)[:, None].contiguous(), q_weight=weight, k_weight=weight)
        cache.write(k[0], v[0], i32(where))
        o, lse = attn.forward_cache4(q[0], cache, i32(packed(step)), k_range=(i32([0, slots]), i32([at[0], slots + at[1]])), max_q=max(step), max_k=slots,
                                     want_lse=True)
        for s, n in enumerate(step):
            if n == 0:
                continue
            rows, now = slice(step[0] if s else 0, (step[0] if s else 0) + n), at[s]
            wq, wk, wv = whole[s]
            want = attention(wq[now - n:now], wk[:now], wv[:now], [0, n], [0], [now], window, sinks, d ** -0.5, max(step) * hq // hk > 64)
            check(o[rows], want["o"], want["o_tol"], f"o of {s} at {now}")
            check(lse[rows], want["lse"], want["lse_tol"], f"lse of {s} at {now}")
    attn.check_status()


@pytest.mark.parametrize("nq", [1, 40])
def test_captured_steps(api, nq):
    """rotary -> write -> attention captured twice, replayed while positions, slots and lengths move on the device; each graph has a
    workspace of its own.  Eager calls beside them on another stream give the same bits."""
    d, hq, hk, slots = 128, 8, 2, 9000
    rot = api.Rotary(d, (d,))
    attn = api.PackedAttn(hq, hk, d, window=5000, sinks=16)
    cache = api.Cache4(attn, slots)
    fill = torch.arange(slots, dtype=torch.int32, device="cuda")
    cache.write(randn((slots, hk, d), BF, 1), randn((slots, hk, d), BF, 2), fill)
    raw = [randn((1, nq, h, d), BF, 3 + i) for i, h in enumerate((hq, hk, hk))]
    pos, where, cu, begin, end = fill[:nq, None].clone(), fill[:nq].clone(), i32([0, nq]), i32([0]), i32([nq])

    def step():
        q, k, v = rot.forward(*raw, pos=pos)
        cache.write(k[0], v[0], where)
        return attn.forward_cache4(q[0], cache, cu, k_range=(begin, end), max_q=nq, max_k=slots, want_lse=True)
    step()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    side = torch.cuda.Stream()
    for now in (nq, 700, 8999):
        for t in raw:
            t.normal_()
        pos.copy_(torch.arange(now - nq, now, device="cuda")[:, None])
        where.copy_(pos[:, 0])
        end.fill_(now)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            q, k, v = rot.forward(*raw, pos=pos)
            there = attn.forward_cache4(q[0], cache, cu, k_range=(begin, end), max_q=nq, max_k=slots, want_lse=True)
        here = attn.forward_cache4(q[0], cache, cu, k_range=(begin, end), max_q=nq, max_k=slots, want_lse=True)
        torch.cuda.synchronize()
        for out in [there, here] + [o for _, o in graphs]:
            assert torch.equal(out[0], here[0]) and torch.equal(out[1], here[1])
    attn.check_status()


def test_caches_of_two_handles_at_once(api):
    d, n = 64, 3000
    a, b = api.PackedAttn(8, 2, d, window=700, sinks=3), api.PackedAttn(4, 4, d, dtype=HALF, causal=False)
    ca, cb = api.Cache4(a, n), api.Cache4(b, n)
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    ka, va, kb, vb = randn((n, 2, d), BF, 1), randn((n, 2, d), BF, 2), randn((n, 4, d), HALF, 3), randn((n, 4, d), HALF, 4)
    ca.write(ka, va, slots)
    cb.write(kb, vb, slots)
    qa, qb = randn((500, 8, d), BF, 5), randn((500, 4, d), HALF, 6)
    cu, kr = i32([0, 500]), (i32([0]), i32([n]))
    wa = a.forward_cache4(qa, ca, cu, k_range=kr, max_q=500, max_k=n)[0]
    wb = b.forward_cache4(qb, cb, cu, k_range=kr, max_q=500, max_k=n)[0]
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(4):
        with torch.cuda.stream(s):
            xa = a.forward_cache4(qa, ca, cu, k_range=kr, max_q=500, max_k=n)[0]
        with torch.cuda.stream(t):
            xb = b.forward_cache4(qb, cb, cu, k_range=kr, max_q=500, max_k=n)[0]
        torch.cuda.synchronize()
        assert torch.equal(xa, wa) and torch.equal(xb, wb)
    # another handle of the same heads, type and device takes the cache too
    other = api.PackedAttn(8, 2, d, window=700, sinks=3)
    assert torch.equal(other.forward_cache4(qa, ca, cu, k_range=kr, max_q=500, max_k=n)[0], wa)


def test_many_sequences_in_passes(api):
    """More keys than are read back at a time: the passes' sequences do not mix."""
    d, hk, n_seq, slots = 128, 8, 40, 16384
    attn = api.PackedAttn(8, hk, d)
    cache = api.Cache4(attn, n_seq * slots)
    lens_q, lens_k = [70 + s % 3 for s in range(n_seq)], [500 + 37 * s for s in range(n_seq)]
    k, v = [], []
    for s, m in enumerate(lens_k):
        k.append(randn((m, hk, d), BF, 2 * s))
        v.append(randn((m, hk, d), BF, 2 * s + 1))
        cache.write(k[-1], v[-1], torch.arange(s * slots, s * slots + m, dtype=torch.int32, device="cuda"))
    cu = packed(lens_q)
    q = randn((cu[-1], 8, d), BF, 99)
    begin = [s * slots for s in range(n_seq)]
    o, lse = attn.forward_cache4(q, cache, i32(cu), k_range=(i32(begin), i32([b + m for b, m in zip(begin, lens_k)])), max_q=max(lens_q), max_k=slots,
                                 want_lse=True)
    attn.check_status()
    for s in (0, 1, 3, 4, 17, 38, 39):
        rows = slice(cu[s], cu[s + 1])
        want = attention(q[rows], k[s], v[s], [0, lens_q[s]], [0], [lens_k[s]], 0, 0, d ** -0.5, True)
        check(o[rows], want["o"], want["o_tol"], f"o of {s}")
        check(lse[rows], want["lse"], want["lse_tol"], f"lse of {s}")


def test_training_step_of_a_layer_with_a_window(api):
    """Projection -> head norm and rotary positions -> attention with a window, and all gradients back, against fp64 differentiation of the
    definition."""
    d, hq, hk, lens, window, sinks = 64, 4, 2, [150, 333, 1], 60, 3
    cu, n = packed(lens), sum(lens)
    x = randn((1, n, hq + 2 * hk, d), BF, 1)
    wq, wk, do = randn((d,), BF, 2, 0.1) + 1, randn((d,), BF, 3, 0.1) + 1, randn((n, hq, d), BF, 4)
    pos = i32([p for m in lens for p in range(m)])[:, None].contiguous()
    rot, attn = api.Rotary(d, (d,), norm="rms"), api.PackedAttn(hq, hk, d, window=window, sinks=sinks)
    q, k, v = x.split([hq, hk, hk], 2)
    Q, K, V = rot.forward(q, k, v, pos=pos, q_weight=wq, k_weight=wk)
    kw = dict(max_q=max(lens), max_k=max(lens))
    o, lse = attn.forward(Q[0], K[0], V[0], i32(cu), want_lse=True, **kw)
    grads = attn.backward(do, Q[0], K[0], V[0], o, lse, i32(cu), **kw)
    (dq, dk, dv), gw = rot.backward(*(g[None] for g in grads), q=q, k=k, pos=pos, q_weight=wq, k_weight=wk)
    attn.check_status()

    leaves = [t.double().requires_grad_() for t in (q[0], k[0], v[0], wq, wk)]
    freq = 10000.0 ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
    turn = torch.polar(torch.ones(n, d // 2, device="cuda", dtype=torch.float64), pos.double() * freq)[:, None]

    def rotated(t, w):
        t = w * t / torch.sqrt((t * t).mean(-1, keepdim=True) + 1e-6)
        z = torch.view_as_complex(t.unflatten(-1, (-1, 2)).contiguous()) * turn
        return torch.view_as_real(z).flatten(-2)
    rq, rk, rv = rotated(leaves[0], leaves[3]), rotated(leaves[1], leaves[4]), leaves[2]
    outs = []
    for a, b in zip(cu[:-1], cu[1:]):
        kk, vv = (t[a:b].repeat_interleave(hq // hk, 1) for t in (rk, rv))
        s = torch.einsum("nhd,mhd->hnm", rq[a:b], kk) / math.sqrt(d)
        s = s.masked_fill(~seen(b - a, b - a, window, sinks, "cuda"), -math.inf)
        outs.append(torch.einsum("hnm,mhd->nhd", torch.softmax(s, -1), vv))
    want = torch.autograd.grad(torch.cat(outs), leaves, do.double())
    # Rounded to bf16 on the way (relative 2^-9 rms each at most): Q, K, P, dS, dq / dk, and the results; V and O take fewer.  Six of them,
    # through sums of independent errors, are 2^-9 sqrt(6) of the norm, twice that as the bound
    bound = 2 * math.sqrt(6) * 2.0 ** -9
    for name, got, ref in zip(("dq", "dk", "dv", "q_weight", "k_weight"), (dq[0], dk[0], dv[0], gw["q_weight"], gw["k_weight"]), want):
        assert float((got.double() - ref).norm() / ref.norm()) <= bound, name
