"""Plain fp64 attention over packed sequences with the tolerances of the kernels' arithmetic, for the GPU tests.

Tolerance of O, per element.  u = eps / 2 of the type: one rounding of the result, u |o|, and one of every probability,
p (1 + d), |d| <= u, in numerator and denominator alike: u sum_j p_j |v_j - o|.  A probability is also off by the
relative error of its exponent: the fp32 product over d channels, (d + 8) 2^-23 of scale |q| |k| (tensor-core adds may
truncate: one unit 2^-23 each, and the scaling's and the subtraction's), and ex2, 2^-21 with the range of its argument.
The sums over n keys add n + 16 units 2^-23 of sum p |v|.  fp16 probabilities below 2^-14 lose up to 2^-25 each, of a
sum that is at least 1.  Splitting and joining adds a handful of 2^-23, inside the 16.
lse: the exponent's error, n + 64 units 2^-24 of the sum, and fp32 rounding of the result.

Gradients: P is off by e (the exponent's error plus that of lse), and rounded (u) before dV; dS = P (dP - delta) by
P times the error of dP and delta, (d + 8) 2^-23 |dO| |v| and the rounding of the O delta is made of, and is rounded
(u) before dQ and dK."""
import math

import torch

UNIT = 2.0 ** -23


def sequences(cu_q, k_begin, k_end):
    for s in range(len(k_begin)):
        yield s, cu_q[s], cu_q[s + 1], k_begin[s], k_end[s]


def reference(q, k, v, cu_q, k_begin, k_end, causal, scale, do=None, o_rest=False):
    """All tensors in fp64 on their device; returns a dict of fp64 results and tolerances (rows outside the sequences
    are zero with tolerance zero).  Lists on the host.  o_rest: delta is formed from O and the remainder of its
    rounding (off by u^2 |o|), and its other errors are bounded as they arise, u sum_j p_j |v_j - o|, not by the sums of
    magnitudes: small sequences only."""
    dtype = q.dtype
    u = torch.finfo(dtype).eps / 2
    fp16 = dtype == torch.float16
    tiny = float(torch.finfo(dtype).tiny)
    hq, hk, d = q.shape[1], k.shape[1], q.shape[2]
    g = hq // hk
    z = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)
    r = {"o": z(q), "o_tol": z(q), "lse": torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=q.device),
         "lse_tol": torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)}
    if do is not None:
        for n, t in (("dq", q), ("dk", k), ("dv", v)):
            r[n], r[n + "_tol"] = z(t), z(t)
    for _, q0, q1, k0, k1 in sequences(cu_q, k_begin, k_end):
        n, m = q1 - q0, k1 - k0
        if n == 0 or m == 0:
            continue
        for h in range(hk):
            Q = q[q0:q1, h * g:(h + 1) * g].double().transpose(0, 1)           # [g, n, d]
            K, V = k[k0:k1, h].double(), v[k0:k1, h].double()                  # [m, d]
            s = scale * (Q @ K.T)
            if causal:
                i = torch.arange(n, device=q.device)[:, None]
                j = torch.arange(m, device=q.device)[None]
                s = s.masked_fill(j > i + (m - n), -math.inf)
            lse = torch.logsumexp(s, -1)
            none = torch.isinf(lse)
            p = torch.exp(s - torch.where(none, torch.zeros_like(lse), lse)[..., None])
            o = p @ V
            smax = scale * Q.norm(dim=-1) * K.norm(dim=-1).max()               # [g, n]
            e = smax * (d + 8) * UNIT + 2.0 ** -21
            absv = p @ V.abs()
            spread = absv + o.abs()                                             # >= sum p |v - o|
            tol = u * o.abs() * (1 + 2 * u) + (u + e)[..., None] * spread * (1 + 4 * u) + (m + 16) * UNIT * absv + tiny
            if fp16:
                tol = tol + m * 2.0 ** -25 * V.abs().max()
            rows, heads = slice(q0, q1), slice(h * g, (h + 1) * g)
            r["o"][rows, heads], r["o_tol"][rows, heads] = o.transpose(0, 1), tol.transpose(0, 1)
            lse_tol = e + (m + 64) * UNIT / 2 + lse.abs().nan_to_num(posinf=0) * UNIT
            r["lse"][rows, heads] = lse.transpose(0, 1)
            r["lse_tol"][rows, heads] = torch.where(none, torch.zeros_like(lse), lse_tol).transpose(0, 1)
            if do is None:
                continue
            dO = do[rows, heads].double().transpose(0, 1)                       # [g, n, d]
            delta = (dO * o).sum(-1, keepdim=True)
            dP = dO @ V.T
            dS = p * (dP - delta)
            ep = (e + lse_tol)[..., None] + UNIT                                # relative error of P
            if o_rest:
                spread = (p[..., None] * (V[None, None] - o[:, :, None]).abs()).sum(-2)
                tol = (u + e)[..., None] * spread * (1 + 4 * u) + (m + 16) * UNIT * absv + 2 * u * u * o.abs() + tiny
                if fp16:
                    tol = tol + m * 2.0 ** -25 * V.abs().max()
            # error of dP - delta: products, and delta's: the rounding of O (u |o| and what came before it)
            size = dO.norm(dim=-1, keepdim=True)
            edp = (d + 8) * UNIT * size * V.norm(dim=-1).max() + (dO.abs() * tol).sum(-1, keepdim=True) \
                + (d + 8) * UNIT * (dO.abs() * o.abs()).sum(-1, keepdim=True)
            # per element of dS, before its own rounding
            eds = p * ep * (dP - delta).abs() + p * (1 + ep) * edp
            low = 2.0 ** -25 if fp16 else 0.0                                   # fp16 rounding of small numbers
            rds = u * (dS.abs() + eds) + low
            rp = (u * (1 + ep) + ep) * p + low
            total_rows = g * n
            r["dv"][k0:k1, h] = (p.transpose(1, 2) @ dO).sum(0)
            r["dv_tol"][k0:k1, h] = (rp.transpose(1, 2) @ dO.abs()).sum(0) + \
                (total_rows + 16) * UNIT * (p.transpose(1, 2) @ dO.abs()).sum(0)
            r["dk"][k0:k1, h] = scale * (dS.transpose(1, 2) @ Q).sum(0)
            r["dk_tol"][k0:k1, h] = scale * (((eds + rds).transpose(1, 2) @ Q.abs()).sum(0)
                                             + (total_rows + 16) * UNIT * (dS.abs().transpose(1, 2) @ Q.abs()).sum(0))
            r["dq"][rows, heads] = (scale * (dS @ K)).transpose(0, 1)
            r["dq_tol"][rows, heads] = (scale * ((eds + rds) @ K.abs() + (m + 16) * UNIT * (dS.abs() @ K.abs()))).transpose(0, 1)
    if do is not None:
        for n in ("dq", "dk", "dv"):
            r[n + "_tol"] += u * r[n].abs() * (1 + 2 * u) + u * r[n + "_tol"] + tiny
    return r


def check(got, want, tol, what):
    got = got.double()
    both_inf = torch.isinf(got) & torch.isinf(want) & (got == want)
    bad = ~(((got - want).abs() <= tol) | both_inf)
    if bad.any():
        i = tuple(int(x) for x in torch.nonzero(bad)[0])
        over = ((got - want).abs() / tol.clamp_min(1e-300))[bad].nan_to_num(nan=math.inf).max()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(over):.3g} times the tolerance; "
                             f"first at {i}: {float(got[i])} for {float(want[i])}, tolerance {float(tol[i])}")


def packed(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def randn(shape, dtype, seed, mul=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (mul * torch.randn(shape, generator=g, device="cuda")).to(dtype)
