"""Plain fp64 attention over packed sequences with a window and first tokens, for the GPU tests.  Arithmetic and tolerances are
those of packed_reference.py (the kernels differ in the keys that they walk, not in what they do with one)."""
import math

import torch

from tests.packed_reference import UNIT, sequences


def seen(n, m, window, sinks, device):
    """[n, m]: query i (position i + m - n) sees key j."""
    at = torch.arange(n, device=device)[:, None] + (m - n)
    j = torch.arange(m, device=device)[None]
    ok = j <= at
    return ok & ((j > at - window) | (j < sinks)) if window else ok


def reference(q, k, v, cu_q, k_begin, k_end, window, sinks, scale, do=None):
    """fp64 results and tolerances; k and v may be fp64 already.  Rows outside the sequences are zero with tolerance zero."""
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
        mask = seen(n, m, window, sinks, q.device)
        rows = slice(q0, q1)
        for h in range(hk):
            heads = slice(h * g, (h + 1) * g)
            Q = q[rows, heads].double().transpose(0, 1)                        # [g, n, d]
            K, V = k[k0:k1, h].double(), v[k0:k1, h].double()                  # [m, d]
            s = (scale * (Q @ K.T)).masked_fill(~mask, -math.inf)
            lse = torch.logsumexp(s, -1)
            none = torch.isinf(lse)
            p = torch.exp(s - torch.where(none, torch.zeros_like(lse), lse)[..., None])
            o = p @ V
            smax = scale * Q.norm(dim=-1) * K.norm(dim=-1).max()
            e = smax * (d + 8) * UNIT + 2.0 ** -21
            absv = p @ V.abs()
            tol = u * o.abs() * (1 + 2 * u) + (u + e)[..., None] * (absv + o.abs()) * (1 + 4 * u) + (m + 16) * UNIT * absv + tiny
            if fp16:
                tol = tol + m * 2.0 ** -25 * V.abs().max()
            r["o"][rows, heads], r["o_tol"][rows, heads] = o.transpose(0, 1), tol.transpose(0, 1)
            lse_tol = e + (m + 64) * UNIT / 2 + lse.abs().nan_to_num(posinf=0) * UNIT
            r["lse"][rows, heads] = lse.transpose(0, 1)
            r["lse_tol"][rows, heads] = torch.where(none, torch.zeros_like(lse), lse_tol).transpose(0, 1)
            if do is None:
                continue
            dO = do[rows, heads].double().transpose(0, 1)
            dP = dO @ V.T
            dS = p * (dP - (dO * o).sum(-1, keepdim=True))
            ep = (e + lse_tol)[..., None] + UNIT
            edp = (d + 8) * UNIT * dO.norm(dim=-1, keepdim=True) * V.norm(dim=-1).max() + (dO.abs() * tol).sum(-1, keepdim=True) \
                + (d + 8) * UNIT * (dO.abs() * o.abs()).sum(-1, keepdim=True)
            eds = dS.abs() * ep + p * (1 + ep) * edp
            low = 2.0 ** -25 if fp16 else 0.0
            rds = u * (dS.abs() + eds) + low
            rp = (u * (1 + ep) + ep) * p + low
            total = g * n
            r["dv"][k0:k1, h] = (p.transpose(1, 2) @ dO).sum(0)
            r["dv_tol"][k0:k1, h] = (rp.transpose(1, 2) @ dO.abs()).sum(0) + (total + 16) * UNIT * (p.transpose(1, 2) @ dO.abs()).sum(0)
            r["dk"][k0:k1, h] = scale * (dS.transpose(1, 2) @ Q).sum(0)
            r["dk_tol"][k0:k1, h] = scale * (((eds + rds).transpose(1, 2) @ Q.abs()).sum(0)
                                             + (total + 16) * UNIT * (dS.abs().transpose(1, 2) @ Q.abs()).sum(0))
            r["dq"][rows, heads] = (scale * (dS @ K)).transpose(0, 1)
            r["dq_tol"][rows, heads] = (scale * ((eds + rds) @ K.abs() + (m + 16) * UNIT * (dS.abs() @ K.abs()))).transpose(0, 1)
    if do is not None:
        for n in ("dq", "dk", "dv"):
            r[n + "_tol"] += u * r[n].abs() * (1 + 2 * u) + u * r[n + "_tol"] + tiny
    return r
