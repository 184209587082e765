"""Plain fp64 form of the 4-bit cache, and attention over it with the tolerances of the kernels' arithmetic, for the GPU tests.

What codes stand for is exact: low + step n has no rounding in fp64.  Attention, per element of O, u = eps / 2 of the tensors' type and
h = 2^-11 of fp16, in which the products over codes run:
  - the result's rounding, u |o|;
  - probabilities rounded to fp16 in numerator and denominator alike, h sum p |v - o|, and once more times the step of every group,
    h sum p step n; both at most 2 h sum p (|low| + 15 step) and h |o|;
  - the exponent: the scores are sums over the codes and over the lowest values, fp32 behind exact products, d + 8 additions of one unit
    2^-23 of scale |q| |(|low| + 15 step)| each (norms over the channels), 8 more where the two sums and the row's factor meet; ex2, 2^-21;
  - fp16 numbers below 2^-14: steps and lowest values are off by 2^-24 of the largest of them, top = max (|low|, 16 step) times 2; probabilities, held
    times 2^13 and at most 2^2 above the reference, by 2^-25 in sums that are at least 2^11: less than 2^-22 top per key;
  - sums over n keys: n + 16 units 2^-23 of sum p (|low| + 15 step).
Calls of more than 64 rows per key/value head (`pieces`) round probabilities to fp16, h sum p |v - o|, and 2^-25 per key of the largest value
below 2^-14; keys and values are in fp16 two numbers each, off by h^2 of an element, in bf16 one number of fp16, off by h of an element and by
2^-39 of the largest (multiples below 2^15, subnormal steps of 2^-24); probabilities are then up to 2^8, so that 2^-25 is 2^-33 of what they may be.
lse: as in packed_reference.py."""
import math

import torch

from tests.packed_reference import UNIT, sequences
from tests.window_reference import seen

GROUP = 32


def quantise(x):
    """x [..., d] of a 16-bit type -> (codes, step, low) in fp64, by the definition."""
    f = x.double().unflatten(-1, (-1, GROUP))
    low, high = f.amin(-1, keepdim=True), f.amax(-1, keepdim=True)
    step = ((high - low) / 15).to(x.dtype)
    # the smallest number of the type that covers the range: the nearest one or a neighbour
    for _ in range(2):
        step = torch.where(15 * step.double() < high - low, (step.view(torch.int16) + 1).view(x.dtype), step)
    below = (step.view(torch.int16) - 1).view(x.dtype)
    step = torch.where((step > 0) & (15 * below.double() >= high - low), below, step).double()
    codes = torch.floor(torch.where(step > 0, (f - low) / step, 0.0) + 0.5)
    return codes, step, low


def values(x):
    """What the cache holds of x, in fp64."""
    codes, step, low = quantise(x)
    return (low + step * codes).flatten(-2)


def sizes(x):
    """|low| + 15 step of every channel's group, and the largest of |low| and 16 step."""
    _, step, low = quantise(x)
    each = (low.abs() + 15 * step).expand(*step.shape[:-1], GROUP).flatten(-2)
    return each, float(torch.maximum(low.abs(), 16 * step).max()) if x.numel() else 0.0


def attention(q, k, v, cu_q, k_begin, k_end, window, sinks, scale, pieces=False, causal=True):
    """k, v: the 16-bit tensors that were written.  -> dict of o, lse and tolerances."""
    u = torch.finfo(q.dtype).eps / 2
    h = 2.0 ** -11
    tiny = float(torch.finfo(q.dtype).tiny)
    hq, hk, d = q.shape[1], k.shape[1], q.shape[2]
    g = hq // hk
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=q.device)
    r = {"o": z(*q.shape), "o_tol": z(*q.shape), "lse": z(*q.shape[:2]) - math.inf, "lse_tol": z(*q.shape[:2])}
    for _, q0, q1, k0, k1 in sequences(cu_q, k_begin, k_end):
        n, m = q1 - q0, k1 - k0
        if n == 0 or m == 0:
            continue
        mask = seen(n, m, window, sinks, q.device) if causal else torch.ones(n, m, dtype=torch.bool, device=q.device)
        for i in range(hk):
            rows, heads = slice(q0, q1), slice(i * g, (i + 1) * g)
            Q = q[rows, heads].double().transpose(0, 1)
            K, V = values(k[k0:k1, i]), values(v[k0:k1, i])
            (Ks, _), (Vs, top) = sizes(k[k0:k1, i]), sizes(v[k0:k1, i])
            s = (scale * (Q @ K.T)).masked_fill(~mask, -math.inf)
            lse = torch.logsumexp(s, -1)
            none = torch.isinf(lse)
            p = torch.exp(s - torch.where(none, torch.zeros_like(lse), lse)[..., None])
            o, size = p @ V, p @ Vs
            e = scale * Q.norm(dim=-1) * Ks.norm(dim=-1).max() * (d + 16) * UNIT + 2.0 ** -21
            tol = u * o.abs() * (1 + 2 * u) + h * o.abs() + (2 * h + e)[..., None] * size * (1 + 4 * h) + e[..., None] * o.abs() \
                + (m + 16) * UNIT * size + (2.0 ** -23 + m * 2.0 ** -22) * top * (p.sum(-1, keepdim=True) > 0) + tiny
            if pieces:
                off = 2 * h * h if q.dtype == torch.float16 else h
                e = e + scale * Q.norm(dim=-1) * (K.norm(dim=-1).max() * off + 2.0 ** -39 * d ** 0.5 * sizes(k[k0:k1, i])[1])
                absv = p @ V.abs()
                tol = u * o.abs() * (1 + 2 * u) + (h + e)[..., None] * (absv + o.abs()) * (1 + 4 * h) + off * absv + (m + 16) * UNIT * absv + tiny \
                    + (m * 2.0 ** -25 * V.abs().max() + 2.0 ** -39 * top) * (p.sum(-1, keepdim=True) > 0)
            r["o"][rows, heads], r["o_tol"][rows, heads] = o.transpose(0, 1), tol.transpose(0, 1)
            # (the exponent's error, as above)
            lse_tol = e + (m + 64) * UNIT / 2 + lse.abs().nan_to_num(posinf=0) * UNIT
            r["lse"][rows, heads] = lse.transpose(0, 1)
            r["lse_tol"][rows, heads] = torch.where(none, torch.zeros_like(lse), lse_tol).transpose(0, 1)
    return r
