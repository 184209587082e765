"""Attention over the 4-bit cache with the size of its rounding errors in norm, for the GPU tests.

The bounds of cache4_reference.py add every rounding of every key up, which no sum of thousands of keys comes near: there an o of zeros
would pass over long caches.  Roundings of different keys are independent, so their squares add up.  Here every rounding counts with its largest
size, half a step, which is sqrt(3) times the root of the mean square of one that is spread evenly: that is the room of the bound
|got - o| <= |rounding| + |sums|, in the Euclidean norm over the tokens and channels of a group of 32 and a head.

h = 2^-11 of fp16, u of the tensors' type, P^ = P over the row's largest (references are at most 2^2 behind it and probabilities held times 2^13, so that half of
the smallest fp16 number is 2^-38 of it; rounded to 0, a number is off by itself at most).  One element of o, few rows:
  - its rounding, u |o|, or half of the type's smallest number;
  - per key: P for its product with the middles, max (h P, 2^-38) |mid|; the middle, max (h |mid|, 2^-38 top) P, held below 2^15 when the largest
    are below 2 top; P times the step, max (h P step, 2^-40 top) |code - 8| (steps held times 8 in the same scale);
  - per key: the exponent, P |v - o| times d + 16 additions of one unit 2^-23 of scale sum |q| (|low| + 15 step), and 2^-21 of ex2.
Many rows: P in numerator and denominator, max (h P, 2^-25) |v - o| (of at most 2^8); the values' fp16 multiples in bf16, max (h |v|, 2^-38 top) P; the
exponent, in bf16 with the keys' multiples, which are off by max (h |k|, 2^-38 of the largest) and by |k| at most.  fp16 values in two pieces are off by h^2.
The sums themselves (`sums`): `terms` additions, one unit 2^-23 each of what is summed, which need not average out."""
import math

import torch

from tests.cache4_reference import GROUP, quantise, sizes, values
from tests.packed_reference import UNIT
from tests.window_reference import seen

H = 2.0 ** -11


def attention(q, k, v, window=0, sinks=0, scale=None, many=False, terms=None):
    """One sequence: q [n, hq, d], k, v [m, hk, d] of a 16-bit type -> dict of o, `rounding` and `sums`, all [n, hq, d]."""
    n, hq, d = q.shape
    m, hk = k.shape[:2]
    g, scale = hq // hk, d ** -0.5 if scale is None else scale
    u, least = torch.finfo(q.dtype).eps / 2, float(torch.finfo(q.dtype).smallest_normal) * torch.finfo(q.dtype).eps / 2
    terms = (m + 63) // 64 * 2 + 16 if terms is None else terms
    mask = seen(n, m, window, sinks, q.device)
    r = {name: torch.zeros(n, hq, d, dtype=torch.float64, device=q.device) for name in ("o", "rounding", "sums")}
    for i in range(hk):
        heads = slice(i * g, (i + 1) * g)
        Q, K, V = q[:, heads].double().transpose(0, 1), values(k[:, i]), values(v[:, i])
        codes, step, low = quantise(v[:, i])
        (Ks, k_top), (Vs, top) = sizes(k[:, i]), sizes(v[:, i])
        s = (scale * (Q @ K.T)).masked_fill(~mask, -math.inf)
        p = torch.softmax(s, -1)
        most = p.amax(-1, keepdim=True)
        o = p @ V
        e = scale * (Q.abs() @ Ks.T) * (d + 16) * UNIT + 2.0 ** -21
        if many and q.dtype == torch.bfloat16:
            off = torch.minimum(torch.clamp_min(H * K.abs(), 2.0 ** -38 * k_top), K.abs())
            e = (e ** 2 + scale ** 2 * (Q ** 2 @ (off ** 2).T)).sqrt()
        flat = lambda x: x.expand(m, d // GROUP, GROUP).flatten(-2)
        around = lambda w: w @ V ** 2 - 2 * o * (w @ V) + o ** 2 * w.sum(-1, keepdim=True)       # sum of w (v - o)^2
        square = torch.clamp_min(u * o.abs(), least) ** 2 + around((p * e) ** 2)
        if many:
            square += around(torch.minimum(torch.maximum(H * p, 2.0 ** -25 * most), p) ** 2)
            off = torch.clamp_min(H * V.abs(), 2.0 ** -38 * top) if q.dtype == torch.bfloat16 else H * H * V.abs() + least
            square += p ** 2 @ off ** 2
        else:
            mid, dev = flat(low + 8 * step), flat(codes - 8)
            square += torch.minimum(torch.maximum(H * p, 2.0 ** -38 * most), p) ** 2 @ mid ** 2
            square += p ** 2 @ torch.clamp_min(H * mid.abs(), 2.0 ** -38 * top) ** 2
            square += (H * p) ** 2 @ (flat(step) * dev) ** 2
            for j in range(d // GROUP):                      # of a group: steps differ from group to group
                tiny = torch.minimum(2.0 ** -40 * top * most, p * step[:, j, 0])
                square[..., j * GROUP:(j + 1) * GROUP] += tiny ** 2 @ dev[:, j * GROUP:(j + 1) * GROUP] ** 2
        r["o"][:, heads], r["rounding"][:, heads] = o.transpose(0, 1), square.clamp_min(0).sqrt().transpose(0, 1)
        r["sums"][:, heads] = (terms * UNIT * (p @ (Vs + flat(8 * step)))).transpose(0, 1)
    return r


def check_norm(got, want, what, rows=slice(None)):
    """Errors in norm per head and group of channels; and a bound that zeros would not pass."""
    norm = lambda x: x[rows].unflatten(-1, (-1, GROUP)).pow(2).sum((0, 3)).sqrt()
    off, room, size = norm(got.double() - want["o"]), norm(want["rounding"]) + norm(want["sums"]), norm(want["o"])
    assert (size > 4 * room).all(), f"{what}: the bound is {float((room / size).max()):.3g} of the result"
    assert (off <= room).all(), f"{what}: {float((off / room).nan_to_num(nan=math.inf).max()):.3g} times the bound; off by " \
                                f"{float((off / size).nan_to_num(nan=math.inf).max()):.3g} of the result"
