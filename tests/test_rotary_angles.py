"""Angles of the rotary calls over the whole range of frequencies and positions: the table of turns on the CPU, and rotated channels
on the GPU, against integer arithmetic of any length."""
import ctypes
import math
from fractions import Fraction

import pytest
import torch

from paper_2608_02504_b200 import build

build.build()
from paper_2608_02504_b200 import api  # noqa: E402

BITS = 400


def _arctan_inverse(n, one):
    total = term = one // n
    k = 1
    while term:
        term //= n * n
        k += 2
        total += -(term // k) if k % 4 == 3 else term // k
    return total


def _inverse_two_pi():
    one = 1 << (BITS + 32)
    pi = 4 * (4 * _arctan_inverse(5, one) - _arctan_inverse(239, one))      # Machin
    return Fraction((one << BITS) // (2 * pi), 1 << BITS)


TURNS_PER_RADIAN = _inverse_two_pi()
FREQUENCIES = [0.0, 1.0, -1.0, 10000.0 ** (-40 / 42), 1e-30, 5e-324, 1e-19, 2.0 ** -64, 0.75, 6.283185307179586, 256.0, 1e6,
               -1e6, 12345678.9, 1e12, 2.0 ** 53 + 2, 1e18, -1.2345678901234567e19, math.nextafter(2.0 ** 64, 0)]


class Handle(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int), ("n_axes", ctypes.c_int), ("halves", ctypes.c_int), ("norm", ctypes.c_int),
                ("eps", ctypes.c_float), ("turn", ctypes.c_uint64 * 128)]


def create(freq, d=64):
    freq = freq + [0.0] * (d // 2 - len(freq))
    cfg = api.tra_rotary_config_t()
    cfg.head_dim, cfg.n_axes = d, 1
    cfg.axis, cfg.inv_freq = (ctypes.c_int * len(freq))(*[0] * len(freq)), (ctypes.c_double * len(freq))(*freq)
    h = ctypes.c_void_p()
    return api._lib.tra_rotary_create(ctypes.byref(h), ctypes.byref(cfg)), h


def test_turns_of_a_position():
    """F_p: the frequency in turns modulo one, rounded once to 64 bits."""
    rc, h = create(FREQUENCIES)
    assert rc == api.TRA_OK
    turn = list(ctypes.cast(h, ctypes.POINTER(Handle)).contents.turn)
    for f, got in zip(FREQUENCIES, turn):
        exact = (Fraction(f) * TURNS_PER_RADIAN % 1) * 2 ** 64
        off = (got - exact + 2 ** 63) % 2 ** 64 - 2 ** 63
        assert abs(off) <= Fraction(1, 2) + Fraction(1, 2 ** 20), (f, got, float(off))
    assert api._lib.tra_rotary_destroy(h) == api.TRA_OK


@pytest.mark.parametrize("f", [2.0 ** 64, -2.0 ** 64, 1e20, 1e308])
def test_frequencies_past_the_range_are_refused(f):
    rc, h = create([1.0, f])
    assert rc == api.TRA_ERR_UNSUPPORTED and not h.value


@pytest.mark.gpu
def test_far_positions_and_high_frequencies():
    """fp32 rows: the pair (1, 0) turns to (cos, sin).  Off by the 64-bit table (2^-65 turn a position), the cut to 32 bits (2^-32 turn),
    its rounding to fp32 (2^-25 half turns) and sincospif's 2 ulp: below 2^-21 together."""
    freq = FREQUENCIES + [0.0] * (32 - len(FREQUENCIES))
    pos = [0, 1, -1, 1000003, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, 2 ** 30 + 12345, -987654321]
    rot = api.Rotary(64, axis=[0] * 32, inv_freq=freq)
    x = torch.zeros(1, len(pos), 1, 64, device="cuda")
    x[..., 0::2] = 1.0
    y, _, _ = rot.forward(x, pos=torch.tensor(pos, dtype=torch.int32, device="cuda")[:, None])
    y = y.cpu()[0, :, 0]
    for i, n in enumerate(pos):
        for p, f in enumerate(freq):
            turn = float((n * Fraction(f) * TURNS_PER_RADIAN + Fraction(1, 2)) % 1 - Fraction(1, 2))
            want = (math.cos(2 * math.pi * turn), math.sin(2 * math.pi * turn))
            assert abs(float(y[i, 2 * p]) - want[0]) <= 2.0 ** -21 and abs(float(y[i, 2 * p + 1]) - want[1]) <= 2.0 ** -21, (n, f)
    rot.close()
