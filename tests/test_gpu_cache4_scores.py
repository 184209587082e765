"""Scores over the 4-bit cache where queries or keys are very large, very small, or both in one row.  The bounds in norm are derived in
cache4_norms.py."""
import pytest
import torch

from tests.cache4_norms import attention, check_norm
from tests.cache4_reference import values
from tests.packed_reference import randn
from tests.test_gpu_cache4_values import attend

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.mark.parametrize("nq", [1, 3, 70])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,log2", [(HALF, 7), (HALF, 10), (BF, 7), (BF, 11)])
def test_small_queries_meet_large_keys(api, dtype, log2, d, nq):
    """Groups of channels of equal weight in the scores, whose queries are 2^(2 log2) apart."""
    m, hq, hk = 300, 4, 2
    q, k, v = randn((nq, hq, d), dtype, 1, 1.5), randn((m, hk, d), dtype, 2), randn((m, hk, d), dtype, 3)
    q[..., :32] *= 2.0 ** log2
    k[..., :32] *= 2.0 ** -log2
    q[..., 32:64] *= 2.0 ** -log2
    k[..., 32:64] *= 2.0 ** log2
    check_norm(attend(api, q, k, v), attention(q, k, v, many=nq * hq // hk > 64), "o")


@pytest.mark.parametrize("nq", [1, 3, 70])
@pytest.mark.parametrize("q_size,k_size", [(1e-35, 1e35), (1e35, 1e-35), (1e-20, 1e20), (1e20, 1e-20)])
def test_queries_and_keys_at_the_ends_of_the_range(api, q_size, k_size, nq):
    m, hq, hk, d = 300, 4, 2, 64
    q, k, v = randn((nq, hq, d), BF, 1, 1.5 * q_size), randn((m, hk, d), BF, 2, k_size), randn((m, hk, d), BF, 3)
    check_norm(attend(api, q, k, v), attention(q, k, v, many=nq * hq // hk > 64), "o")


@pytest.mark.parametrize("nq", [1, 3])
def test_the_largest_queries(api, nq):
    """Scores of 0 beside ones of 2^130: the largest takes all."""
    m, d = 40, 64
    q = torch.full((nq, 2, d), 2.0 ** 126, dtype=BF, device="cuda")
    k, v = torch.zeros(m, 1, d, dtype=BF, device="cuda"), randn((m, 1, d), BF, 3)
    k[5], k[6] = 1.0, -1.0
    o = attend(api, q, k, v).double()
    want = values(v[5, 0])
    # P is 1: the result's rounding, and that of the middle and of the step in fp16
    assert ((o - want).abs() <= 2.0 ** -8 * want.abs() + 2 * 2.0 ** -11 * v.abs().max() * 2).all()


@pytest.mark.parametrize("nq", [1, 3, 70])
@pytest.mark.parametrize("size", [1e20, 1e36])
def test_large_keys_that_large_queries_do_not_meet(api, nq, size):
    """Queries in one group of channels, keys in the other: every score is 0, and o the mean of the values seen."""
    m, d = 200, 64
    q, k, v = randn((nq, 2, d), BF, 1, size), randn((m, 1, d), BF, 2, size), randn((m, 1, d), BF, 3)
    q[..., 32:], k[..., :32] = 0.0, 0.0
    check_norm(attend(api, q, k, v), attention(q, k, v, many=nq * 2 > 64), "o")
