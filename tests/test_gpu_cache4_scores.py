"""Scores over the 4-bit cache where queries or keys are very large, very small, or both in one row.  The bounds in norm are derived in
cache4_norms.py."""
import pytest
import torch

from tests.cache4_norms import attention, check_norm
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
