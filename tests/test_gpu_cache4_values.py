"""Attention over the 4-bit cache where values differ much in size: groups of channels far below others, and a large value that no query weights or
that the order hides from them.  The bounds in norm are derived in cache4_norms.py."""
import pytest
import torch

from tests.cache4_norms import attention, check_norm
from tests.packed_reference import i32, randn

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def attend(api, q, k, v, causal=True):
    (n, hq, d), (m, hk) = q.shape, k.shape[:2]
    attn = api.PackedAttn(hq, hk, d, dtype=q.dtype, causal=causal)
    cache = api.Cache4(attn, m)
    cache.write(k, v, torch.arange(m, dtype=torch.int32, device="cuda"))
    o, _ = attn.forward_cache4(q, cache, i32([0, n]), k_range=(i32([0]), i32([m])), max_q=n, max_k=m)
    attn.check_status()
    return o


@pytest.mark.parametrize("nq", [1, 3, 70])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,log2", [(HALF, -8), (HALF, -12), (HALF, -16), (BF, -8), (BF, -14), (BF, -20)])
def test_groups_of_different_sizes(api, dtype, log2, d, nq):
    m, hq, hk = 300, 4, 2
    q, k, v = randn((nq, hq, d), dtype, 1, 1.5), randn((m, hk, d), dtype, 2), randn((m, hk, d), dtype, 3)
    v[..., 32:64] *= 2.0 ** log2
    v[..., 96:] *= 2.0 ** (log2 // 2)
    check_norm(attend(api, q, k, v), attention(q, k, v, many=nq * hq // hk > 64), "o")


@pytest.mark.parametrize("m", [30, 300])
@pytest.mark.parametrize("nq", [1, 4, 70])
@pytest.mark.parametrize("dtype,size,large", [(HALF, 0.01, 6e4), (BF, 1.0, 2.0 ** 26)])
def test_a_large_value_without_weight(api, dtype, size, large, nq, m):
    d, hq, hk = 64, 4, 2
    nq = min(nq, m)
    q, k, v = randn((nq, hq, d), dtype, 1), randn((m, hk, d), dtype, 2), randn((m, hk, d), dtype, 3, size)
    q[..., 0], k[..., 0] = 8.0, 0.0
    at = m // 2 if nq < 70 else 0
    k[at, :, 0] = -120.0                                     # a score of -120
    v[at] = randn((hk, d), dtype, 4, large / 4).clamp(-large, large)
    check_norm(attend(api, q, k, v), attention(q, k, v, many=nq * hq // hk > 64), "o")


@pytest.mark.parametrize("dtype,size,large", [(HALF, 0.01, 6e4), (BF, 1.0, 2.0 ** 26)])
@pytest.mark.parametrize("nq,m", [(4, 30), (4, 300), (70, 300)])
def test_a_large_value_that_the_order_hides(api, dtype, size, large, nq, m):
    d, hq, hk = 128, 4, 2
    q, k, v = randn((nq, hq, d), dtype, 1), randn((m, hk, d), dtype, 2), randn((m, hk, d), dtype, 3, size)
    v[-1] = randn((hk, d), dtype, 4, large / 4).clamp(-large, large)
    check_norm(attend(api, q, k, v), attention(q, k, v, many=nq * hq // hk > 64), "o", slice(0, nq - 1))
