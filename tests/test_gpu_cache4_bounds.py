"""Bounds that callers of attention over the 4-bit cache hand over."""
import pytest
import torch

from tests.packed_reference import i32, randn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.mark.parametrize("nq", [1, 70])
def test_bounds_past_every_cache_are_refused(api, nq):
    d, m = 64, 40
    attn = api.PackedAttn(2, 1, d)
    cache = api.Cache4(attn, m)
    q = randn((nq, 2, d), BF, 1)
    for max_k in (m + 1, 1 << 28, 1 << 30, (1 << 30) + 1, 2_000_000_000, 2 ** 31 - 1):
        with pytest.raises(api.TraError):
            attn.forward_cache4(q, cache, i32([0, nq]), k_range=(i32([0]), i32([m])), max_q=nq, max_k=max_k)
    attn.check_status()
