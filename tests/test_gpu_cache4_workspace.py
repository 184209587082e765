"""Workspaces of attention over the 4-bit cache that start on 16 bytes and no more, through the C entry point: the same bits as from an allocation's
start, and nothing written around them."""
import ctypes

import pytest
import torch

from tests.packed_reference import i32, randn

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.mark.parametrize("offset", [16, 32, 48, 240])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64), (BF, 64), (HALF, 128)])
@pytest.mark.parametrize("nq,m,n_seq", [(70, 500, 2), (100, 20001, 1), (1, 40001, 1)])
def test_a_workspace_that_starts_on_16_bytes(api, nq, m, n_seq, dtype, d, offset):
    hq, hk = 2, 1
    attn = api.PackedAttn(hq, hk, d, dtype=dtype)
    cache = api.Cache4(attn, m)
    cache.write(randn((m, hk, d), dtype, 1), randn((m, hk, d), dtype, 2), torch.arange(m, dtype=torch.int32, device="cuda"))
    q, cu = randn((n_seq * nq, hq, d), dtype, 3), i32([nq * s for s in range(n_seq + 1)])
    begin, end = i32([3 * s for s in range(n_seq)]), i32([m - s for s in range(n_seq)])
    want, want_lse = attn.forward_cache4(q, cache, cu, k_range=(begin, end), max_q=nq, max_k=m, want_lse=True)
    size = api._lib.tra_packed_attn_cache4_workspace_bytes(attn._h, n_seq, q.shape[0], nq, m)
    assert size > 0
    room = torch.full((size + 512,), 171, dtype=torch.uint8, device="cuda")
    assert room.data_ptr() % 256 == 0
    o, lse = torch.empty_like(q), torch.empty_like(want_lse)
    a = attn._args(q, None, None, o, lse, None, cu, None, (begin, end), nq, m, None, cached=cache.tokens)
    call = lambda at, n: api._lib.tra_packed_attn_cache4(attn._h, a, cache._desc(), room.data_ptr() + at, n, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert call(8, size) == api.TRA_ERR_INVALID_ARG and call(offset, size - 1) == api.TRA_ERR_CAPACITY
    assert call(offset, size) == api.TRA_OK
    attn.check_status()
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    assert (room[:offset] == 171).all() and (room[offset + size:] == 171).all()
