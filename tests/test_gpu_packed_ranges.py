"""Ranges on the device that the packed-attention calls have to report: longer than the stated maximum, also when that is zero, and
bounds that run backwards in the middle of many."""
import pytest
import torch

from tests.packed_reference import i32, randn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def tensors(n, m, d=64, heads=2):
    return randn((n, heads, d), BF, 1), randn((m, heads, d), BF, 2), randn((m, heads, d), BF, 3)


@pytest.mark.parametrize("max_q,max_k", [(0, 50), (0, 0)])
def test_maximum_of_zero(api, max_q, max_k):
    """Queries that a maximum of zero leaves out are reported; nothing is written."""
    attn = api.PackedAttn(2, 2, 64, causal=False)
    q, k, v = tensors(40, 50)
    cu, none = i32([0, 40]), i32([0, 0])
    o, lse = torch.full_like(q, 7.0), torch.full((40, 2), 5.0, device="cuda")
    attn.forward(q, k, v, cu, i32([0, max_k]), max_q=max_q, max_k=max_k, o=o, lse=lse)
    assert attn.status() == api.TRA_ERR_INVALID_ARG and attn.status() == api.TRA_OK
    assert (o == 7).all() and (lse == 5).all()
    attn.forward(q, k, v, none, i32([0, max_k]), max_q=max_q, max_k=max_k, o=o, lse=lse)
    attn.check_status()
    out = [torch.full_like(t, 9.0) for t in (q, k, v)]
    kw = dict(max_q=max_q, max_k=max_k, dq=out[0], dk=out[1], dv=out[2])
    attn.backward(q, q, k, v, o, lse, cu, i32([0, max_k]), **kw)
    assert attn.status() == api.TRA_ERR_INVALID_ARG
    assert (out[0] == 9).all()
    attn.backward(q, q, k, v, o, lse, none, i32([0, max_k]), **kw)
    attn.check_status()
    assert (out[0] == 9).all() and (out[1][max_k:] == 9).all() and (out[1][:max_k] == 0).all()


@pytest.mark.parametrize("keys,max_k", [([0, 0, 50], 0), ([0, 60], 50), ([0, 70], 50)])
def test_no_queries_but_ranges_of_keys(api, keys, max_k):
    """Without a query the keys' ranges are still looked at."""
    attn = api.PackedAttn(2, 2, 64, causal=True)
    q, k, v = tensors(0, 60)
    attn.forward(q, k, v, i32([0] * len(keys)), i32(keys), max_q=0, max_k=max_k)
    assert attn.status() == api.TRA_ERR_INVALID_ARG
    attn.forward(q, k, v, i32([0, 5]), i32([0, 60]), max_q=0, max_k=60)
    assert attn.status() == api.TRA_ERR_INVALID_ARG
    none = q[:0]
    attn.forward(none, none, none, i32([0, 1]), max_q=0, max_k=0)
    assert attn.status() == api.TRA_ERR_INVALID_ARG
    lse = torch.empty(0, 2, device="cuda")
    attn.backward(none, none, none, none, none, lse, i32([0, 1]), max_q=0, max_k=0)
    assert attn.status() == api.TRA_ERR_INVALID_ARG


def bounds(n_seq, step, at):
    """Ascending bounds, but the one behind sequence `at` lies in front of it."""
    cu = [i * step for i in range(n_seq + 1)]
    cu[at] += 4 * step
    return cu


@pytest.mark.parametrize("n_seq,at", [(3, 1), (3, 2), (40, 1), (40, 17), (40, 39), (1200, 700)])
@pytest.mark.parametrize("step", [30, 150])
@pytest.mark.parametrize("side", ["q", "k"])
def test_bounds_that_run_backwards(api, n_seq, at, step, side):
    total = (n_seq + 4) * step
    attn = api.PackedAttn(1, 1, 64, causal=False)
    q, k, v = tensors(total, total, heads=1)
    good, bad = i32([i * step for i in range(n_seq + 1)]), i32(bounds(n_seq, step, at))
    kw = dict(max_q=total, max_k=total)
    o, lse = attn.forward(q, k, v, good, want_lse=True, **kw)
    attn.check_status()
    cu_q, cu_k = (bad, good) if side == "q" else (good, bad)
    attn.forward(q, k, v, cu_q, cu_k, **kw)
    assert attn.status() == api.TRA_ERR_INVALID_ARG
    attn.backward(q, q, k, v, o, lse, cu_q, cu_k, **kw)
    assert attn.status() == api.TRA_ERR_INVALID_ARG
    attn.backward(q, q, k, v, o, lse, good, **kw)
    attn.check_status()
