"""Groups that span the whole range of the type: attention over them stays finite."""
import pytest
import torch

from tests.cache4_norms import attention, check_norm
from tests.cache4_reference import attention as elements, values
from tests.packed_reference import check, i32, randn
from tests.test_gpu_cache4_values import attend

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.mark.parametrize("m", [1, 3, 40])
@pytest.mark.parametrize("nq", [1, 2, 70])
@pytest.mark.parametrize("dtype", [BF, HALF])
def test_values_of_the_whole_range(api, dtype, nq, m):
    """One key takes all: o is its values, rounded, within 2^-11 of the largest for the roundings of the middle and of the step, or of the multiple."""
    d = 64
    most = torch.finfo(dtype).max
    x = torch.rand(m, 1, d, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 2 - 1
    v = (x.double() * 0.96 * most).to(dtype)
    v[:, 0, 3], v[:, 0, 40] = 0.96 * most, -0.96 * most
    q, k = torch.full((nq, 1, d), 8.0, dtype=dtype, device="cuda"), torch.full((m, 1, d), -8.0, dtype=dtype, device="cuda")
    k[0] = 8.0
    attn = api.PackedAttn(64 if nq > 2 else 1, 1, d, dtype=dtype, causal=False)
    q = q.expand(nq, attn.heads, d).contiguous()
    cache = api.Cache4(attn, m)
    cache.write(k, v, torch.arange(m, dtype=torch.int32, device="cuda"))
    o, _ = attn.forward_cache4(q, cache, i32([0, nq]), k_range=(i32([0]), i32([m])), max_q=nq, max_k=m)
    attn.check_status()
    want = values(v[0, 0])
    assert o.isfinite().all()
    assert ((o.double() - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() * (1 + 2.0 ** -8) + 2 * 2.0 ** -11 * most).all()


def test_many_rows_of_values_past_the_largest_number(api):
    """low + 15 step of a group next to the type's range, 1.4 % above the largest number: its multiple has to be one of fp16 as well."""
    nq, d = 70, 64
    most = torch.finfo(BF).max
    v = torch.zeros(2, 1, d, dtype=BF, device="cuda")
    v[0, 0, ::2], v[0, 0, 1::2] = most, -most * (1 - 26 * 2.0 ** -8)
    q, k = torch.zeros(nq, 1, d, dtype=BF, device="cuda"), torch.zeros(2, 1, d, dtype=BF, device="cuda")
    o = attend(api, q, k, v, causal=False)
    want = values(v).mean(0)
    assert values(v).max() > 1.01 * most
    assert ((o.double() - want).abs() <= (2.0 ** -9 + 2.0 ** -11) * want.abs() * (1 + 2.0 ** -8)).all()


@pytest.mark.parametrize("nq,window,sinks", [(1, 0, 0), (3, 0, 0), (3, 100, 5), (70, 0, 0)])
@pytest.mark.parametrize("m", [300, 20000])
@pytest.mark.parametrize("size", [2e37, 1e30, 1e-30])
def test_sums_of_large_and_small_values(api, size, m, nq, window, sinks):
    """Sums over many keys, in clusters and in parts, of values whose sum is past fp32's largest number, or next to its smallest."""
    d, hq, hk = 64, 4, 2
    q, k, v = randn((nq, hq, d), BF, 1), randn((m, hk, d), BF, 2), randn((m, hk, d), BF, 3, size)
    attn = api.PackedAttn(hq, hk, d, window=window, sinks=sinks)
    cache = api.Cache4(attn, m)
    cache.write(k, v, torch.arange(m, dtype=torch.int32, device="cuda"))
    o, lse = attn.forward_cache4(q, cache, i32([0, nq]), k_range=(i32([0]), i32([m])), max_q=nq, max_k=m, want_lse=True)
    attn.check_status()
    many = nq * hq // hk > 64
    check_norm(o, attention(q, k, v, window, sinks, many=many, terms=128), "o")
    want = elements(q, k, v, [0, nq], [0], [m], window, sinks, d ** -0.5, many)
    check(lse, want["lse"], want["lse_tol"], "lse")
