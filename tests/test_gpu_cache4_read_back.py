"""Groups that span the whole range of the type: what is read back stays finite."""
import pytest
import torch

from tests.cache4_reference import values

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("d", [64, 128])
def test_finite_rows_read_back_finite(api, dtype, d):
    """low + 15 step may pass the largest number by what the step was rounded up: it is read back as that number."""
    n, most = 60, torch.finfo(dtype).max
    x = torch.rand(n, 1, d, device="cuda", generator=torch.Generator("cuda").manual_seed(1)) * 2 - 1
    x = (x.double() * torch.linspace(0.9, 1.0, n, device="cuda", dtype=torch.float64)[:, None, None] * most).to(dtype)
    x[0, 0, ::2], x[0, 0, 1::2] = most, -most
    x[1, 0], x[1, 0, 5] = 0.0, most
    x[2:, 0, 3], x[2:, 0, 40] = most, -most
    attn = api.PackedAttn(1, 1, d, dtype=dtype)
    cache = api.Cache4(attn, n)
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    cache.write(x, x.flip(0), slots)
    k, v = cache.read(slots)
    want = values(x)
    assert (want > most).any()
    assert k.isfinite().all() and torch.equal(k, v.flip(0))
    want = want.clamp(-most, most)
    assert ((k.double() - want).abs() <= torch.finfo(dtype).eps / 2 * want.abs() * (1 + 2.0 ** -10)).all()
    bad = x.clone()
    bad[4, 0, 7], bad[5, 0, 8], bad[6, 0, 9] = float("nan"), float("inf"), float("-inf")
    cache.write(bad, bad, slots)
    for y in cache.read(slots):
        assert y[4:7, 0, :32].isnan().all() and int(y.isnan().sum()) == 3 * 32
