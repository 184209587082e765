"""Attention over long 4-bit caches against bounds in norm (cache4_norms.py), which lost parts, lost bits of long sums and results of zeros do not pass.
Values have an offset per head and channel and a drift along the keys, so that results are of their size."""
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


def drifting(m, hk, d, dtype, seed):
    along = torch.linspace(-1, 1, m, device="cuda")[:, None, None]
    return (randn((m, hk, d), torch.float32, seed) + randn((hk, d), torch.float32, seed + 1, 2.0) + along * randn((hk, d), torch.float32, seed + 2, 2.0)).to(dtype)


@pytest.mark.parametrize("dtype,d,hq,hk,nq,m,window,sinks", [
    (BF, 128, 2, 2, 1, 40000, 0, 0), (HALF, 64, 12, 2, 8, 30001, 0, 0), (HALF, 128, 10, 2, 1, 9001, 0, 0), (BF, 64, 4, 4, 3, 20000, 0, 0),
    (HALF, 128, 2, 1, 1, 65500, 30000, 100), (BF, 64, 16, 1, 1, 9001, 3000, 7),
    (BF, 128, 4, 2, 97, 40000, 0, 0), (HALF, 64, 2, 1, 100, 30001, 0, 0), (BF, 64, 6, 1, 130, 30001, 9000, 33), (HALF, 128, 4, 2, 70, 20000, 9000, 130)])
def test_one_sequence(api, dtype, d, hq, hk, nq, m, window, sinks):
    q, k, v = randn((nq, hq, d), dtype, 1), randn((m, hk, d), dtype, 2), drifting(m, hk, d, dtype, 3)
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, window=window, sinks=sinks)
    cache = api.Cache4(attn, m)
    cache.write(k, v, torch.arange(m, dtype=torch.int32, device="cuda"))
    o, _ = attn.forward_cache4(q, cache, i32([0, nq]), k_range=(i32([0]), i32([m])), max_q=nq, max_k=m)
    attn.check_status()
    # (few sequences are split into as many parts as fill the GPU: at most about 1,000 keys a part here, and 64 additions of 16 keys)
    check_norm(o, attention(q, k, v, window, sinks, many=nq * hq // hk > 64, terms=128), "o")


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("nq", [1, 70])
def test_many_sequences(api, dtype, nq):
    """Ranges of one cache that overlap; read back in passes, the last of fewer sequences."""
    m, d = 200000, 64
    n_seq = 40 if nq == 1 else 11 if dtype is BF else 6
    k, v = randn((m, 1, d), dtype, 1), drifting(m, 1, d, dtype, 2)
    q = randn((n_seq * nq, 1, d), dtype, 5)
    attn = api.PackedAttn(1, 1, d, dtype=dtype)
    cache = api.Cache4(attn, m)
    cache.write(k, v, torch.arange(m, dtype=torch.int32, device="cuda"))
    begin, end = [700 * s for s in range(n_seq)], [m - 3100 * s for s in range(n_seq)]
    cu = [nq * s for s in range(n_seq + 1)]
    o, _ = attn.forward_cache4(q, cache, i32(cu), k_range=(i32(begin), i32(end)), max_q=nq, max_k=m)
    attn.check_status()
    for s in (0, 1, n_seq - 2, n_seq - 1):
        rows = slice(cu[s], cu[s + 1])
        # parts of up to 22,000 keys; an addition per 16 keys (fp16 pieces: two), in the few rows' kernel two per 64
        terms = 22000 // (64 if nq == 1 else 16) * 2
        check_norm(o[rows], attention(q[rows], k[begin[s]:end[s]], v[begin[s]:end[s]], many=nq > 64, terms=terms), f"o of {s}")
