"""Values that are not finite inside a sequence of the packed-attention calls: they reach exactly the rows whose scores they
enter, whichever kernel runs (few rows: one block, a cluster, a workspace; 128-row tiles, whole and split)."""
import math

import pytest
import torch

from tests.packed_reference import i32, randn

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, torch.float16
NAN = float("nan")
# at most 16 rows per key/value head go to the kernel for few rows; keys: one block, a cluster of eight, a workspace
ROWS = [1, 3, 16, 17, 300]
KEYS = [100, 1000, 40000]


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


def forward(attn, q, k, v):
    n, m = q.shape[0], k.shape[0]
    o, lse = attn.forward(q, k, v, i32([0, n]), i32([0, m]), max_q=n, max_k=m, want_lse=True)
    attn.check_status()
    return o, lse


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("m", KEYS)
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_query_of_nan(api, dtype, d, n, m):
    attn = api.PackedAttn(1, 1, d, dtype=dtype, causal=False)
    q, k, v = randn((n, 1, d), dtype, 1), randn((m, 1, d), dtype, 2), randn((m, 1, d), dtype, 3)
    clean, clean_lse = forward(attn, q, k, v)
    row = n // 2
    q[row, 0, 5] = NAN
    o, lse = forward(attn, q, k, v)
    assert o[row].isnan().all() and lse[row].isnan().all()
    others = torch.arange(n, device="cuda") != row
    assert torch.equal(o[others], clean[others]) and torch.equal(lse[others], clean_lse[others])


# which keys are NaN: one; the sixteen that one warp takes of every 64, in the first part or in all; all of them
SHARES = {"one": lambda j: j == 37, "a warp's": lambda j: (j % 64) // 16 == 1, "a warp's of the first tiles":
          lambda j: ((j % 64) // 16 == 1) & (j < 512), "all": lambda j: j >= 0}


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("m", KEYS)
@pytest.mark.parametrize("share", SHARES)
@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_keys_of_nan(api, dtype, d, n, m, share):
    attn = api.PackedAttn(1, 1, d, dtype=dtype, causal=False)
    q, k, v = randn((n, 1, d), dtype, 1), randn((m, 1, d), dtype, 2), randn((m, 1, d), dtype, 3)
    k[SHARES[share](torch.arange(m, device="cuda"))] = NAN
    o, lse = forward(attn, q, k, v)
    assert o.isnan().all() and lse.isnan().all()


@pytest.mark.parametrize("n", [4, 40])
@pytest.mark.parametrize("m", KEYS)
def test_hidden_key_of_nan(api, n, m):
    """Causal: a key's NaN stays with the queries that see it (its value is finite)."""
    d = 64
    attn = api.PackedAttn(2, 1, d, causal=True)
    q, k, v = randn((n, 2, d), BF, 1), randn((m, 1, d), BF, 2), randn((m, 1, d), BF, 3)
    clean, clean_lse = forward(attn, q, k, v)
    k[-2] = NAN                                         # seen by the last two queries
    o, lse = forward(attn, q, k, v)
    assert o[-2:].isnan().all() and lse[-2:].isnan().all()
    assert torch.equal(o[:-2], clean[:-2]) and torch.equal(lse[:-2], clean_lse[:-2])


@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("m", KEYS)
def test_infinite_scores(api, n, m):
    """A score of +inf has no softmax; keys whose scores are all -inf weigh nothing beside others, and a row of nothing but them is
    like one that sees no key."""
    d = 64
    attn = api.PackedAttn(1, 1, d, causal=False)
    q, k, v = randn((n, 1, d), BF, 1).abs(), randn((m, 1, d), BF, 2), randn((m, 1, d), BF, 3)
    up = k.clone()
    up[37, 0, 3] = math.inf
    o, lse = forward(attn, q, up, v)
    assert o.isnan().all() and lse.isnan().all()
    down = k.clone()
    j = torch.arange(m, device="cuda")
    hidden = (j % 64) // 16 == 1
    down[hidden, 0, 3] = -math.inf
    o, lse = forward(attn, q, down, v)
    want, want_lse = forward(attn, q, k[~hidden].contiguous(), v[~hidden].contiguous())
    # the same sums in another grouping: either is off by u |o| + u sum p |v - o| <= 3 u max |v|, u = 2^-8, and the sums of m terms
    # by m units 2^-24 at most
    assert (o - want).abs().max() <= 6.1 * 2.0 ** -8 * v.abs().max()
    assert (lse - want_lse).abs().max() <= 1e-3 + (m + 64) * 2.0 ** -23
    down[:, 0, 3] = -math.inf
    o, lse = forward(attn, q, down, v)
    assert (o == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype,d", [(BF, 128), (HALF, 64)])
def test_gradients_of_nan(api, dtype, d):
    """A NaN query, and a query whose dO is NaN: their own dq, the dk and dv of the keys they see, and nothing of another
    sequence."""
    lens, hq, hk = [150, 70], 4, 2
    n = sum(lens)
    attn = api.PackedAttn(hq, hk, d, dtype=dtype, causal=True)
    q, k, v, do = (randn((n, h, d), dtype, 1 + i) for i, h in enumerate((hq, hk, hk, hq)))
    cu = i32([0, 150, n])
    do[100] *= 0.5                                       # not the largest row

    def step():
        o, lse = attn.forward(q, k, v, cu, max_q=150, max_k=150, want_lse=True)
        return attn.backward(do, q, k, v, o, lse, cu, max_q=150, max_k=150)

    clean = step()
    for t in (q, do):
        keep = t[100].clone()
        t[100] = NAN
        dq, dk, dv = step()
        t[100] = keep
        rows = torch.arange(n, device="cuda") != 100
        assert dq[100].isnan().all() and torch.equal(dq[rows], clean[0][rows])
        assert dk[:101].isnan().all() and dv[:101].isnan().all()
        assert torch.equal(dk[150:], clean[1][150:]) and torch.equal(dv[150:], clean[2][150:])
    attn.check_status()
