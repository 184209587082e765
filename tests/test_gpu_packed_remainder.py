"""What rounding took from o (``o_rest``): passed explicitly, kept beside an lse that the call made, refused where it no longer
belongs to the lse, left out on request."""
import copy
import io

import pytest
import torch

from tests.packed_reference import i32, randn

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def api():
    from paper_2608_02504_b200 import api as a
    return a


@pytest.fixture()
def case(api):
    d, hq, hk, cu = 64, 4, 2, [0, 2, 5, 130]
    q, k, v, do = (randn((cu[-1], h, d), BF, 1 + i, 2.0 if i == 0 else 1.0) for i, h in enumerate((hq, hk, hk, hq)))
    return api.PackedAttn(hq, hk, d), (q, k, v), do, i32(cu), dict(max_q=125, max_k=125)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_explicit_remainder(case):
    attn, qkv, do, cu, kw = case
    o, lse = attn.forward(*qkv, cu, want_lse=True, **kw)
    kept = attn.backward(do, *qkv, o, lse, cu, **kw)
    rest = torch.empty_like(o)
    o2, own = attn.forward(*qkv, cu, lse=torch.empty_like(lse), o_rest=rest, **kw)
    assert torch.equal(o, o2) and torch.equal(lse, own) and torch.equal(rest, lse.o_rest)
    # an lse that was copied, cut or stored has no remainder beside it: it is passed
    plain = own.clone()
    assert same(kept, attn.backward(do, *qkv, o, plain, cu, o_rest=rest, **kw))
    without = attn.backward(do, *qkv, o, plain, cu, **kw)
    assert not same(kept, without)
    assert same(without, attn.backward(do, *qkv, o, lse, cu, o_rest=False, **kw))
    # made here, but given away by name
    rest2 = torch.empty_like(o)
    _, lse2 = attn.forward(*qkv, cu, want_lse=True, o_rest=rest2, **kw)
    assert torch.equal(rest2, rest) and lse2.o_rest is rest2


def test_no_remainder_on_request(case):
    attn, qkv, do, cu, kw = case
    o, lse = attn.forward(*qkv, cu, want_lse=True, **kw)
    o2, plain = attn.forward(*qkv, cu, want_lse=True, o_rest=False, **kw)
    assert getattr(plain, "o_rest", None) is None and torch.equal(o, o2) and torch.equal(lse, plain)
    # an lse used again without one drops the one that was there
    attn.forward(*qkv, cu, lse=lse, o_rest=False, **kw)
    assert getattr(lse, "o_rest", None) is None
    assert same(attn.backward(do, *qkv, o, lse, cu, **kw), attn.backward(do, *qkv, o, plain, cu, **kw))


def test_stale_remainder_is_refused(case):
    attn, (q, k, v), do, cu, kw = case
    o, lse = attn.forward(q, k, v, cu, want_lse=True, **kw)
    o2, lse2 = attn.forward(q * 0.5, k, v, cu, want_lse=True, **kw)
    want = attn.backward(do, q * 0.5, k, v, o2, lse2, cu, **kw)
    lse.copy_(lse2)                                     # another call's lse beside this call's remainder
    with pytest.raises(ValueError):
        attn.backward(do, q * 0.5, k, v, o2, lse, cu, **kw)
    assert same(want, attn.backward(do, q * 0.5, k, v, o2, lse, cu, o_rest=lse2.o_rest, **kw))
    attn.backward(do, q * 0.5, k, v, o2, lse, cu, o_rest=False, **kw)
    # a forward call into it brings its remainder up to date
    attn.forward(q * 0.5, k, v, cu, o=o, lse=lse, **kw)
    assert same(want, attn.backward(do, q * 0.5, k, v, o, lse, cu, **kw))


def test_inference_tensors(case):
    attn, qkv, do, cu, kw = case
    o, lse = attn.forward(*qkv, cu, want_lse=True, **kw)
    want = attn.backward(do, *qkv, o, lse, cu, **kw)
    with torch.inference_mode():
        o, lse = attn.forward(*qkv, cu, want_lse=True, **kw)
        assert same(want, attn.backward(do, *qkv, o, lse, cu, **kw))


def test_refusals(case):
    attn, (q, k, v), do, cu, kw = case
    o, lse = attn.forward(q, k, v, cu, want_lse=True, **kw)
    for bad in (torch.empty_like(o)[1:], torch.empty_like(o).half(), torch.empty(o.shape, dtype=BF), o.transpose(0, 1)):
        with pytest.raises(ValueError):
            attn.forward(q, k, v, cu, want_lse=True, o_rest=bad, **kw)
        with pytest.raises(ValueError):
            attn.backward(do, q, k, v, o, lse, cu, o_rest=bad, **kw)
    with pytest.raises(ValueError):
        attn.forward(q, k, v, cu, o_rest=torch.empty_like(o), **kw)        # nothing to go with: no lse


def test_lse_used_by_other_handles(api, case):
    """A remainder that does not fit the call's tensors is left behind, not refused."""
    attn, (q, k, v), do, cu, kw = case
    o, lse = attn.forward(q, k, v, cu, want_lse=True, **kw)
    half = api.PackedAttn(4, 2, 64, dtype=torch.float16)
    half.forward(q.half(), k.half(), v.half(), cu, lse=lse, **kw)
    assert lse.o_rest is None
    # a call that is refused changes nothing
    o, lse = attn.forward(q, k, v, cu, want_lse=True, **kw)
    rest = lse.o_rest
    with pytest.raises(api.TraError):
        attn.forward(q, k, v, cu, lse=lse, o_rest=False, max_q=10 ** 6, max_k=125)
    assert lse.o_rest is rest


def test_copies_that_carry_the_remainder_along(case):
    """Deep copies, stored and loaded tensors, and buffers into which both are copied keep lse and remainder together."""
    attn, (q, k, v), do, cu, kw = case
    o, lse = attn.forward(q, k, v, cu, want_lse=True, **kw)
    want = attn.backward(do, q, k, v, o, lse, cu, **kw)
    stored = io.BytesIO()
    torch.save(lse, stored)
    stored.seek(0)
    for other in (copy.deepcopy(lse), torch.load(stored, weights_only=False)):
        assert torch.equal(other.o_rest, lse.o_rest)
        assert same(want, attn.backward(do, q, k, v, o, other, cu, **kw))
    _, buffer = attn.forward(q * 0.5, k, v, cu, want_lse=True, **kw)
    buffer.copy_(lse)
    with pytest.raises(ValueError):
        attn.backward(do, q, k, v, o, buffer, cu, **kw)
    buffer.o_rest.copy_(lse.o_rest)
    assert same(want, attn.backward(do, q, k, v, o, buffer, cu, **kw))
    with pytest.raises(ValueError):
        attn.forward(q, k, v, cu, want_lse=True, o_rest=True, **kw)
