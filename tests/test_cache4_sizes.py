"""The workspace query of attention over the 4-bit cache at the ends of its arguments, on the CPU: it answers, whatever the sizes, and what the call refuses
needs nothing."""
import ctypes

import pytest

from paper_2608_02504_b200 import build

build.build()
from paper_2608_02504_b200 import api  # noqa: E402
from tests.test_packed_refusals import Handle  # noqa: E402

MOST = 1 << 30


def size(n_seq, total_q, max_q, max_k, dtype=api.TRA_BF16, window=0, sinks=0):
    h = Handle(api.tra_packed_config_t(40, 8, 128, dtype, 1, window, sinks), -7, 148, None)
    return api._lib.tra_packed_attn_cache4_workspace_bytes(ctypes.byref(h), n_seq, total_q, max_q, max_k)


@pytest.mark.parametrize("dtype", [api.TRA_BF16, api.TRA_FP16])
@pytest.mark.parametrize("max_q", [1, 100])
@pytest.mark.parametrize("window,sinks", [(0, 0), (4096, 16), (MOST, MOST)])
def test_more_keys_than_a_cache_holds(dtype, max_q, window, sinks):
    for max_k in (MOST + 1, 2_000_000_000, 2 ** 31 - 8, 2 ** 31 - 1):
        for n_seq in (1, 7, 2 ** 31 - 1):
            assert size(n_seq, 100, max_q, max_k, dtype, window, sinks) == 0
    assert size(1, MOST + 1, max_q, 100, dtype, window, sinks) == 0 and size(1, 2 ** 31 - 1, 2 ** 31 - 1, 100, dtype, window, sinks) == 0


@pytest.mark.parametrize("dtype", [api.TRA_BF16, api.TRA_FP16])
def test_the_most_keys_that_a_cache_holds(dtype):
    # one sequence at a time: keys and values of eight heads, in two numbers each for fp16, and the queries beside them
    keys = 2 * MOST * 8 * 128 * (2 if dtype == api.TRA_BF16 else 4)
    for max_k in (MOST - 7, MOST - 1, MOST):
        for n_seq in (1, 7):
            assert keys <= size(n_seq, 100, 100, max_k, dtype) < keys + (1 << 30)
    assert size(2 ** 31 - 1, 100, 100, MOST, dtype) < keys + (1 << 30)
    assert 0 < size(64, 64, 1, MOST, dtype) < 1 << 30                # parts of a row each
    assert size(1, MOST, MOST, 100, dtype) > 0


@pytest.mark.parametrize("dtype", [api.TRA_BF16, api.TRA_FP16])
def test_every_size_has_an_answer(dtype):
    for n_seq in (1, 3, 400):
        for max_q in (0, 1, 12, 13, 14, 64, 1000):
            for max_k in (0, 1, 7, 8, 9, 4095, 1 << 20, MOST - 1, MOST):
                for window, sinks in ((0, 0), (1, 0), (5, 300), (4096, 4)):
                    assert size(n_seq, 1000, max_q, max_k, dtype, window, sinks) < 1 << 45
