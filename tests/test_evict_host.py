"""Limits of the eviction's sizes, without a GPU."""
import ctypes

import pytest
import torch

from paper_2605_18753_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    from paper_2605_18753_b200 import build
    build.build()
    return B.lib()


@pytest.mark.parametrize("keep,code", [((1 << 31) - 1, -2), ((1 << 31) - 4000, -2), ((1 << 30) + 1, -2), (1 << 30, None)])
def test_a_list_beyond_32_bits_of_steps_is_refused(lib, keep, code):
    """The blocks fill the list behind the kept slots with -1 in steps of up to 4096: from 2^31 - 4096 on their counter ran over."""
    if code is None and torch.cuda.is_available():
        pytest.skip("an accepted call would launch on addresses that are none")
    pool, table = torch.zeros(3, 16, 1, 64), torch.zeros(1, 2, dtype=torch.int32)
    p = B.params_for_paged(pool, pool, table, h_q=1, rows=0)
    got = lib.dash_attn_evict_paged(ctypes.byref(p), keep, 0, 0, 16, 32, 48, 64, 64, 80, 96, 112, 2, 3, 128, 128, 144, None)
    assert got == code if code else got not in (-1, -2)
