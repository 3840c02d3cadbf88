"""Settings of kd_sample that its parameter block's 32 bits do not hold."""
import ctypes

import pytest

from paper_2603_01875_amd import kdloss as K


@pytest.mark.parametrize("top_k,kept", [(0, 0), (7, 7), ((1 << 31) - 1, (1 << 31) - 1), (1 << 31, (1 << 31) - 1), ((1 << 32) + 5, (1 << 31) - 1), (10 ** 15, (1 << 31) - 1)])
def test_a_top_k_of_more_than_any_row_keeps_all(top_k, kept):
    assert K.make_sample_params(4, 100, top_k=top_k).top_k == kept


@pytest.mark.parametrize("top_k", [-1, -(1 << 31) - 1, -(1 << 32), -(1 << 32) + 5])
def test_a_negative_top_k_is_refused(top_k):
    n = ctypes.c_size_t(0)
    assert K.lib().kd_sample_workspace_size(ctypes.byref(K.make_sample_params(4, 100, top_k=top_k)), ctypes.byref(n)) == 4
