"""Calls beyond the limits that the attention over caches counts rows with, by dry runs."""
import ctypes

import pytest

from paper_2608_21541_amd import _lib
from test_abi import FAKE, problem
from test_mx_abi import attend_call


@pytest.mark.parametrize("name", ["mx", "tree"])
def test_more_rows_than_are_counted_are_unsupported(name):
    # 32 layers x 4 heads x 2^24 rows are 2^31; a bound on a segment's rows admits more layers
    p = problem(L=31, seqlens=(1 << 24,))
    assert _lib.lib().certkv_decode_cache_workspace_size(ctypes.byref(p), 1, 1, 0, 0) > 0
    p = problem(L=33, seqlens=(1 << 24,))
    assert _lib.lib().certkv_decode_cache_workspace_size(ctypes.byref(p), 1, 1, 0, 0) == 0
    for ws in (None, FAKE):  # (a workspace of the size that is given, none, is NULL)
        for size in (0, 1 << 40):
            assert attend_call(name, p=p, ws=ws, size=size) == _lib.CERTKV_EUNSUPPORTED
    assert attend_call(name, p=p, max_rows=1 << 20) == _lib.CERTKV_OK
