"""Rotary positions and attention over bf16 rows: calls with nothing in them, without a GPU."""
import ctypes as C

import pytest

from paper_2601_17818_b200 import binding as vb
from paper_2601_17818_b200.build import build_library

NULL, AT = None, [C.c_void_p(x << 20) for x in range(16, 32)]


@pytest.fixture(scope="module")
def L():
    build_library()
    return vb.lib()


def _rotary(L, q, k, B, Hq, Hk, N):
    s = (64 * 64, 64, 64)
    return L.vitcop_rotary_axes(q, k, B, Hq, Hk, N, 64, *s, *s, AT[0], 3, max(N, 0), NULL, NULL, AT[1], AT[2], 32, 0, q, *s, k, *s, NULL)


@pytest.mark.parametrize("B,Hq,Hk,N", [(0, 4, 2, 8), (2, 4, 2, 0), (2, 0, 0, 8), (0, 0, 0, 0)])
def test_turning_tensors_of_no_elements_is_nothing_to_do(L, B, Hq, Hk, N):
    """They have no address: an empty batch reaches the call as NULL."""
    assert _rotary(L, NULL, NULL, B, Hq, Hk, N) == vb.OK


@pytest.mark.parametrize("B,Hq,Hk,N", [(1, 4, 2, 8), (2, 4, 0, 1), (1, 0, 1, 1)])
def test_turning_nothing_where_there_are_rows_is_refused(L, B, Hq, Hk, N):
    assert _rotary(L, NULL, NULL, B, Hq, Hk, N) == vb.ERR_INVALID_ARG


@pytest.mark.parametrize("sizes", [dict(B=-1), dict(Hq=-1), dict(Hk=-1), dict(N=-1)])
def test_sizes_below_nothing_are_refused(L, sizes):
    assert _rotary(L, NULL, NULL, **{**dict(B=0, Hq=0, Hk=0, N=0), **sizes}) == vb.ERR_INVALID_ARG
