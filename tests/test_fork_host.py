"""Sizes that a fork refuses before anything touches a GPU."""
import ctypes

import pytest

from paper_2512_13368_amd import binding as B
from test_paged_host import params

vp = ctypes.c_void_p
A, A2, A3 = vp(4096), vp(8192), vp(12288)  # made-up addresses: every call must fail before they are used


def fork(p, N):
    return B.lib().blossom_kv_fork(ctypes.byref(p.c()), N, 1, A, A, A, A, A2, A2, A2, A3, A3, A, 1 << 40, None)


@pytest.mark.parametrize("many", [(1 << 20) + 1, 1 << 22, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, 1 << 26])
def test_more_sequences_than_each_can_look_through_are_refused(many):
    # (from 2^25 on a wavefront's number was taken from a thread's as one of 31 bits: rows before the first)
    assert fork(params(max_pages=1), many) == -2
    assert fork(params(S=many, H=1, G=1, max_pages=1), 3) == -2
