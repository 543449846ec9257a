"""What the rotary, recurrence and orthogonalisation calls refuse because no launch can hold it, or because results would depend on timing; on addresses
that nobody reads.  A launch has fewer than 2^32 threads."""
import ctypes

import pytest

from paper_2006_09503_amd import binding as B

P = 1 << 20     # an aligned address: refused calls only


def fwd(dtype, b, s, h):
    return B.lib().k2bw_recurrence_fwd(dtype, b, s, h, None, P, None, None, P, None, P, None)


def bwd(dtype, b, s, h):
    return B.lib().k2bw_recurrence_bwd(dtype, b, s, h, None, P, P, P, None, None, P, None, 0, P, None)


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("case", [
    (1, 1, 1 << 30, 8), (0, 1, 1 << 30, 8),               # 2^24 and 2^23 tiles of 512 threads
    (1, 1, 2 ** 31 - 64, 8), (0, 1, 2 ** 31 - 1, 8),
    (1, 1 << 26, 1, 8), (0, 1 << 27, 1, 8),               # a wave each
    (1, 1 << 20, 1, 1 << 13),
], ids=str)
def test_recurrence_refuses_more_than_a_launch_holds(case, call):
    assert call(*case) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("case", [(1, 1, 1 << 24, 64, 128, 64, 0), (0, 1 << 12, 1 << 13, 16, 128, 64, 0), (1, 1 << 10, (1 << 20) + 1, 1, 8, 4, 1)], ids=str)
def test_rotary_refuses_more_than_a_launch_holds(case):
    dtype, b, s, a, dh, n, pairing = case
    axis, freq = (ctypes.c_uint8 * 64)(), (ctypes.c_double * 64)(*([1.0] * 64))
    assert B.lib().k2bw_rotary(dtype, b, s, a, dh, n, pairing, axis, freq, 1, None, 0, P, None) == B.ERR_INVALID_ARG
