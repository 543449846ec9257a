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


@pytest.mark.parametrize("freq", [float("nan"), float("inf"), 1e300, -1.7e308])
def test_rotary_refuses_frequencies_whose_angles_are_not_finite(freq):
    axis, f = (ctypes.c_uint8 * 4)(), (ctypes.c_double * 4)(1.0, 1.0, 1.0, freq)
    assert B.lib().k2bw_rotary(0, 1, 1, 1, 8, 4, 0, axis, f, 1, None, 0, P, None) == B.ERR_INVALID_ARG


def orthogonalize(count, rows, cols, ld_in, stride_in, ld_out, stride_out, out=2 * P):
    return B.lib().k2bw_orthogonalize(1, count, rows, cols, P, ld_in, stride_in, out, ld_out, stride_out, 5, None, 4 * P, None)


def muon(count, rows, cols, ld, stride):
    return B.lib().k2bw_muon(1, count, rows, cols, ld, stride, P, P, None, 2 * P, 3 * P, 1e-3, 0.9, 0.0, 1.0, 1, 1, 5, None, 4 * P, None)


def share_an_element(count, rows, cols, ld, stride):
    at = [{i * stride + r * ld + c for r in range(rows) for c in range(cols)} for i in range(count)]
    return len(set().union(*at)) < sum(map(len, at))


@pytest.mark.parametrize("case", [(2, 16, 16, 16, 248), (2, 16, 16, 16, 8), (3, 8, 16, 40, 8), (3, 8, 16, 24, 16), (2, 8, 16, 64, 248), (4, 8, 8, 24, 8), (5, 2, 8, 64, 16)], ids=str)
def test_matrices_that_share_elements_are_refused(case):
    """They would hold what the last to arrive wrote."""
    count, rows, cols, ld, stride = case
    assert share_an_element(*case)
    assert muon(*case) == B.ERR_INVALID_ARG
    assert orthogonalize(count, rows, cols, ld, 8 * ld * rows, ld, stride) == B.ERR_INVALID_ARG


def test_several_matrices_in_place_keep_their_layout():
    assert orthogonalize(2, 16, 16, 16, 256, 24, 512, out=P) == B.ERR_INVALID_ARG
    assert orthogonalize(2, 16, 16, 16, 256, 16, 512, out=P) == B.ERR_INVALID_ARG
