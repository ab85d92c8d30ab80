"""Which sizes the linear projection takes (CPU; every call here is refused
before any HIP call)."""
import ctypes

import pytest

from paper_2506_20686_amd import binding as B

P = 0x10000  # fake, 16-byte aligned, never touched


def fwd(m, k, n):
    # without x: a call whose sizes are taken is refused as an invalid argument
    return B.tri_linear_fwd(B.BF16, m, k, n, 0, None, P, None, None, P, None, None)


def bwd_ws(m, k, n):
    return B.lib().tri_linear_bwd_workspace_bytes(B.BF16, m, k, n, 0,
                                                  ctypes.byref(ctypes.c_size_t()))


@pytest.mark.parametrize("m,k,n", [(1 << 23, 8192, 64), (1 << 24, 8192, 1), ((1 << 29) - 64, 65, 100),
                                   ((1 << 30) - 64, 128, 64), (1 << 17, 8192, 8192 - 64)])
def test_forward_is_bounded_by_its_outputs_alone(m, k, n):
    # fewer than 2^24 tiles of 64 x 64 outputs, however long the sums are
    assert -(-m // 64) * -(-n // 64) < 1 << 24
    assert fwd(m, k, n) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("m,k,n", [(1 << 30, 1, 64), (1 << 29, 1, 65), (1 << 23, 64, 8192)])
def test_forward_with_too_many_outputs(m, k, n):
    assert fwd(m, k, n) == B.ERR_UNSUPPORTED


def test_backward_is_bounded_by_both():
    assert bwd_ws(1 << 23, 8192, 64) == bwd_ws(1 << 23, 64, 8192) == B.ERR_UNSUPPORTED
    assert bwd_ws((1 << 23) - 64, 8192, 64) == bwd_ws((1 << 23) - 64, 64, 8192) == B.OK
