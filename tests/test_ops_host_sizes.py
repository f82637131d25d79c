"""Sizes whose workspace no memory holds, through the C ABI and without a GPU:
refused by the query and by the call, before anything is enqueued."""
import ctypes as C
import os

import pytest

from paper_1610_05838_amd import mfsgd as M

EINVAL = -1
A, B, D = 1 << 32, 2 << 32, 3 << 32  # aligned addresses far apart that no refused call may touch
INT32_MAX = 2**31 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(M.LIB_PATH):
        from paper_1610_05838_amd import _build
        _build.build()
    return M.lib()


def refused(lib, fn, args, text):
    assert getattr(lib, fn)(*args) == EINVAL, (fn, args)
    assert text in lib.mfsgd_last_error(), (fn, args, lib.mfsgd_last_error())


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("sizes", [(INT32_MAX, 1, INT32_MAX), (1 << 30, INT32_MAX, 1 << 30), (INT32_MAX, INT32_MAX, 1),
                                   (1, INT32_MAX, INT32_MAX), (INT32_MAX, INT32_MAX, INT32_MAX)])
def test_a_gradient_too_large_for_any_workspace_is_refused(lib, dtype, sizes):
    n = C.c_int64(-7)
    refused(lib, "mfsgd_linear_grad_workspace", (*sizes, dtype, C.byref(n)), b"workspace")
    assert n.value == -7


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_gradient_workspaces_grow_with_their_sizes(lib, dtype):
    """Each matrix the gradient keeps is in the sum, up to sizes just below the refused ones."""
    n, es = C.c_int64(-1), 4 if dtype == 0 else 2
    for sizes in ((1 << 20, 1 << 20, 1 << 20), (1 << 28, 1 << 28, 1), (1 << 28, 1, 1 << 28), (1, 1 << 28, 1 << 28)):
        m, k, before = sizes[0], sizes[2], 0
        assert lib.mfsgd_linear_grad_workspace(*sizes, dtype, C.byref(n)) == 0
        assert n.value >= es * (2 * m * sizes[1] + m * k + sizes[1] * k)
        for part in range(1, 5):
            assert lib.mfsgd_linear_grad_workspace(*(s * part // 4 for s in sizes), dtype, C.byref(n)) == 0
            assert n.value > before
            before = n.value


def test_a_bias_gradient_of_a_refused_size_is_refused(lib):
    """dbias alone takes no matrix of K columns, but the workspace is laid out for one."""
    args = (A, 1, None, 0, None, 0, None, 0, INT32_MAX, 1, INT32_MAX, 0, 0, None, 0, None, 0, B, D, (1 << 63) - 1, None)
    refused(lib, "mfsgd_linear_grad", args, b"workspace")
