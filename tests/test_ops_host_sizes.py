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


def test_embed_grad_workspace_of_a_table(lib):
    """Never more than the one that is enough for any table, and the call asks for no more."""
    any_table, n = C.c_int64(-1), C.c_int64(-1)
    for count in (0, 1, 2048, 2049, 8192, 8193, 300_000):
        assert lib.mfsgd_embed_grad_workspace(count, 40, C.byref(any_table)) == 0
        for rows in (1, 3, 100, 1_000_000, INT32_MAX):
            assert lib.mfsgd_embed_grad_workspace_rows(count, 40, rows, C.byref(n)) == 0
            assert 0 <= n.value <= any_table.value
    for count, k, rows in ((-1, 8, 5), (INT32_MAX + 1, 8, 5), (5, 0, 5), (5, 8, 0), (5, 8, -1), (5, 8, INT32_MAX + 1)):
        refused(lib, "mfsgd_embed_grad_workspace_rows", (count, k, rows, C.byref(n)), b"must be")
    refused(lib, "mfsgd_embed_grad_workspace_rows", (5, 8, 5, None), b"NULL")
    # 5,000 tokens of 3 rows need one
    refused(lib, "mfsgd_embed_grad", (A, 8, B, 1, 5000, 8, 0, 1.0, D, 3, 8, 0, None, 0, None), b"workspace")
