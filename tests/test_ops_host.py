"""What the operators of include/mfsgd.h refuse, through the C ABI and without a
GPU: every argument that a kernel could not take safely is turned away before
anything is enqueued, with a text that says why."""
import ctypes as C
import os

import pytest

from paper_1610_05838_amd import mfsgd as M

EINVAL, ESTATE = -1, -4
A = 0x10000  # an aligned address that no refused call may touch
BIG = 1 << 62
INT32_MAX = 2**31 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(M.LIB_PATH):
        from paper_1610_05838_amd import _build
        _build.build()
    return M.lib()


def refused(lib, fn, args, code=EINVAL):
    assert getattr(lib, fn)(*args) == code, (fn, args)
    assert lib.mfsgd_last_error(), fn


def changed(base, **what):
    got = dict(base)
    got.update(what)
    return tuple(got.values())


EMBED = dict(table=A, rows=10, ld=8, k=8, dtype=0, ids=A, ids_stride=1, count=4, scale=1.0, out=A, ld_out=8,
             stream=None)
GRAD = dict(dout=A, ld_dout=8, ids=A, ids_stride=1, count=4, k=8, dtype=0, scale=1.0, dtable=A, rows=10, ld=8,
            accumulate=0, work=None, nbytes=0, stream=None)


@pytest.mark.parametrize("what", [
    dict(table=None), dict(table=A + 2), dict(rows=0), dict(rows=-1), dict(rows=2**31), dict(ld=7), dict(k=0),
    dict(k=-3), dict(dtype=3), dict(dtype=-1), dict(ids=None), dict(ids=A + 1), dict(ids_stride=0),
    dict(ids_stride=-1), dict(ids_stride=2**28 + 1), dict(k=2**22 + 1, ld=2**23, ld_out=2**23), dict(count=-1), dict(count=2**31), dict(out=None), dict(out=A + 1), dict(ld_out=7),
    dict(ld=BIG), dict(dtype=1, table=A + 1)])
def test_embed_refuses(lib, what):
    refused(lib, "mfsgd_embed", changed(EMBED, **what))


@pytest.mark.parametrize("what", [
    dict(dout=None), dict(dout=A + 2), dict(ld_dout=7), dict(ids=None), dict(ids=A + 2), dict(ids_stride=0),
    dict(count=-1), dict(count=2**31), dict(k=0), dict(k=2**22 + 1, ld=2**23, ld_dout=2**23), dict(dtype=9), dict(dtable=None), dict(dtable=A + 1),
    dict(rows=0), dict(rows=2**31), dict(ld=3),
    dict(count=100_000, work=None, nbytes=BIG), dict(count=100_000, work=A, nbytes=64),
    dict(count=100_000, work=A + 8, nbytes=BIG), dict(count=100_000, work=A, nbytes=-1)])
def test_embed_grad_refuses(lib, what):
    refused(lib, "mfsgd_embed_grad", changed(GRAD, **what))


def test_empty_calls_are_no_errors(lib):
    """No tokens: nothing to read or write (the gradient only where it adds)."""
    assert lib.mfsgd_embed(*changed(EMBED, count=0, ids=None, out=None)) == 0
    assert lib.mfsgd_embed_grad(*changed(GRAD, count=0, ids=None, dout=None, accumulate=1)) == 0
    assert lib.mfsgd_last_error() == b""


def test_embed_grad_workspace(lib):
    n = C.c_int64(-1)
    assert lib.mfsgd_embed_grad_workspace(10, 128, C.byref(n)) == 0 and n.value == 0
    assert lib.mfsgd_embed_grad_workspace(1_000_000, 128, C.byref(n)) == 0 and n.value >= 16_000_000
    assert lib.mfsgd_embed_grad_workspace(INT32_MAX, 1 << 22, C.byref(n)) == 0 and n.value > 1 << 45
    for count, k in ((-1, 8), (2**31, 8), (5, 0), (5, 2**22 + 1)):
        refused(lib, "mfsgd_embed_grad_workspace", (count, k, C.byref(n)))
    refused(lib, "mfsgd_embed_grad_workspace", (5, 8, None))


def test_model_rows_need_a_model(lib):
    assert lib.mfsgd_finalize() in (0, -3)
    refused(lib, "mfsgd_rows", (0, A, 1, 4, 8, 0, 1.0, A, 8, None), ESTATE)
    refused(lib, "mfsgd_add_rows", (0, A, 8, A, 1, 4, 8, 0, 1.0, None, 0, None), ESTATE)


def entries(*ts):
    a = (M.TensorList._Entry * max(len(ts), 1))()
    for e, (p, n, d) in zip(a, ts):
        e.data, e.n, e.dtype = p, n, d
    return a


GOOD = (A, 100, 0)


@pytest.mark.parametrize("t", [(None, 5, 0), (A + 2, 5, 0), (A + 1, 5, 1), (A, -1, 0), (A, (1 << 40) + 1, 0), (A, 5, 3),
                               (A, 5, -1)])
def test_norm_refuses_a_tensor(lib, t):
    a = entries(GOOD, t)
    refused(lib, "mfsgd_grad_norm", (a, 2, A, A, BIG, None))
    refused(lib, "mfsgd_clip_grads", (a, 2, 1.0, A, A, BIG, None))
    refused(lib, "mfsgd_sgd_step", (a, a, 2, 0.1, 0.0, 1.0, A, A, BIG, None))


@pytest.mark.parametrize("call", [
    dict(count=-1), dict(count=(1 << 20) + 1), dict(list=None), dict(norm=None), dict(norm=A + 4), dict(work=None),
    dict(work=A + 8), dict(nbytes=100), dict(nbytes=-1)])
def test_norm_refuses(lib, call):
    base = dict(list=entries(GOOD), count=1, norm=A, work=A, nbytes=BIG, stream=None)
    refused(lib, "mfsgd_grad_norm", changed(base, **call))


def test_norm_refuses_too_many_elements(lib):
    a = entries(*[(A, 1 << 40, 1)] * 9)
    refused(lib, "mfsgd_grad_norm", (a, 9, A, A, BIG, None))


@pytest.mark.parametrize("max_norm", [-1.0, float("nan")])
def test_clip_refuses_a_bound(lib, max_norm):
    refused(lib, "mfsgd_clip_grads", (entries(GOOD), 1, max_norm, A, A, BIG, None))


def test_clip_refuses_overlap(lib):
    for b in ((A, 100, 0), (A + 396, 10, 0), (A + 200, 1, 1), (A - 4, 2, 0)):
        refused(lib, "mfsgd_clip_grads", (entries(GOOD, b), 2, 1.0, A, A, BIG, None))
        refused(lib, "mfsgd_clip_grads", (entries(b, GOOD), 2, 1.0, A, A, BIG, None))
    # inside one that a later one follows
    refused(lib, "mfsgd_clip_grads", (entries((A, 1000, 0), (A + 400, 10, 0), (A + 3000, 10, 0)), 3, 1.0, A, A, BIG,
                                      None))


def test_step_refuses(lib):
    g = (A + 4096, 100, 0)
    for p in ((A, 99, 0), (A, 100, 1), (A + 4096, 100, 0), (A + 4092, 100, 0), (A + 3700, 100, 0)):
        refused(lib, "mfsgd_sgd_step", (entries(p), entries(g), 1, 0.1, 0.0, 1.0, A, A, BIG, None))
    for lr, lam, most in ((float("inf"), 0.0, 1.0), (float("nan"), 0.0, 1.0), (0.1, float("inf"), 1.0),
                          (0.1, 0.0, -2.0), (0.1, 0.0, float("nan"))):
        refused(lib, "mfsgd_sgd_step", (entries(GOOD), entries(g), 1, lr, lam, most, A, A, BIG, None))
    # one parameter twice
    refused(lib, "mfsgd_sgd_step", (entries(GOOD, GOOD), entries(g, g), 2, 0.1, 0.0, 1.0, A, A, BIG, None))


def test_norm_workspace(lib):
    n = C.c_int64(-1)
    assert lib.mfsgd_norm_workspace(0, C.byref(n)) == 0 and n.value > 0
    a = n.value
    assert lib.mfsgd_norm_workspace(1000, C.byref(n)) == 0 and n.value > a
    for count in (-1, (1 << 20) + 1):
        refused(lib, "mfsgd_norm_workspace", (count, C.byref(n)))
    refused(lib, "mfsgd_norm_workspace", (1, None))


LINEAR = dict(x=A, ldx=8, w=A, ldw=8, bias=None, residual=None, ldr=6, M=4, N=6, K=8, dtype=0, act=0, y=A, ldy=6,
              z=None, ldz=0, work=None, nbytes=0, stream=None)
LGRAD = dict(dy=A, lddy=6, z=A, ldz=6, x=A, ldx=8, w=A, ldw=8, M=4, N=6, K=8, dtype=0, act=4, dx=A, lddx=8, dw=A,
             lddw=8, dbias=A, work=A, nbytes=BIG, stream=None)


@pytest.mark.parametrize("what", [
    dict(x=None), dict(x=A + 1), dict(ldx=7), dict(w=None), dict(ldw=7), dict(bias=A + 2), dict(residual=A + 1),
    dict(residual=A, ldr=5), dict(M=-1), dict(N=-1), dict(K=-1), dict(M=2**31), dict(N=2**31), dict(K=2**31, ldx=2**31),
    dict(dtype=3), dict(act=5), dict(act=-1), dict(y=None), dict(ldy=5), dict(z=A, ldz=5), dict(z=A + 2, ldz=6),
    dict(M=64, N=64, K=65536, ldx=65536, ldw=65536, ldy=64), dict(ldx=BIG)])
def test_linear_refuses(lib, what):
    refused(lib, "mfsgd_linear", changed(LINEAR, **what))


@pytest.mark.parametrize("what", [
    dict(dy=None), dict(dy=A + 1), dict(lddy=5), dict(z=None), dict(ldz=5), dict(x=None), dict(ldx=7), dict(w=None),
    dict(ldw=7), dict(M=-1), dict(N=2**31), dict(K=-1), dict(dtype=7), dict(act=9), dict(dx=A + 2), dict(lddx=7),
    dict(dw=A + 2), dict(lddw=7), dict(dbias=A + 2), dict(work=None), dict(work=A + 64), dict(nbytes=16),
    dict(nbytes=-1)])
def test_linear_grad_refuses(lib, what):
    refused(lib, "mfsgd_linear_grad", changed(LGRAD, **what))


def test_product_workspaces(lib):
    n = C.c_int64(-1)
    assert lib.mfsgd_linear_workspace(1, 17770, 128, 1, C.byref(n)) == 0 and n.value == 0
    assert lib.mfsgd_linear_workspace(64, 64, 65536, 0, C.byref(n)) == 0 and n.value > 0
    for sizes in ((0, 0, 0), (40, 0, 7), (0, 40, 7), (40, 40, 0), (40, 0, 0), (INT32_MAX, 1, 1), (1, INT32_MAX, 1)):
        for fn in (lib.mfsgd_linear_workspace, lib.mfsgd_linear_grad_workspace):
            assert fn(*sizes, 0, C.byref(n)) == 0 and n.value >= 0
    assert lib.mfsgd_linear_grad_workspace(100, 100, 100, 2, C.byref(n)) == 0 and n.value >= 4 * 20_000
    for fn in ("mfsgd_linear_workspace", "mfsgd_linear_grad_workspace"):
        for bad in ((-1, 1, 1, 0), (1, 2**31, 1, 0), (1, 1, -5, 0), (1, 1, 1, 3)):
            refused(lib, fn, (*bad, C.byref(n)))
        refused(lib, fn, (1, 1, 1, 0, None))


def test_the_sums_of_slices_stay_within_the_caches(lib):
    n = C.c_int64(-1)
    for dtype in (0, 1, 2):
        for sizes in ((4096, 4096, 1 << 20), (17, 17, INT32_MAX), (300, 5000, 1 << 24), (20_000, 20_000, 1 << 16)):
            assert lib.mfsgd_linear_workspace(*sizes, dtype, C.byref(n)) == 0
            assert 0 <= n.value <= 256 << 20


def test_scores_need_a_model(lib):
    n = C.c_int64(-1)
    refused(lib, "mfsgd_scores_workspace", (5, C.byref(n)), ESTATE)
    refused(lib, "mfsgd_scores", (A, 1, 4, 100, 0, None, 0, A, 100, A, BIG, None), ESTATE)
