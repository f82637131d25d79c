"""Arrays of a call that overlap where one of them is written, through the C ABI
and without a GPU: refused before anything is enqueued."""
import os

import pytest

from paper_1610_05838_amd import mfsgd as M

EINVAL = -1
A, B, D, E, F, G, H = (i << 32 for i in range(1, 8))  # aligned addresses far apart that no refused call may touch
BIG = 1 << 62


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(M.LIB_PATH):
        from paper_1610_05838_amd import _build
        _build.build()
    return M.lib()


def refused(lib, fn, args, text):
    assert getattr(lib, fn)(*args) == EINVAL, (fn, args)
    assert text in lib.mfsgd_last_error(), (fn, args, lib.mfsgd_last_error())


def changed(base, **what):
    got = dict(base)
    got.update(what)
    return tuple(got.values())


EMBED = dict(table=A, rows=10, ld=8, k=8, dtype=0, ids=B, ids_stride=3, count=4, scale=1.0, out=D, ld_out=8,
             stream=None)


@pytest.mark.parametrize("what", [
    dict(out=A), dict(out=A + 4), dict(out=A + 10 * 32 - 4), dict(out=A - 4 * 32 + 4),  # the table
    dict(out=A + 16, ld_out=16), dict(ld=16, out=A + 28, ld_out=16), dict(ld=24, out=A + 68, ld_out=12),
    dict(out=B), dict(out=B + 36), dict(out=B - 124),  # the ids: bytes 0-3, 12-15, 24-27, 36-39
    dict(out=B - 112, k=2, ld_out=9),  # its rows' bytes from B: -112..-105, -76..-69, -40..-33, -4..3
])
def test_embed_refuses_overlap(lib, what):
    refused(lib, "mfsgd_embed", changed(EMBED, **what), b"overlap")


GRAD = dict(dout=A, ld_dout=8, ids=B, ids_stride=1, count=9000, k=8, dtype=0, scale=1.0, dtable=D, rows=10, ld=8,
            accumulate=0, work=E, nbytes=BIG, stream=None)


@pytest.mark.parametrize("what", [
    dict(dtable=A), dict(dtable=A + 8999 * 32), dict(dtable=B + 100), dict(work=A), dict(work=B), dict(work=D),
    dict(dtable=E + 1024), dict(dtable=A, accumulate=1)])
def test_embed_grad_refuses_overlap(lib, what):
    refused(lib, "mfsgd_embed_grad", changed(GRAD, **what), b"overlap")


LINEAR = dict(x=A, ldx=8, w=B, ldw=8, bias=D, residual=E, ldr=8, M=8, N=8, K=8, dtype=0, act=0, y=F, ldy=8,
              z=G, ldz=8, work=None, nbytes=0, stream=None)


@pytest.mark.parametrize("what", [
    dict(y=A), dict(y=B), dict(y=D), dict(z=A), dict(z=B), dict(z=D), dict(z=E), dict(z=F), dict(y=A + 252),
    dict(y=E + 4), dict(y=E, ldy=9),  # the residual may be y itself, no other part of it
    dict(ldx=20, y=A + 28, ldy=20), dict(ldx=20, y=A + 52, ldy=20), dict(ldx=24, y=A + 40, ldy=12)])
def test_linear_refuses_overlap(lib, what):
    refused(lib, "mfsgd_linear", changed(LINEAR, **what), b"overlap")


@pytest.mark.parametrize("at", [A, B, D, E, F, G])
def test_linear_refuses_a_workspace_in_use(lib, at):
    refused(lib, "mfsgd_linear", changed(LINEAR, M=64, N=64, K=65536, ldx=65536, ldw=65536, ldr=64, ldy=64, ldz=64,
                                         work=at, nbytes=BIG), b"overlap")


LGRAD = dict(dy=A, lddy=8, z=B, ldz=8, x=D, ldx=8, w=E, ldw=8, M=8, N=8, K=8, dtype=0, act=4, dx=F, lddx=8, dw=G,
             lddw=8, dbias=H, work=H + 4096, nbytes=BIG, stream=None)


@pytest.mark.parametrize("out", ["dx", "dw", "dbias", "work"])
@pytest.mark.parametrize("at", [A, B, D, E, F, G, H, H + 4096])
def test_linear_grad_refuses_overlap(lib, out, at):
    if LGRAD[out] != at:
        refused(lib, "mfsgd_linear_grad", changed(LGRAD, **{out: at}), b"overlap")


def entries(*ts):
    a = (M.TensorList._Entry * max(len(ts), 1))()
    for e, (p, n, d) in zip(a, ts):
        e.data, e.n, e.dtype = p, n, d
    return a


@pytest.mark.parametrize("norm,work", [(A, E), (A + 392, E), (D, A), (D, A + 256), (E, E), (E + 64, E), (A - 4 + 4, E)])
def test_norms_refuse_overlap(lib, norm, work):
    g, p = entries((A, 100, 0)), entries((B, 100, 0))
    refused(lib, "mfsgd_grad_norm", (g, 1, norm, work, BIG, None), b"overlap")
    refused(lib, "mfsgd_clip_grads", (g, 1, 1.0, norm, work, BIG, None), b"overlap")
    refused(lib, "mfsgd_sgd_step", (p, g, 1, 0.1, 0.0, 1.0, norm, work, BIG, None), b"overlap")
    refused(lib, "mfsgd_sgd_step", (g, p, 1, 0.1, 0.0, 1.0, norm, work, BIG, None), b"overlap")
