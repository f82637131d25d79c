"""Products with bias, activation and residual, and their gradient
(mfsgd_linear, mfsgd_linear_grad, mfsgd_scores) against 64 bits.

Most inputs are small integers (or such times a power of two): every product
and sum is then exact in binary32 in any order, and the results have to be the
exact ones, rounded once.  eps / 2 of a type is the largest relative error of a
rounding to it."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402

DTYPES = (torch.float32, torch.float16, torch.bfloat16)
ID = {torch.float32: "fp32", torch.float16: "fp16", torch.bfloat16: "bf16"}
ACTS = ("none", "relu", "sigmoid", "silu", "gelu")


def ints(g, low, high, *shape):
    return torch.randint(low, high + 1, shape, generator=g, device="cuda").double()


def placed(x64, dtype, pad=0, shift=0, beside=math.nan):
    """x64 as a matrix of pitch width + pad that starts `shift` elements into its storage, `beside` around it."""
    rows, width = x64.shape
    store = torch.full((shift + rows * (width + pad) + 16,), beside, dtype=dtype, device="cuda")
    view = store[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width] if rows else store[:0].view(
        0, width)
    view.copy_(x64)
    return view, store


def act64(z, act):
    f = dict(none=lambda v: v, relu=torch.relu, sigmoid=torch.sigmoid, silu=torch.nn.functional.silu,
             gelu=torch.nn.functional.gelu)
    return f[act](z)


# few rows; tiles of 64, 128 and 256 rows; one slice of the depth and several; whole and ragged pieces
SHAPES = [(0, 5, 3), (5, 0, 3), (1, 1, 1), (1, 17, 0), (40, 9, 0), (3, 1000, 7), (16, 65, 64), (16, 333, 1500), (2, 50, 4096), (14, 51, 2619),
          (16, 9000, 2050), (17, 16, 8), (64, 300, 100), (33, 129, 2048), (64, 5000, 65), (65, 64, 31), (128, 128, 64), (130, 257, 72),
          (300, 40, 511), (1000, 333, 500), (257, 4100, 1), (700, 3000, 40), (128, 128, 4096), (4000, 3500, 520)]


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("odd", [False, True], ids=["aligned", "odd"])
def test_linear_is_the_exact_sum(dtype, m, n, k, odd):
    g = torch.Generator("cuda").manual_seed(m * 31 + n * 7 + k)
    pad, shift = (3, 1) if odd else (0, 0)
    x, _ = placed(ints(g, -3, 3, m, k), dtype, pad, shift)
    w, _ = placed(ints(g, -2, 2, n, k), dtype, pad, shift)
    bias, res = ints(g, -9, 9, n), ints(g, -9, 9, m, n)
    want = (x.double() @ w.double().t().contiguous()) if k else torch.zeros(m, n, dtype=torch.float64, device="cuda")
    assert torch.equal(M.linear(x, w).double(), want.to(dtype).double())
    out, store = placed(torch.zeros(m, n, device="cuda"), dtype, pad + 1, shift, beside=5.0)
    r, _ = placed(res, dtype, pad, shift)
    y, z = M.linear(x, w, bias=bias.to(dtype), residual=r, act="relu", out=out, keep_z=True)
    assert y is out
    assert torch.equal(z, (want + bias).to(dtype))
    assert torch.equal(y, (torch.relu(want + bias) + res).to(dtype))
    out.fill_(5.0)
    assert bool((store == 5.0).all())  # nothing beside y's columns
    # in place of the residual
    out.copy_(res)
    M.linear(x, w, residual=out, out=out)
    assert torch.equal(out, (want + res).to(dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,n,k", [(5, 100, 33), (70, 90, 64), (300, 260, 100)])
def test_activations(dtype, act, m, n, k):
    """On exact pre-activations: what is left is the activation's own error.  16-bit types: exponentials of
    relative error (|z| + 2) 2^-23 and erf to 1.5e-7; binary32: a few roundings."""
    g = torch.Generator("cuda").manual_seed(n)
    x, w = (ints(g, -3, 3, m, k) / 8).to(dtype), (ints(g, -2, 2, n, k) / 2).to(dtype)
    bias = (ints(g, -160, 160, n) / 16).to(dtype)
    z64 = x.double() @ w.double().t().contiguous() + bias.double()
    want = act64(z64, act)
    y, z = M.linear(x, w, bias=bias, act=act, keep_z=True)
    assert torch.equal(z, z64.to(dtype))
    eps = torch.finfo(dtype).eps / 2
    own = want.abs() * (z64.abs() + 8) * 2.0**-22 + (z64.abs() * 2.0**-21 if act == "gelu" else 0.0)
    assert bool(((y.double() - want).abs() <= want.abs() * eps + own * 1.01 + 1e-7 * (dtype == torch.float16)).all())


def test_special_values():
    """A NaN or infinity reaches its own row alone, and relu keeps a NaN."""
    for dtype in DTYPES:
        for m, n, k in ((4, 40, 24), (200, 300, 72), (40, 30, 13)):
            x, w = torch.ones(m, k, device="cuda", dtype=dtype), torch.ones(n, k, device="cuda", dtype=dtype)
            x[1, 3], x[2, 0] = math.nan, -math.inf
            for act in ("none", "relu"):
                y = M.linear(x, w, act=act)
                assert bool(torch.isnan(y[1]).all()) and bool((y[2] == (-math.inf if act == "none" else 0.0)).all())
                assert bool((y[0] == k).all()) and bool((y[3:] == k).all())
            assert bool((M.linear(x, w, act="sigmoid")[2] == 0.0).all())


def test_a_nan_before_the_activation_reaches_its_gradient():
    for dtype in DTYPES:
        x, w = torch.ones(40, 8, device="cuda", dtype=dtype), torch.ones(24, 8, device="cuda", dtype=dtype)
        z = torch.ones(40, 24, device="cuda", dtype=dtype)
        z[3, 5] = math.nan
        for act in ACTS[1:]:
            dx, dw, db = M.linear_grad(torch.ones_like(z), x, w, z=z, act=act)
            assert bool(torch.isnan(dx[3]).all()) and bool(torch.isnan(dw[5]).all()) and math.isnan(float(db[5]))
            assert int(torch.isnan(dx).sum()) == 8 and int(torch.isnan(dw).sum()) == 8 and int(torch.isnan(db).sum()) == 1


def test_large_arguments():
    """Activations far out, where the exponential overflows or vanishes."""
    z = torch.tensor([[-1e4], [-200.0], [-90.0], [-20.0], [0.0], [20.0], [90.0], [200.0], [1e4]], device="cuda")
    for dtype in DTYPES:
        x = z.to(dtype)
        one = torch.ones(1, 1, device="cuda", dtype=dtype)
        for act in ACTS:
            y, s = M.linear(x, one, act=act)[:, 0].double(), x[:, 0].double()
            want = act64(s, act)
            assert bool(((y - want).abs() <= want.abs() * (torch.finfo(dtype).eps / 2 + 2e-5) + 1e-7 * s.abs()).all()), (
                dtype, act, y, want)
            dx, _, _ = M.linear_grad(torch.ones_like(x), x, one, z=x, act=act)
            sr = s.clone().requires_grad_(True)
            slope, = torch.autograd.grad(act64(sr, act).sum(), sr)
            assert bool(((dx[:, 0].double() - slope).abs() <= slope.abs() * torch.finfo(dtype).eps + 2e-6).all()), (
                dtype, act, dx, slope)


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("m,n,k", [s for s in SHAPES if s != (4000, 3500, 520)] + [
    (4000, 1800, 520), (3000, 40, 3), (20000, 40, 24), (9000, 260, 700), (40, 9000, 130)])
@pytest.mark.parametrize("act,odd", [("none", False), ("none", True), ("relu", False), ("relu", True)])
def test_linear_grad_is_the_exact_sum(dtype, m, n, k, act, odd):
    g = torch.Generator("cuda").manual_seed(m + n * 3 + k * 5)
    pad, shift = (5, 1) if odd else (0, 0)
    x64, w64, dy64, z64 = ints(g, -3, 3, m, k), ints(g, -2, 2, n, k), ints(g, -2, 2, m, n), ints(g, -2, 2, m, n)
    x, w, dy, z = (placed(t, dtype, pad, shift)[0] for t in (x64, w64, dy64, z64))
    dz = dy64 * (z64 > 0) if act == "relu" else dy64
    dx, dw, db = M.linear_grad(dy, x, w, z=z if act == "relu" else None, act=act)
    assert torch.equal(dx, (dz @ w64).to(dtype))
    assert torch.equal(dw, (dz.t().contiguous() @ x64).to(dtype))
    assert torch.equal(db, dz.sum(0).to(dtype))
    # each alone is the same
    one = M.linear_grad(dy, x, w, z=z, act=act, dw=False, dbias=False)
    assert torch.equal(one[0], dx) and one[1] is None and one[2] is None
    assert torch.equal(M.linear_grad(dy, x, w, z=z, act=act, dx=False, dbias=False)[1], dw)
    assert torch.equal(M.linear_grad(dy, x, w, z=z, act=act, dx=False, dw=False)[2], db)


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("act", ACTS[2:])
@pytest.mark.parametrize("m,n,k", [(7, 60, 40), (200, 130, 96)])
def test_linear_grad_of_activations(dtype, act, m, n, k):
    """dZ is rounded to the type before the products: each of a sum's terms is off by eps / 2, its slope by a
    few 2^-20 at these z; the binary32 sums by (terms) 2^-24 of the magnitudes."""
    g = torch.Generator("cuda").manual_seed(k)
    x, w = (torch.randn(s, k, generator=g, device="cuda").to(dtype) for s in (m, n))
    dy, z = (torch.randn(m, n, generator=g, device="cuda").to(dtype) for _ in range(2))
    z64 = z.double().requires_grad_(True)
    dz, = torch.autograd.grad(act64(z64, act), z64, dy.double())
    got = M.linear_grad(dy, x, w, z=z, act=act)
    eps = torch.finfo(dtype).eps / 2
    near = dy.double().abs()  # a slope's error is absolute where its terms cancel
    for a, want, mag, n_terms, terms in (
            (got[0], dz @ w.double(), dz.abs() @ w.double().abs(), n, near @ w.double().abs()),
            (got[1], dz.t().contiguous() @ x.double(), dz.abs().t().contiguous() @ x.double().abs(), m,
             near.t().contiguous() @ x.double().abs()),
            (got[2], dz.sum(0), dz.abs().sum(0), m, near.sum(0))):
        tol = want.abs() * eps + mag * (eps + n_terms * 2.0**-24) * 1.01 + terms * 2.0**-20
        tol = tol + torch.finfo(dtype).smallest_normal * eps * (n_terms + 1)
        assert bool(((a.double() - want).abs() <= tol).all())
    again = M.linear_grad(dy, x, w, z=z, act=act)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("act", ACTS)
def test_linear_grad_against_differences(act):
    """Central differences of the operator along a direction.  Their own error: h^2 / 6 times the third
    derivative (below 2 for these functions) times the cubed change, and the results' rounding over 2 h."""
    g = torch.Generator("cuda").manual_seed(8)
    m, n, k, h = 9, 21, 30, 2.0**-6
    x, w = (torch.randn(s, k, generator=g, device="cuda") / 4 for s in (m, n))
    b, dy = torch.randn(n, generator=g, device="cuda") + 0.3, torch.randn(m, n, generator=g, device="cuda")
    dxd, dwd, dbd = torch.randn_like(x) / 8, torch.randn_like(w) / 8, torch.randn_like(b) / 8

    def value(t):
        y = M.linear((x.double() + t * dxd).float(), (w.double() + t * dwd).float(),
                     bias=(b.double() + t * dbd).float(), act=act)
        return y.double()

    y, z = M.linear(x, w, bias=b, act=act, keep_z=True)
    dx, dw, db = M.linear_grad(dy, x, w, z=z, act=act)
    analytic = float((dx.double() * dxd).sum() + (dw.double() * dwd).sum() + (db.double() * dbd).sum())
    hi, lo = value(h), value(-h)
    change = (dxd.double() @ w.double().t() + x.double() @ dwd.double().t() + dbd.double()).abs() + h
    if act == "relu":  # elements whose sign changes on the way have no derivative
        far = (z.double().abs() > 2 * h * change + 1e-3).double()
        dx, dw, db = M.linear_grad((dy * far).float(), x, w, z=z, act=act)
        analytic = float((dx.double() * dxd).sum() + (dw.double() * dwd).sum() + (db.double() * dbd).sum())
    else:
        far = torch.ones_like(change)
    numeric = float((dy.double() * far * (hi - lo)).sum()) / (2 * h)
    tol = float((dy.double().abs() * (h * h * 2 * (change + 1) ** 3 + (y.double().abs() + 4) * 2.0**-20 / h)).sum())
    assert abs(numeric - analytic) <= tol, (numeric, analytic, tol)


def test_offsets_past_32_bits():
    """Rows of X and Y beyond 2^31 elements (binary16)."""
    m, k, n = 36_000_000, 64, 8
    x = torch.zeros(m, k, dtype=torch.float16, device="cuda")
    x[m - 1], x[33_554_433], x[5] = 1.0, 2.0, 3.0
    w = torch.arange(1, n + 1, device="cuda", dtype=torch.float16)[:, None].expand(n, k).contiguous()
    y = M.linear(x, w, act="relu")
    at = torch.tensor([m - 1, 33_554_433, 5, 6], device="cuda")
    assert y[at, 7].tolist() == [512.0, 1024.0, 1536.0, 0.0] and int(torch.count_nonzero(y[:, 0])) == 3
    wide = M.linear(x[-4:], x[:, :].view(m, k), act="none")  # one answer against a table of 2^31 elements and more
    assert wide[3, [m - 1, 33_554_433, 5, 6]].tolist() == [64.0, 128.0, 192.0, 0.0]


def test_streams_and_graphs():
    g = torch.Generator("cuda").manual_seed(1)
    shapes = [(3, 100, 40), (70, 90, 512), (300, 300, 64)]
    data = [tuple(torch.randn(s, generator=g, device="cuda").half() for s in ((m, k), (n, k), (m, n)))
            for m, n, k in shapes]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [M.linear(x, w, residual=r, act="gelu", stream=side) for x, w, r in data]
    side.synchronize()
    for y, (x, w, r) in zip(got, data):
        assert torch.equal(y, M.linear(x, w, residual=r, act="gelu"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [(M.linear(x, w, residual=r, act="silu", keep_z=True), M.linear_grad(r, x, w, z=r, act="silu"))
                for x, w, r in data]
    for step in range(4):
        for t in data:
            for a in t:
                a.copy_(torch.randn(a.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for ((y, z), grads), (x, w, r) in zip(held, data):
            y2, z2 = M.linear(x, w, residual=r, act="silu", keep_z=True)
            assert torch.equal(y, y2) and torch.equal(z, z2)
            assert all(torch.equal(a, b) for a, b in zip(grads, M.linear_grad(r, x, w, z=r, act="silu")))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("k", [32, 100])
def test_scores(dtype, k):
    """The model's scores: for one user, a batch, users outside the model."""
    m, n = 400, 1111
    M.reset_options()
    M.set_option("dtype", dtype)
    M.init(m, n, k, 5)
    g = torch.Generator("cuda").manual_seed(k)
    P, Q = (ints(g, -3, 3, r, k).to(torch.float16 if dtype else torch.float32) for r in (m, n))
    M.set_factors(P, Q)
    bias = ints(g, -5, 5, n).to(P.dtype)
    for count in (0, 1, 30, 700):
        users = torch.randint(-1, m + 1, (count, 3), generator=g, device="cuda", dtype=torch.int32)[:, 0]
        there = ((users >= 0) & (users < m)).double()[:, None]
        rows = P[users.clamp(0, m - 1).long()].double() * there
        want = rows @ Q.double().t().contiguous()
        assert torch.equal(M.scores(users, n).double(), want.to(P.dtype).double())
        assert torch.equal(M.scores(users, n, bias=bias, act="relu"), torch.relu(want + bias.double()).to(P.dtype))
        out, store = placed(torch.zeros(count, n, device="cuda"), P.dtype, 4, 0, beside=2.0)
        M.scores(users, n, out=out)
        assert torch.equal(out, want.to(P.dtype))
        out.fill_(2.0)
        assert bool((store == 2.0).all())
    for bad in (dict(n=n + 1), dict(dtype=torch.bfloat16)):
        with pytest.raises(M.MfsgdError) as e:
            M.scores(**{**dict(users=users, n=n, dtype=P.dtype), **bad})
        assert e.value.code == M.EINVAL
    M.reset_options()
    M.finalize()
    with pytest.raises(M.MfsgdError) as e:
        M.scores(users, n, dtype=P.dtype)
    assert e.value.code == M.ESTATE


def test_binding_refuses():
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(5, 8, device="cuda")
    for bad in (w.cpu(), w.half(), w[0]):
        with pytest.raises(TypeError):
            M.linear(x, bad)
    for kw in (dict(w=w[:, :7]), dict(w=torch.zeros(8, 5, device="cuda").t()), dict(bias=torch.zeros(4, device="cuda")),
               dict(residual=torch.zeros(4, 4, device="cuda")), dict(out=torch.zeros(5, 5, device="cuda"))):
        with pytest.raises(ValueError):
            M.linear(**{**dict(x=x, w=w), **kw})
    with pytest.raises(KeyError):
        M.linear(x, w, act="tanh")
    dy = torch.zeros(4, 5, device="cuda")
    with pytest.raises(ValueError):
        M.linear_grad(dy, x, w, act="gelu")
    with pytest.raises(ValueError):
        M.linear_grad(dy.t(), x, w)
