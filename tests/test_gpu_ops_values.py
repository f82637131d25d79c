"""Values of the activations and their slopes where formulas cancel or overflow:
infinities, the lower tail of gelu, the upper tail of sigmoid's slope.

x times a single weight of 1 makes any value of a type the pre-activation, and
dY = 1 makes dX the slope, each rounded once: by at most eps / 2 of itself, or
half the smallest number of the type."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402

DTYPES = (torch.float32, torch.float16, torch.bfloat16)
ID = {torch.float32: "fp32", torch.float16: "fp16", torch.bfloat16: "bf16"}
INF = math.inf


def through(z, act):
    """act(z) and act'(z) of a vector, by the product and its gradient."""
    x, one = z[:, None].contiguous(), torch.ones(1, 1, dtype=z.dtype, device="cuda")
    y = M.linear(x, one, act=act)
    dx, _, _ = M.linear_grad(torch.ones_like(x), x, one, z=x, act=act)
    return y[:, 0].double(), dx[:, 0].double()


def within(got, want, dtype, own):
    """own: the function's relative error before the rounding."""
    f = torch.finfo(dtype)
    return bool(((got - want).abs() <= want.abs() * (f.eps / 2 + own * 1.01) + f.smallest_normal * f.eps / 2 * 1.01).all())


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
def test_slopes_at_infinity(dtype):
    """The limits, 0 and 1: a kept Z is infinite where the type did not hold it."""
    z = torch.tensor([-INF, INF] * 20, dtype=dtype, device="cuda")
    for act, above in (("relu", 1.0), ("sigmoid", 0.0), ("silu", 1.0), ("gelu", 1.0)):
        _, slope = through(z, act)
        assert bool((slope[::2] == 0.0).all()) and bool((slope[1::2] == above).all()), (act, slope[:2])


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("m", [5, 40])
def test_a_layer_whose_pre_activation_leaves_binary16(act, m):
    """Z = -70000 and 70000 are kept as infinities; the result and every gradient are those of the finite values."""
    x = torch.full((m, 7), 100.0, dtype=torch.float16, device="cuda")
    w = torch.full((20, 7), 100.0, dtype=torch.float16, device="cuda")
    w[::2] *= -1.0
    y, z = M.linear(x, w, act=act, keep_z=True)
    assert bool((z[:, ::2] == -INF).all()) and bool((z[:, 1::2] == INF).all())
    assert bool((y[:, ::2] == 0.0).all()) and bool((y[:, 1::2] == INF).all())
    dx, dw, db = M.linear_grad(torch.ones_like(y), x, w, z=z, act=act)
    assert bool((dx == 1000.0).all())
    assert bool((dw[::2] == 0.0).all()) and bool((dw[1::2] == 100.0 * m).all())
    assert bool((db[::2] == 0.0).all()) and bool((db[1::2] == m).all())


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("act", ["sigmoid", "silu", "gelu"])
def test_a_column_masked_by_minus_infinity_is_zero(dtype, act):
    """A bias of -inf, or of the lowest value of the type, takes a column out."""
    for m, n, k in ((3, 50, 24), (200, 300, 72), (40, 30, 13)):
        x, w = torch.ones(m, k, dtype=dtype, device="cuda"), torch.ones(n, k, dtype=dtype, device="cuda")
        bias = torch.zeros(n, dtype=dtype, device="cuda")
        bias[2::3], bias[1::3] = -INF, torch.finfo(dtype).min
        y = M.linear(x, w, bias=bias, act=act)
        assert bool((y[:, 2::3] == 0.0).all()) and bool((y[:, 1::3] == 0.0).all()) and bool((y[:, ::3] > 0.5).all())
        bias[2::3] = math.nan
        assert bool(torch.isnan(M.linear(x, w, bias=bias, act=act)[:, 2::3]).all())


def tail_points(dtype, low, high):
    z = torch.linspace(low, high, 3001, device="cuda").to(dtype)
    return z, z.double()


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
def test_gelu_lower_tail(dtype):
    """Relative to its own size.  16 bits: the normal distribution's tail to 3e-5; all: z^2 2^-22 of exp(-z^2 / 2),
    whose argument is rounded, and a few roundings."""
    z, z64 = tail_points(dtype, -12.5, -1.5)
    cdf = 0.5 * torch.erfc(-z64 / math.sqrt(2.0))
    density = torch.exp(-0.5 * z64 * z64) / math.sqrt(2.0 * math.pi)
    own = (z64 * z64 + 16.0) * 2.0**-22 + (0.0 if dtype == torch.float32 else 3e-5)
    y, slope = through(z, "gelu")
    assert within(y, z64 * cdf, dtype, own)
    # the slope's two terms have different signs: each is off by `own` of itself
    want = cdf + z64 * density
    assert within(slope, want, dtype, own * ((cdf + z64.abs() * density) / want.abs()))


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
def test_sigmoid_slope_in_both_tails(dtype):
    """exp(-|z|) / (1 + exp(-|z|))^2, relative to its own size: the exponential to (|z| + 2) 2^-23, a few roundings."""
    for low, high in ((-16.0, -1.0), (1.0, 16.0), (20.0, 80.0)):
        z, z64 = tail_points(dtype, low, high)
        e = torch.exp(-z64.abs())
        _, slope = through(z, "sigmoid")
        assert within(slope, e / (1.0 + e)**2, dtype, (z64.abs() + 16.0) * 2.0**-22)
