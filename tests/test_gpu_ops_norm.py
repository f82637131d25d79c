"""The global gradient norm, clipping and the clipped SGD update
(mfsgd_grad_norm, mfsgd_clip_grads, mfsgd_sgd_step) against 64 bits.

Norms are binary64 sums: off by at most n 2^-53 of the sum of squares, far
below the 1e-12 asked here.  Elements: c is rounded to binary32 once, each
product or sum of the formula once more, the result to its type."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def make(spec, seed, std=1.0):
    """Tensors of (elements, dtype, elements of shift from an aligned start)."""
    g = torch.Generator("cuda").manual_seed(seed)
    got = []
    for n, dtype, shift in spec:
        store = torch.zeros(n + shift + 8, dtype=dtype, device="cuda")
        t = store[shift:shift + n]
        t.copy_(torch.randn(n, generator=g, device="cuda") * std)
        got.append(t)
    return got


def norm64(ts):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in ts))


SPECS = {
    "nothing": [],
    "empty": [(0, F32, 0), (0, BF16, 0)],
    "one": [(1, F16, 0)],
    "small": [(32_000, F32, 0), (16_000, F32, 0), (7, F16, 1)],
    "odd": [(8191, F32, 1), (8192, F16, 3), (8193, BF16, 5), (0, F32, 0), (1, F32, 0), (2_000_003, F16, 1), (5, BF16, 0)],
    "many": [(17 + 61 * i % 4000, (F32, F16, BF16)[i % 3], i % 4) for i in range(300)],
    "large": [(17_000_000, F16, 0)] + [(3, F32, 0)] * 120 + [(40_000, BF16, 1)],
}


def check_clip(old, new, c64):
    c = float(np.float32(c64))
    for a, b in zip(old, new):
        eps = torch.finfo(a.dtype).eps / 2
        want = a.double() * c
        tol = want.abs() * (eps + 2.0**-24) * 1.01 + torch.finfo(a.dtype).smallest_normal * eps
        assert bool(((b.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("name", SPECS)
def test_norm_and_clip(name):
    ts = make(SPECS[name], len(name))
    old = [t.clone() for t in ts]
    want = norm64(ts)
    norm = M.grad_norm(ts)
    assert norm.dtype == torch.float64 and norm.dim() == 0
    assert abs(float(norm) - want) <= 1e-12 * want
    # above the norm: nothing changes
    assert float(M.clip_grads(ts, want * 1.001 + 1.0)) == float(norm)
    assert all(torch.equal(a, b) for a, b in zip(old, ts))
    assert float(M.clip_grads(ts, want / 3)) == float(norm)
    check_clip(old, ts, (want / 3) / want if want else 1.0)
    # a list laid out once gives the same
    again = M.TensorList(old)
    assert float(M.grad_norm(again)) == float(norm) == float(M.grad_norm(again))


@pytest.mark.parametrize("name", SPECS)
@pytest.mark.parametrize("bound", [0.4, math.inf])
def test_step(name, bound):
    g, p = make(SPECS[name], 1), make(SPECS[name], 2, std=0.5)
    old, grads = [t.clone() for t in p], [t.clone() for t in g]
    want = norm64(g)
    lr, lam = float(np.float32(0.03)), float(np.float32(0.05))
    norm = M.sgd_step(p, g, lr, lam=lam, max_norm=bound * want if bound < math.inf else math.inf)
    assert abs(float(norm) - want) <= 1e-12 * want
    c = float(np.float32(bound)) if bound < 1 else 1.0
    for a, b, d, d0 in zip(old, p, g, grads):
        assert torch.equal(d, d0)
        eps = torch.finfo(a.dtype).eps / 2
        new = a.double() - lr * (c * d.double() + lam * a.double())
        # c, c g, lam p, their sum, lr times it and the difference: 2^-24 of each's magnitude
        mag = a.double().abs() + lr * (4 * c * d.double().abs() + 3 * lam * a.double().abs()) + new.abs()
        tol = mag * 2.0**-24 * 1.05 + new.abs() * eps * 1.01 + torch.finfo(a.dtype).smallest_normal * eps
        assert bool(((b.double() - new).abs() <= tol).all())


def test_nothing_beside_the_tensors_is_written():
    store = torch.full((50_000,), 3.0, device="cuda")
    ts = [store[7:9001], store[9003:9004], store[9100:40_000]]
    M.clip_grads(ts, 1e-3)
    for a, b in ((0, 7), (9001, 9003), (9004, 9100), (40_000, 50_000)):
        assert bool((store[a:b] == 3.0).all())
    assert float(store[7:9001].max()) < 1e-3


def test_values_whose_squares_leave_binary32():
    for v, dtype in ((1e30, F32), (1e-30, F32), (1e38, BF16), (1e-38, BF16), (65504.0, F16), (6e-8, F16)):
        t = torch.full((1000,), v, dtype=dtype, device="cuda")
        x = float(t[0])
        want = x * math.sqrt(1000)
        assert abs(float(M.grad_norm([t])) - want) <= 1e-12 * want
        M.clip_grads([t], want / 2)
        assert abs(float(t[0]) - x / 2) <= x / 2 * (torch.finfo(dtype).eps + 2.0**-23) + 1e-45 * 2 + (
            6e-8 if dtype == F16 else 1e-40)


def test_special_norms():
    zeros = torch.zeros(100, device="cuda")
    assert float(M.clip_grads([zeros], 0.0)) == 0.0 and not bool(zeros.any())
    ones = torch.ones(100, device="cuda")
    M.clip_grads([ones], 0.0)
    assert not bool(ones.any())
    t = torch.ones(100, device="cuda")
    t[5] = math.inf
    assert float(M.clip_grads([t], 1.0)) == math.inf
    assert math.isnan(float(t[5])) and float(t[4]) == 0.0  # c = 0
    t = torch.ones(100, device="cuda")
    t[5] = math.nan
    p = torch.ones(100, device="cuda")
    assert math.isnan(float(M.sgd_step([p], [t], 0.1, max_norm=1.0)))
    assert bool(torch.isnan(p).all())
    t[5] = -math.inf
    assert float(M.clip_grads([t], math.inf)) == math.inf and float(t[4]) == 1.0  # inf <= inf: as they are


def test_an_infinite_bound_clips_nothing():
    for bad in (math.nan, math.inf):
        t = torch.ones(100, device="cuda")
        t[5] = bad
        p = torch.ones(100, device="cuda")
        norm = float(M.sgd_step([p], [t], 0.5))
        assert math.isnan(norm) or norm == math.inf
        assert not math.isfinite(float(p[5]))
        p[5] = 0.5
        assert bool((p == 0.5).all())
        M.clip_grads([t], math.inf)
        t[5] = 1.0
        assert bool((t == 1.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_larger_than_the_caches(dtype):
    """More than 256 MB, in odd pieces that start off their alignment."""
    each = 24_000_001 if dtype == F32 else 47_000_003
    spec = [(each, dtype, 1), (257, F16, 3), (each, dtype, 3), (each + 7, dtype, 2)]
    g, p = make(spec, 5), make(spec, 6, std=0.5)
    old, grads = [t.clone() for t in p], [t.clone() for t in g]
    want = norm64(g)
    lr, lam, bound = float(np.float32(0.03)), float(np.float32(0.05)), 0.5
    assert abs(float(M.grad_norm(g)) - want) <= 1e-12 * want
    assert abs(float(M.sgd_step(p, g, lr, lam=lam, max_norm=bound * want)) - want) <= 1e-12 * want
    for a, b, d in zip(old, p, g):
        eps = torch.finfo(a.dtype).eps / 2
        new = a.double() - lr * (bound * d.double() + lam * a.double())
        mag = a.double().abs() + lr * (4 * bound * d.double().abs() + 3 * lam * a.double().abs()) + new.abs()
        tol = mag * 2.0**-24 * 1.05 + new.abs() * eps * 1.01 + torch.finfo(a.dtype).smallest_normal * eps
        assert bool(((b.double() - new).abs() <= tol).all())
    M.clip_grads(g, want / 3)
    check_clip(grads, g, 1 / 3)


def test_one_tensor_twice_counts_twice():
    t = torch.full((50,), 2.0, device="cuda")
    assert abs(float(M.grad_norm([t, t])) - 20.0) < 1e-12


def test_streams_and_graphs():
    """Captured once, replayed on new values; another graph and eager calls of their own between."""
    ts, ps = make(SPECS["odd"], 3), make(SPECS["odd"], 4)
    grads, params = M.TensorList(ts), M.TensorList(ps)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norm = M.grad_norm(grads, stream=side)
    side.synchronize()
    assert float(norm) == float(M.grad_norm(grads))
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        n1 = M.sgd_step(params, grads, 0.5, lam=0.1, max_norm=1.0)
    with torch.cuda.graph(two):
        n2 = M.clip_grads(grads, 2.0)
    for step in range(4):
        for t, v in zip(ts, make(SPECS["odd"], 10 + step)):
            t.copy_(v)
        want = [t.clone() for t in ps]
        n0 = M.sgd_step(want, [t.clone() for t in ts], 0.5, lam=0.1, max_norm=1.0)
        one.replay()
        torch.cuda.synchronize()
        assert float(n0) == float(n1) and all(torch.equal(a, b) for a, b in zip(want, ps))
        want = [t.clone() for t in ts]
        n0 = M.clip_grads(want, 2.0)
        two.replay()
        torch.cuda.synchronize()
        assert float(n0) == float(n2) and all(torch.equal(a, b) for a, b in zip(want, ts))


def test_binding_refuses():
    t = torch.zeros(4, 8, device="cuda")
    for bad in ([t.cpu()], [t.t()], [t.double()], [t, 3]):
        with pytest.raises(TypeError):
            M.grad_norm(bad)
    with pytest.raises(ValueError):
        M.sgd_step([t], [], 0.1)
    with pytest.raises(M.MfsgdError) as e:
        M.clip_grads([t, t[1:2]], 1.0)
    assert e.value.code == M.EINVAL
    with pytest.raises(M.MfsgdError):
        M.sgd_step([t], [t], 0.1)
