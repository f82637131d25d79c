"""The product's gradient where its two products differ much in size or depth:
dX has the batch as its rows, dW as its depth.

Small integers again, whose sums are exact in any order.  Times are compared
with those of the same work cut otherwise, with room for a factor."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402

DTYPES = (torch.float32, torch.float16, torch.bfloat16)
ID = {torch.float32: "fp32", torch.float16: "fp16", torch.bfloat16: "bf16"}


def ints(g, low, high, *shape):
    return torch.randint(low, high + 1, shape, generator=g, device="cuda")


def exact(m, n, k, dtype, act="relu"):
    g = torch.Generator("cuda").manual_seed(m + n + k)
    x, w, dy, z = (ints(g, -2, 2, *s).to(dtype) for s in ((m, k), (n, k), (m, n), (m, n)))
    dz = dy.double() * (z > 0)
    dx, dw, db = M.linear_grad(dy, x, w, z=z, act=act)
    assert torch.equal(dx, (dz @ w.double()).to(dtype))
    assert torch.equal(dw, (dz.t().contiguous() @ x.double()).to(dtype))
    assert torch.equal(db, dz.sum(0).to(dtype))
    again = M.linear_grad(dy, x, w, z=z, act=act)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw) and torch.equal(again[2], db)


def microseconds(call):
    for _ in range(3):
        call()
    best = float("inf")
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(5):
            call()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) * 200.0)
    return best


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("m,n,k", [(2800, 2790, 2816), (3100, 2490, 2810), (24_576, 512, 512), (24_600, 500, 520),
                                   (6144, 512, 2048)])
def test_gradients_of_large_layers(dtype, m, n, k):
    """The first two run in tiles of 256 rows, both products and the bias in one launch; the others have so long a
    batch that dW's few tiles are cut along their depth."""
    exact(m, n, k, dtype)


@pytest.mark.parametrize("m,n,k", [(24_576, 512, 512), (16_384, 768, 768), (12_288, 1024, 1024)])
def test_a_long_batch_costs_its_work(m, n, k):
    """One gradient of a batch takes at most 1.5 times those of its halves together."""
    g = torch.Generator("cuda").manual_seed(1)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, k), (n, k), (m, n)))
    whole = microseconds(lambda: M.linear_grad(dy, x, w))
    half = microseconds(lambda: M.linear_grad(dy[:m // 2], x[:m // 2], w))
    assert whole <= 1.5 * 2 * half, (whole, half)


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("m,n,k", [(1, 40, 200_000), (16, 100, 70_001), (16, 2048, 8192), (16, 2049, 8192), (3, 2000, 8191),
                                   (5, 1, 9000), (16, 1, 100_003)])
def test_few_rows_of_a_deep_product(dtype, m, n, k):
    g = torch.Generator("cuda").manual_seed(m + n + k)
    x, w = (ints(g, -2, 2, s, k).to(dtype) for s in (m, n))
    bias, res = ints(g, -9, 9, n).to(dtype), ints(g, -9, 9, m, n).to(dtype)
    want = x.double() @ w.double().t().contiguous() + bias.double()
    y, z = M.linear(x, w, bias=bias, residual=res, act="relu", keep_z=True)
    assert torch.equal(z, want.to(dtype)) and torch.equal(y, (torch.relu(want) + res.double()).to(dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("m,n,k", [(100_000, 1, 128), (100_001, 16, 100), (30_000, 17, 128), (8192, 2, 2500), (8191, 9, 40)])
def test_gradient_of_few_outputs_over_a_long_batch(dtype, m, n, k):
    exact(m, n, k, dtype)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=ID.get)
def test_few_rows_cost_no_more_than_many(dtype):
    """16 outputs over a batch of 100,000 take at most twice what 17 do, forward and backward (1.2 times; without slices
    of the depth 3 to 8)."""
    g = torch.Generator("cuda").manual_seed(2)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").to(dtype) for s in ((100_000, 128), (17, 128), (100_000, 17)))
    xt, dyt = x.t().contiguous(), dy.t().contiguous()
    few, many = (microseconds(lambda: M.linear(dyt[:n], xt)) for n in (16, 17))
    assert few <= 2.0 * many, (few, many)
    few, many = (microseconds(lambda: M.linear_grad(dy[:, :n], x, w[:n])) for n in (16, 17))
    assert few <= 2.0 * many, (few, many)


def test_a_bias_of_more_columns_than_one_launch_takes():
    """2^29 columns: 64 to a workgroup of 512 threads are more threads than a grid counts."""
    n = (1 << 29) + 100
    dy = torch.zeros(2, n, dtype=torch.float16, device="cuda")
    dy[:, -1], dy[1, 0], dy[0, 1 << 28], dy[1, (1 << 29) - 1] = 2.0, 3.0, 5.0, 7.0
    x, w = torch.zeros(2, 0, dtype=dy.dtype, device="cuda"), torch.zeros(n, 0, dtype=dy.dtype, device="cuda")
    _, _, db = M.linear_grad(dy, x, w, dx=False, dw=False)
    at = torch.tensor([0, 1, 1 << 28, (1 << 29) - 1, n - 1], device="cuda")
    assert db[at].tolist() == [3.0, 0.0, 5.0, 7.0, 4.0] and int(torch.count_nonzero(db)) == 4


def test_more_rows_than_one_launch_takes():
    """2^29 rows: more tiles than a launch has workgroups, and rows of the exchanged matrices that pass 32 bits."""
    m = (1 << 29) + 100
    x = torch.zeros(m, 2, dtype=torch.float16, device="cuda")
    at = torch.tensor([0, 1 << 28, (1 << 29) - 1, 1 << 29, m - 1], device="cuda")
    x[at] = torch.tensor([[1, 2], [3, 4], [5, 6], [7, 8], [9, 10]], dtype=torch.float16, device="cuda")
    w = torch.tensor([[2.0, -1.0]], dtype=torch.float16, device="cuda")
    y = M.linear(x, w)
    assert y[at, 0].tolist() == [0.0, 2.0, 4.0, 6.0, 8.0] and int(torch.count_nonzero(y)) == 4
    y[0] = 1.0
    dx, dw, db = M.linear_grad(y, x, w)
    assert dx[at].tolist() == [[2.0 * d, -d] for d in (1.0, 2.0, 4.0, 6.0, 8.0)]
    assert int(torch.count_nonzero(dx[:, 0])) == 5
    assert dw.tolist() == [[1.0 + 6 + 20 + 42 + 72, 2.0 + 8 + 24 + 48 + 80]] and db.tolist() == [21.0]


def test_captured_with_slices():
    """Forms that join slices, in a graph: every replay sees the inputs as they are then."""
    g = torch.Generator("cuda").manual_seed(3)
    data = [tuple(torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, k), (n, k), (m, n)))
            for m, n, k in ((3, 200, 9000), (20_000, 2, 130), (24_576, 256, 256))]

    def run():
        return [(M.linear(x, w, residual=r, act="gelu"), *M.linear_grad(r, x, w, z=r, act="gelu")) for x, w, r in data]

    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for _ in range(4):
        for t in data:
            for a in t:
                a.copy_(torch.randn(a.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, run()):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
