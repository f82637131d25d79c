"""The lookup's gradient for tables of few rows, where each row has much of the
tokens: exact sums of small integers, and times beside those of more rows."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402

DTYPES = (torch.float32, torch.float16, torch.bfloat16)
ID = {torch.float32: "fp32", torch.float16: "fp16", torch.bfloat16: "bf16"}


@pytest.mark.parametrize("dtype", DTYPES, ids=ID.get)
@pytest.mark.parametrize("count,rows,k", [(2048, 3, 40), (2049, 1, 7), (2049, 32, 64), (2049, 33, 64), (4000, 10, 130),
                                          (5000, 3, 300), (8192, 127, 512), (8192, 128, 33), (8192, 2, 1000)])
def test_exact_sums(dtype, count, rows, k):
    g = torch.Generator("cuda").manual_seed(count + rows)
    dout = torch.randint(-4, 5, (count, k), generator=g, device="cuda").to(dtype)
    ids = torch.randint(-1, rows + 1, (count, 3), generator=g, device="cuda", dtype=torch.int32)[:, 1]
    there = (ids >= 0) & (ids < rows)
    want = torch.zeros(rows, k, dtype=torch.float64, device="cuda")
    want.index_add_(0, ids[there].long(), dout[there].double())
    got = M.embed_grad(dout, ids, rows, scale=0.25)
    assert torch.equal(got, (want / 4).to(dtype))
    base = torch.randint(-8, 9, (rows, k), generator=g, device="cuda").to(dtype)
    out = base.clone()
    M.embed_grad(dout, ids, rows, scale=0.25, out=out, accumulate=True)
    assert torch.equal(out, (base.double() + want / 4).to(dtype))


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


def test_few_rows_cost_no_more_than_twice_the_tokens():
    """8,192 tokens take at most 1.5 times what 16,384 do, for 3 rows and for 30."""
    dout = torch.ones(16_384, 512, device="cuda")
    for rows in (3, 30):
        ids = torch.randint(0, rows, (16_384,), device="cuda", dtype=torch.int32)
        few, many = (microseconds(lambda: M.embed_grad(dout[:c], ids[:c], rows)) for c in (8192, 16_384))
        assert few <= 1.5 * many, (rows, few, many)
