"""Products whose matrices have unusual pitches, through the C ABI (the binding
passes the pitch of no matrix that is left out)."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402


@pytest.mark.parametrize("ld_out", [1 << 62, 1 << 61, -1, 0])
def test_the_pitch_of_a_matrix_left_out_counts_for_nothing(ld_out):
    """Y's rows are 8.4 MB apart, so its tiles pass 31 bits of offset, whatever stands for the pitches of the
    residual and of Z, which are NULL."""
    m, n, k, ldy = 300, 140, 64, (1 << 22) + 8
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randint(-3, 4, (m, k), generator=g, device="cuda").half()
    w = torch.randint(-3, 4, (n, k), generator=g, device="cuda").half()
    store = torch.full((m * ldy,), 7.0, dtype=torch.float16, device="cuda")
    y = store.view(m, ldy)[:, :n]
    work = torch.empty(max(M._bytes("mfsgd_linear_workspace", m, n, k, M.FP16), 256), dtype=torch.uint8, device="cuda")
    rc = M.lib().mfsgd_linear(x.data_ptr(), k, w.data_ptr(), k, None, None, ld_out, m, n, k, M.FP16, 0, y.data_ptr(),
                              ldy, None, ld_out, work.data_ptr(), work.numel(), M._current_stream(0))
    assert rc == M.OK, M.lib().mfsgd_last_error()
    assert torch.equal(y.double(), x.double() @ w.double().t().contiguous())
    y.fill_(7.0)
    assert bool((store == 7.0).all())


def columns(buf, rows, pitch, at, width):
    """A rows x width view of `buf`, its rows `pitch` apart from element `at` on."""
    return buf[:rows * pitch].view(rows, pitch)[:, at:at + width]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("pitch_out", [50, 100, 150])
def test_columns_of_one_buffer_do_not_overlap(dtype, pitch_out):
    """What is read and what is written lie between each other's rows, at equal pitches and at others: no overlap."""
    m, n, k, pitch = 90, 17, 20, 150
    g = torch.Generator("cuda").manual_seed(pitch_out)
    buf = torch.full((m * pitch + 64,), 5.0, dtype=dtype, device="cuda")
    x, out = columns(buf, m, pitch, 0, k), columns(buf, m, pitch_out, 25, n)
    w = torch.randint(-2, 3, (n, k), generator=g, device="cuda").to(dtype)
    x.copy_(torch.randint(-3, 4, (m, k), generator=g, device="cuda"))
    before = buf.clone()
    want = (columns(before, m, pitch, 0, k).double() @ w.double().t().contiguous()).to(dtype)
    columns(before, m, pitch_out, 25, n).copy_(want)
    M.linear(x, w, out=out)
    assert torch.equal(buf, before)
    ids = torch.randint(-1, m, (m,), generator=g, device="cuda", dtype=torch.int32)
    there = (ids >= 0)[:, None]
    columns(before, m, pitch_out, 25, n).copy_(x[ids.clamp(min=0).long(), :n] * there)
    M.embed(x[:, :n], ids, out=out)
    assert torch.equal(buf, before)


def test_overlap_is_refused():
    """Results that would be read before or after they are written."""
    t = torch.zeros(64, 64, device="cuda")
    ids = torch.arange(64, dtype=torch.int32, device="cuda")
    buf = torch.zeros(64 * 128, device="cuda")
    near, far = columns(buf, 64, 128, 0, 64), columns(buf, 64, 128, 63, 64)  # both hold column 63
    for call in (lambda: M.linear(t, t.clone(), out=t), lambda: M.linear(t.clone(), t, out=t),
                 lambda: M.linear(t, t, residual=near, out=far), lambda: M.embed(t, ids, out=t),
                 lambda: M.embed(near, ids, out=far), lambda: M.embed_grad(t, ids, 64, out=t),
                 lambda: M.embed_grad(t, ids, 64, out=t, accumulate=True)):
        with pytest.raises(M.MfsgdError) as e:
            call()
        assert e.value.code == M.EINVAL and "overlap" in str(e.value)
    assert not bool(t.any()) and not bool(buf.any())
    M.linear(t, t, residual=far, out=far)  # the residual may be the result itself
