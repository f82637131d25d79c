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
