"""The operators beside autograd: it does not see them, but it must notice that
a tensor whose value it saved was changed in place by one."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402


def square(n):
    return torch.ones(n, n, device="cuda")


IDS = [0, 3, 3, -1, 2, 1, 5, 7]


def ids():
    return torch.tensor(IDS, dtype=torch.int32, device="cuda")


CHANGES = {
    "embed": lambda t: M.embed(square(8), ids(), out=t),
    "embed_grad": lambda t: M.embed_grad(square(8), ids(), 8, out=t),
    "embed_grad added": lambda t: M.embed_grad(square(8), ids(), 8, out=t, accumulate=True),
    "linear": lambda t: M.linear(square(8), square(8), out=t),
    "linear onto its residual": lambda t: M.linear(square(8), square(8), residual=t, out=t),
    "clip_grads": lambda t: M.clip_grads([square(3), t], 0.5),
    "clip_grads of a list": lambda t: M.clip_grads(M.TensorList([t, square(3)]), 0.5),
    "sgd_step": lambda t: M.sgd_step([t], [square(8)], 0.1),
}


@pytest.mark.parametrize("name", CHANGES)
@pytest.mark.parametrize("leaf", [True, False], ids=["leaf", "result"])
def test_a_saved_tensor_that_was_changed_is_noticed(name, leaf):
    t = square(8).requires_grad_(True)
    saved = t if leaf else t * 2.0
    y = saved.square().sum()
    y.backward(retain_graph=True)
    CHANGES[name](saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_on_the_model():
    M.reset_options()
    M.init(9, 8, 8, 1)
    for call in (lambda t: M.rows(M.Q, ids(), 8, out=t), lambda t: M.scores(ids(), 8, out=t)):
        t = square(8).requires_grad_(True)
        y = t.square().sum()
        call(t)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    M.finalize()


def test_what_is_read_stays_as_saved():
    """Parameters and gradients that a call only reads do not count as changed."""
    t, g = square(8).requires_grad_(True), square(8).requires_grad_(True)
    y = (t.square() * g).sum()
    M.embed(t, ids())
    M.embed_grad(t, ids(), 8)
    M.linear(t, g, residual=t, act="gelu", keep_z=True)
    M.linear_grad(t, g, g)
    M.grad_norm([t, g])
    M.sgd_step([square(8)], [t], 0.1)
    y.backward()
    assert torch.equal(t.grad, 2.0 * t.detach())


def test_results_require_no_gradient():
    t = square(8).requires_grad_(True)
    for got in (M.embed(t, ids()), M.embed_grad(t, ids(), 8), M.linear(t, t), M.linear_grad(t, t, t)[0], M.grad_norm([t])):
        assert not got.requires_grad
    with torch.inference_mode():
        frozen = square(8)
        M.linear(frozen, frozen, out=square(8))  # such tensors have no version to count
        M.clip_grads([frozen], 0.5)
