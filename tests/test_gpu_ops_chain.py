"""The operators together, as a program uses them: a dense head on the model's
factors is trained -- rows looked up, two products, their gradients, the rows'
gradients, everything clipped by one norm and updated -- and every step is
compared with the same step in 64 bits by automatic differentiation.

Binary32 throughout; a step's results are held to 1e-4 of their largest
magnitude: at most 300 terms a sum (300 * 2^-24 = 2e-5 of the terms' magnitudes)
over four operators."""
import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_1610_05838_amd import mfsgd as M  # noqa: E402

USERS, ITEMS, K, HIDDEN, BATCH = 300, 90, 20, 33, 257


def near(a, b):
    return float((a.double() - b).abs().max()) <= 1e-4 * float(b.abs().max()) + 1e-9


class Head:
    """score(u, v) = w2 . gelu(W1 p_u + b1) + p_u . q_v's own part through the residual: 64-bit twin included."""

    def __init__(self):
        g = torch.Generator("cuda").manual_seed(12)
        self.P = torch.randn(USERS, K, generator=g, device="cuda") / math.sqrt(K)
        self.Q = torch.randn(ITEMS, K, generator=g, device="cuda") / math.sqrt(K)
        self.W1 = torch.randn(HIDDEN, K, generator=g, device="cuda") / math.sqrt(K)
        self.b1 = torch.randn(HIDDEN, generator=g, device="cuda") / 8
        self.W2 = torch.randn(K, HIDDEN, generator=g, device="cuda") / math.sqrt(HIDDEN)
        self.params = [self.P, self.Q, self.W1, self.b1, self.W2]

    def step(self, users, items, target, lr, lam, bound):
        """One training step; the gradients before clipping and the norm."""
        pu = M.embed(self.P, users)
        qv = M.embed(self.Q, items)
        h, z = M.linear(pu, self.W1, bias=self.b1, act="gelu", keep_z=True)
        t = M.linear(h, self.W2, residual=pu)  # the users' rows, transformed
        e = (t * qv).sum(1, keepdim=True) - target[:, None]
        dt, dq = e * qv, e * t
        dh, dW2, _ = M.linear_grad(dt, h, self.W2, dbias=False)
        dp, dW1, db1 = M.linear_grad(dh, pu, self.W1, z=z, act="gelu")
        dp = dp + dt
        grads = [M.embed_grad(dp, users, USERS), M.embed_grad(dq, items, ITEMS), dW1, db1, dW2]
        norm = M.sgd_step(self.params, grads, lr, lam=lam, max_norm=bound)
        return grads, norm


def step64(params, users, items, target, lr, lam, bound):
    P, Q, W1, b1, W2 = (p.double().requires_grad_(True) for p in params)
    there = (users >= 0) & (users < USERS)
    pu = P[torch.where(there, users, 0).long()] * there[:, None]
    h = torch.nn.functional.gelu(pu @ W1.t() + b1)
    t = h @ W2.t() + pu
    e = (t * Q[items.long()]).sum(1) - target.double()
    grads = torch.autograd.grad(0.5 * e.square().sum(), (P, Q, W1, b1, W2))
    norm = torch.sqrt(sum(g.square().sum() for g in grads))
    c = min(1.0, bound / float(norm))
    new = [(p - lr * (c * g + lam * p)).detach() for p, g in zip((P, Q, W1, b1, W2), grads)]
    return grads, norm, new


def batch(g):
    users = torch.randint(-1, USERS, (BATCH,), generator=g, device="cuda", dtype=torch.int32)  # -1: unknown user
    items = torch.randint(0, ITEMS, (BATCH, 3), generator=g, device="cuda", dtype=torch.int32)[:, 1]
    return users, items, torch.randn(BATCH, generator=g, device="cuda")


def test_training_steps():
    head, g = Head(), torch.Generator("cuda").manual_seed(3)
    for n, bound in enumerate((1.0, 1e9, 5.0)):
        users, items, target = batch(g)
        want, norm64, new = step64(head.params, users, items, target, 0.05, 0.01, bound)
        grads, norm = head.step(users, items, target, 0.05, 0.01, bound)
        assert near(norm[None], norm64[None].detach())
        for a, b in zip(grads, want):
            assert near(a, b)
        for a, b in zip(head.params, new):
            assert near(a, b), n


def test_training_steps_captured():
    """The whole step in a graph: the same bits as the eager step on the same batches."""
    eager, held = Head(), Head()
    g = torch.Generator("cuda").manual_seed(4)
    users, items, target = batch(g)
    static = [t.clone() for t in (users, torch.stack([items] * 3, 1), target)]
    graph = torch.cuda.CUDAGraph()
    keep = [p.clone() for p in held.params]
    with torch.cuda.graph(graph):
        grads, norm = held.step(static[0], static[1][:, 1], static[2], 0.02, 0.0, 2.0)
    for p, k in zip(held.params, keep):
        assert torch.equal(p, k)  # captured, not run
    for _ in range(4):
        users, items, target = batch(g)
        static[0].copy_(users)
        static[1][:, 1].copy_(items)
        static[2].copy_(target)
        graph.replay()
        torch.cuda.synchronize()
        want, n2 = eager.step(users, items, target, 0.02, 0.0, 2.0)
        assert float(norm) == float(n2)
        assert all(torch.equal(a, b) for a, b in zip(grads, want))
        assert all(torch.equal(a, b) for a, b in zip(eager.params, held.params))


def test_the_library_model_learns_from_a_batch():
    """A batch step on the library's own factors: rows out, their gradients clipped, added back in place; then
    scores and the test RMSE see the new factors."""
    M.reset_options()
    M.init(USERS, ITEMS, K, 7)
    P, Q = M.get_factors(USERS, ITEMS, K)
    g = torch.Generator("cuda").manual_seed(5)
    samples = torch.stack([torch.randint(0, USERS, (BATCH,), generator=g, device="cuda", dtype=torch.int32),
                           torch.randint(0, ITEMS, (BATCH,), generator=g, device="cuda", dtype=torch.int32),
                           torch.rand(BATCH, generator=g, device="cuda").view(torch.int32)], 1).contiguous()
    u, v, r = samples[:, 0], samples[:, 1], samples[:, 2].contiguous().view(torch.float32)
    pu, qv = M.rows(M.P, u, K), M.rows(M.Q, v, K)
    e = r - (pu * qv).sum(1)
    dp, dq = -e[:, None] * qv, -e[:, None] * pu
    norm = M.clip_grads([dp, dq], 0.5)
    M.add_rows(M.P, dp, u, -0.1)
    M.add_rows(M.Q, dq, v, -0.1)
    P64, Q64 = P.double(), Q.double()
    e64 = r.double() - (P64[u.long()] * Q64[v.long()]).sum(1)
    gp, gq = -e64[:, None] * Q64[v.long()], -e64[:, None] * P64[u.long()]
    n64 = math.sqrt(float(gp.square().sum() + gq.square().sum()))
    assert abs(float(norm) - n64) <= 1e-5 * n64
    c = min(1.0, 0.5 / n64)
    P64.index_add_(0, u.long(), -0.1 * c * gp)
    Q64.index_add_(0, v.long(), -0.1 * c * gq)
    P2, Q2 = M.get_factors(USERS, ITEMS, K)
    assert near(P2, P64) and near(Q2, Q64) and not torch.equal(P, P2)
    s = M.scores(u[:40], ITEMS)
    assert near(s, P64[u[:40].long()] @ Q64.t())
    want = math.sqrt(float((r.double() - (P64[u.long()] * Q64[v.long()]).sum(1)).square().mean()))
    assert abs(M.rmse(samples) - want) <= 1e-5 * want
    M.finalize()


def test_two_streams_at_once():
    """Different operators enqueued in turn on two streams, nothing waited for between: what each gives alone."""
    g = torch.Generator("cuda").manual_seed(6)
    ids = torch.randint(-1, 500, (20_000,), generator=g, device="cuda", dtype=torch.int32)
    rows = torch.randn(20_000, 72, generator=g, device="cuda")
    x, w, dy = (torch.randn(a, b, generator=g, device="cuda") for a, b in ((3000, 200), (64, 200), (3000, 64)))
    want_rows = M.embed_grad(rows, ids, 500)
    want = M.linear_grad(dy, x, w)
    want_norm = float(M.grad_norm([rows, x, w]))
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for n in range(12):
        a, b = (one, two) if n % 2 else (two, one)
        got.append((M.embed_grad(rows, ids, 500, stream=a), M.linear_grad(dy, x, w, stream=b),
                    M.grad_norm([rows, x, w], stream=a)))
    torch.cuda.synchronize()
    for table, grads, norm in got:
        assert torch.equal(table, want_rows) and float(norm) == want_norm
        assert all(torch.equal(p, q) for p, q in zip(grads, want))
