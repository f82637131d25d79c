"""The operators around the trained factors that this library is timed on:
looking rows of a table up and the gradient of that, products with bias,
activation and residual (scores of users against items, dense layers on top of
the factors) and their gradient, and the gradients' global norm with clipping,
in place and inside the update.

Tables have the sizes of ``paper_1610_05838_amd.datagen``'s workloads or generic
ones.  Ids are drawn Zipf-like through a random permutation (popular users and
items all over the table), as in the seeded workloads; -1 stands for no row
(padding).
"""
import math
import random

import torch

own = False

DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
ACTS = ("none", "relu", "sigmoid", "silu", "gelu")


def listed():
    return [
        # one page of a server's answer: the rows of 50 items, binary16
        dict(name="embed_page", op="embed", rows=17_770, k=128, count=50, dtype="fp16", scale=1.0, zipf=True, pad=0.0,
             column=False),
        # the users of the Netflix-shaped test set, ids read out of the 12-byte samples
        dict(name="embed_test_users", op="embed", rows=480_189, k=128, count=1_408_395, dtype="fp32", scale=1.0,
             zipf=True, pad=0.0, column=True),
        # a ragged batch padded to one length, rows scaled by sqrt(k), bfloat16
        dict(name="embed_padded_batch", op="embed", rows=50_003, k=500, count=40_960, dtype="bf16",
             scale=math.sqrt(500.0), zipf=True, pad=0.3, column=False),
        # the item gradient of a large batch of ratings: a few items hold much of it
        dict(name="grad_hot_items", op="embed_grad", rows=17_770, k=128, count=262_144, dtype="fp16", scale=1.0,
             zipf=True, pad=0.0, column=True, accumulate=False),
        # the gradient of a wide table under a long padded batch, bfloat16
        dict(name="grad_wide_table", op="embed_grad", rows=50_003, k=512, count=131_072, dtype="bf16", scale=0.5,
             zipf=True, pad=0.1, column=False, accumulate=False),
        # an online batch's row updates, added to the table in place (an SGD step of the touched rows)
        dict(name="grad_online_update", op="embed_grad", rows=50_000, k=64, count=4_001, dtype="fp32", scale=-1e-5,
             zipf=True, pad=0.0, column=True, accumulate=True),
        # one user's scores against all items of the Netflix shape, binary16 (latency)
        dict(name="score_one_user", op="linear", M=1, N=17_770, K=128, dtype="fp16", act="none", bias=True,
             residual=False, keep_z=False),
        # a batch of users against all items of the Hugewiki shape: the output is the work
        dict(name="score_users", op="linear", M=2_048, N=39_780, K=128, dtype="fp16", act="sigmoid", bias=True,
             residual=False, keep_z=False),
        # a dense layer in training: bias, gelu, residual, the pre-activation kept
        dict(name="layer_train", op="linear", M=4_096, N=4_096, K=4_096, dtype="bf16", act="gelu", bias=True,
             residual=True, keep_z=True),
        # the gradient of a dense layer
        dict(name="layer_grad", op="linear_grad", M=4_096, N=2_048, K=2_048, dtype="bf16", act="gelu"),
        # the gradient of a small layer of odd sizes in binary32
        dict(name="layer_grad_odd", op="linear_grad", M=1_001, N=333, K=500, dtype="fp32", act="silu"),
        # the clipped update of the Netflix-shaped factors and of the 70 tensors of a head on them
        dict(name="step_factors_head", op="step", m=480_189, n=17_770, k=128, head=70, width=512, dtype="fp32",
             clip=0.5),
    ]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "linear", "linear", "linear_grad", "step"))
    dt = rng.choice(("fp32", "fp16", "bf16"))
    if op in ("embed", "embed_grad"):
        k = rng.choice((_log(rng, 1, 512), rng.choice((32, 64, 100, 128, 256, 300, 512))))
        rows = _log(rng, 100, 500_000)
        count = min(_log(rng, 1, 1_400_000), 100_000_000 // k)
        c = dict(op=op, rows=rows, k=k, count=count, dtype=dt, scale=rng.choice((1.0, round(rng.uniform(0.1, 20.0), 3))),
                 zipf=rng.random() < 0.7, pad=rng.choice((0.0, 0.0, 0.2)), column=rng.random() < 0.5)
        if op == "embed_grad":
            c["accumulate"] = dt == "fp32" and rng.random() < 0.3
            if c["accumulate"]:
                c["scale"] = -1e-5
        return c
    if op == "linear":
        M = rng.choice((_log(rng, 1, 64), _log(rng, 1, 4_096)))
        N, K = _log(rng, 16, 40_000), _log(rng, 16, 4_096)
        N = max(1, min(N, 60_000_000_000 // (M * K)))
        return dict(op=op, M=M, N=N, K=K, dtype=dt, act=rng.choice(ACTS), bias=rng.random() < 0.7,
                    residual=rng.random() < 0.4, keep_z=rng.random() < 0.3)
    if op == "linear_grad":
        M, N, K = _log(rng, 1, 4_096), _log(rng, 16, 4_096), _log(rng, 16, 2_048)
        M = max(1, min(M, 16_000_000_000 // (N * K)))
        return dict(op=op, M=M, N=N, K=K, dtype=dt, act=rng.choice(ACTS))
    return dict(op=op, m=_log(rng, 100, 400_000), n=_log(rng, 100, 17_770), k=rng.choice((32, 50, 100, 128)),
                head=rng.randint(0, 70), width=_log(rng, 16, 512), dtype=dt, clip=rng.choice((0.5, 2.0)))


def _gen(seed):
    return torch.Generator("cuda").manual_seed(int(seed))


def _normal(g, *shape, dtype=torch.float32, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _ids(g, case):
    rows, count = case["rows"], case["count"]
    u = torch.rand(count, generator=g, device="cuda", dtype=torch.float64)
    if case["zipf"]:  # P(rank r) about 1 / r
        rank = (torch.exp(u * math.log(rows + 1.0)) - 1.0).long().clamp_(0, rows - 1)
    else:
        rank = (u * rows).long().clamp_(0, rows - 1)
    ids = torch.randperm(rows, generator=g, device="cuda")[rank].int()
    if case["pad"]:
        ids[torch.rand(count, generator=g, device="cuda") < case["pad"]] = -1
    if case["column"]:  # the u column of (u, v, r) records
        records = torch.zeros(count, 3, dtype=torch.int32, device="cuda")
        records[:, 0] = ids
        return records[:, 0]
    return ids


def _sizes(case):
    """Elements of every tensor of a step: the two tables, then a head's weights and biases."""
    rng, w = random.Random(case["head"] * 1_000_003 + case["width"]), case["width"]
    head = [rng.choice((w * w, w, w, w * (w // 2 + 1), 1)) for _ in range(case["head"])]
    return [case["m"] * case["k"], case["n"] * case["k"]] + head


def _views(flat, sizes):
    got, at = [], 0
    for s in sizes:
        got.append(flat[at:at + s])
        at += s
    return got


def prepare(case, seed):
    g, op, dt = _gen(seed), case["op"], DT[case["dtype"]]
    st = dict(case=case)
    if op == "embed":
        st["table"] = _normal(g, case["rows"], case["k"], dtype=dt, std=1.0 / math.sqrt(case["k"]))
        st["ids"] = _ids(g, case)
    elif op == "embed_grad":
        st["dout"] = _normal(g, case["count"], case["k"], dtype=dt)
        st["ids"] = _ids(g, case)
        if case["accumulate"]:
            st["table"] = _normal(g, case["rows"], case["k"], dtype=dt, std=1.0 / math.sqrt(case["k"]))
    elif op in ("linear", "linear_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        st["x"] = _normal(g, M, K, dtype=dt)
        st["w"] = _normal(g, N, K, dtype=dt, std=1.0 / math.sqrt(K))
        if op == "linear":
            st["bias"] = _normal(g, N, dtype=dt) if case["bias"] else None
            st["residual"] = _normal(g, M, N, dtype=dt) if case["residual"] else None
        else:
            st["z"] = _normal(g, M, N, dtype=dt)
            st["dy"] = _normal(g, M, N, dtype=dt)
    else:
        sizes = _sizes(case)
        st["flat_p"] = _normal(g, sum(sizes), dtype=dt, std=0.1)
        st["flat_g"] = _normal(g, sum(sizes), dtype=dt, std=0.01)
        st["p"], st["g"] = _views(st["flat_p"], sizes), _views(st["flat_g"], sizes)
        # half the norm (always clipped) or twice it (never)
        st["max_norm"] = case["clip"] * 0.01 * math.sqrt(sum(sizes))
        st["lr"], st["lam"] = 1e-4, 0.05
        if own:
            from paper_1610_05838_amd import mfsgd
            st["params"], st["grads"] = mfsgd.TensorList(st["p"]), mfsgd.TensorList(st["g"])
    return st


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0.0).to(z.dtype)
    if act == "sigmoid":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 - s)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return torch.ones_like(z)


def _run_own(st):
    from paper_1610_05838_amd import mfsgd
    case, op = st["case"], st["case"]["op"]
    if op == "embed":
        return mfsgd.embed(st["table"], st["ids"], scale=case["scale"])
    if op == "embed_grad":
        if case["accumulate"]:
            return mfsgd.embed_grad(st["dout"], st["ids"], case["rows"], scale=case["scale"], out=st["table"],
                                    accumulate=True)
        return mfsgd.embed_grad(st["dout"], st["ids"], case["rows"], scale=case["scale"])
    if op == "linear":
        got = mfsgd.linear(st["x"], st["w"], bias=st["bias"], residual=st["residual"], act=case["act"],
                           keep_z=case["keep_z"])
        return dict(y=got[0], z=got[1]) if case["keep_z"] else dict(y=got)
    if op == "linear_grad":
        dx, dw, dbias = mfsgd.linear_grad(st["dy"], st["x"], st["w"], z=st["z"], act=case["act"])
        return dict(dx=dx, dw=dw, dbias=dbias)
    norm = mfsgd.sgd_step(st["params"], st["grads"], st["lr"], lam=st["lam"], max_norm=st["max_norm"])
    return dict(p=st["flat_p"], norm=norm)


def run(st):
    if own:
        return _run_own(st)
    case, op, dt = st["case"], st["case"]["op"], DT[st["case"]["dtype"]]
    if op == "embed":
        ids = st["ids"].long()
        there = (ids >= 0) & (ids < case["rows"])
        rows = st["table"][torch.where(there, ids, 0)].float() * case["scale"]
        return torch.where(there[:, None], rows, 0.0).to(dt)
    if op == "embed_grad":
        ids = st["ids"].long()
        there = (ids >= 0) & (ids < case["rows"])
        sums = torch.zeros(case["rows"], case["k"], device="cuda")
        sums.index_add_(0, torch.where(there, ids, 0), torch.where(there[:, None], st["dout"].float(), 0.0))
        sums *= case["scale"]
        if case["accumulate"]:
            return st["table"].copy_(st["table"].float() + sums)
        return sums.to(dt)
    if op == "linear":
        z = st["x"].float() @ st["w"].float().T
        if case["bias"]:
            z = z + st["bias"].float()
        y = _act(z, case["act"])
        if case["residual"]:
            y = y + st["residual"].float()
        return dict(y=y.to(dt), z=z.to(dt)) if case["keep_z"] else dict(y=y.to(dt))
    if op == "linear_grad":
        dz = st["dy"].float() * _slope(st["z"].float(), case["act"])
        return dict(dx=(dz @ st["w"].float()).to(dt), dw=(dz.T @ st["x"].float()).to(dt), dbias=dz.sum(0).to(dt))
    norm = torch.stack([g.double().square().sum() for g in st["g"]]).sum().sqrt()
    c = torch.clamp(st["max_norm"] / norm, max=1.0).float()
    new = [p.float() - st["lr"] * (c * g.float() + st["lam"] * p.float()) for p, g in zip(st["p"], st["g"])]
    st["flat_p"].copy_(torch.cat(new))
    return dict(p=st["flat_p"], norm=norm)


def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op in ("embed", "embed_grad"):
        rows, k, count = case["rows"], case["k"], case["count"]
        live = count * (1.0 - case["pad"])
        if case["zipf"]:  # distinct rows among the drawn: rank r is missed with probability exp(-live / (h r))
            h, steps, seen = math.log(rows + 1.0), 400, 0.0
            for i in range(steps):
                a, b = math.exp(h * i / steps), math.exp(h * (i + 1) / steps)
                seen += (b - a) * -math.expm1(-live / (h * math.sqrt(a * b)))
        else:
            seen = rows * -math.expm1(-live / rows)
        seen = min(seen, rows, live)
        if op == "embed":
            return dict(bytes=4.0 * count + e * k * (seen + count), flops=float(count * k))
        table = 2.0 * seen if case["accumulate"] else float(rows)
        return dict(bytes=4.0 * count + e * k * (live + table), flops=float(live * k))
    if op == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        out = M * N * (1 + case["residual"] + case["keep_z"]) + N * case["bias"]
        return dict(bytes=float(e * (M * K + N * K + out)), flops=2.0 * M * N * K)
    if op == "linear_grad":
        M, N, K = case["M"], case["N"], case["K"]
        read = 2 * M * N + M * K + N * K
        return dict(bytes=float(e * (read + M * K + N * K + N)), flops=4.0 * M * N * K)
    n = sum(_sizes(case))
    return dict(bytes=4.0 * e * n, flops=7.0 * n)


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "embed":
        padded = torch.cat([st["table"].double() * case["scale"], torch.zeros(1, case["k"], device="cuda").double()])
        ids = st["ids"].long()
        return padded[torch.where((ids < 0) | (ids >= case["rows"]), case["rows"], ids)]
    if op == "embed_grad":
        ids, order = torch.sort(st["ids"].long(), stable=True)
        first = torch.searchsorted(ids, torch.arange(case["rows"] + 1, device="cuda"))
        total = torch.zeros(case["rows"], case["k"], dtype=torch.float64, device="cuda")
        for a in range(0, case["k"], 64):  # prefix sums, a part of the columns at a time
            run_sum = st["dout"][:, a:a + 64].double()[order].cumsum(0)
            run_sum = torch.cat([torch.zeros_like(run_sum[:1]), run_sum])
            total[:, a:a + 64] = (run_sum[first[1:]] - run_sum[first[:-1]]) * case["scale"]
        return st["table"].double() + total if case["accumulate"] else total
    if op in ("linear", "linear_grad"):
        x, w = st["x"].double(), st["w"].double()
        f = dict(none=lambda z: z, relu=torch.relu, sigmoid=torch.sigmoid, silu=torch.nn.functional.silu,
                 gelu=torch.nn.functional.gelu)[case["act"]]
        if op == "linear":
            z = torch.mm(x, w.t().contiguous())
            z = z + st["bias"].double() if case["bias"] else z
            y = f(z)
            y = y + st["residual"].double() if case["residual"] else y
            return dict(y=y, z=z) if case["keep_z"] else dict(y=y)
        z = st["z"].double().requires_grad_(True)
        dz, = torch.autograd.grad(f(z), z, st["dy"].double())
        return dict(dx=torch.mm(dz, w), dw=torch.mm(dz.t().contiguous(), x), dbias=dz.sum(0))
    g, p = st["flat_g"].double(), st["flat_p"].double()
    norm = torch.linalg.vector_norm(g)
    c = min(1.0, st["max_norm"] / float(norm))
    return dict(p=(1.0 - st["lr"] * st["lam"]) * p - st["lr"] * c * g, norm=norm)
