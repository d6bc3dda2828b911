"""Timed cases of the operators at both ends of a stack of MoE blocks and of the matrices' update: embedding
lookup, softmax cross entropy over a vocabulary, orthogonalised updates.

A case is one pass of one operator: a forward alone, a forward with its gradients (a training
step), or one update of a set of expert matrices. With ``own`` false, ``run`` computes it in
elementary 32-bit torch operations; with ``own`` true it calls the framework's entry points. Model
widths, expert counts and token counts are those of the repository's workloads (``synth``) and the
batches around them; vocabularies are of generic sizes, whole powers of two and odd ones.

``embed``  out[t] = scale * W[id_t] (id < 0: a row of zeros); the step adds dW, the sum of the
           output gradients of each id's tokens, zeros for ids without tokens.
``loss``   z = h W^T, the cross entropy of each token's target and its weighted sum (a target < 0:
           none); the step adds dh and dW. Without weights a token counts 1 / (tokens with a target).
``orth``   the momentum m' = beta m + g, u = g + beta m', and u's matrices orthogonalised by five
           Newton-Schulz products; a matrix whose group has no tokens is left alone.
"""
import math
import random

import numpy as np
import torch

own = False

COEF, STEPS, BETA = (3.4445, -4.7750, 2.0315), 5, 0.95


def _embed(step, dtype, T, d, V, padded, **name):
    return dict(name, kind="embed", step=step, dtype=dtype, T=T, d=d, V=V, padded=padded)


def _loss(step, dtype, T, d, V, masked, weighted, **name):
    return dict(name, kind="loss", step=step, dtype=dtype, T=T, d=d, V=V, masked=masked, weighted=weighted)


def _orth(dtype, G, rows, cols, momentum, skipped, **name):
    return dict(name, kind="orth", dtype=dtype, G=G, rows=rows, cols=cols, momentum=momentum, skipped=skipped)


def listed():
    return [
        # the token of a decode step: launch and latency
        _embed(False, "bf16", 1, 4096, 131072, False, name="embed_fwd_1"),
        # a ragged fp32 batch of padded sequences
        _embed(True, "f32", 2999, 1000, 50021, True, name="embed_step_ragged_f32"),
        # training batches: a small model, the largest one
        _embed(True, "bf16", 4096, 1024, 32768, False, name="embed_step_4096"),
        _embed(True, "bf16", 16384, 4096, 131072, False, name="embed_step_16384"),
        # the loss of a few tokens, as a scorer has it
        _loss(False, "bf16", 7, 2048, 65536, False, False, name="loss_fwd_7"),
        # a ragged fp32 step, and a ragged bf16 one of padded sequences with weights of their own
        _loss(True, "f32", 501, 256, 10007, False, False, name="loss_step_ragged_f32"),
        _loss(True, "bf16", 1003, 1152, 50021, True, True, name="loss_step_ragged_bf16"),
        # training batches: a small model, the largest vocabulary and width
        _loss(True, "bf16", 4096, 1024, 32768, False, False, name="loss_step_4096"),
        _loss(True, "bf16", 8192, 4096, 131072, True, False, name="loss_step_8192"),
        # the gate and up matrices of a small fp32 pool, of a ragged bf16 one with an expert that no token
        # called, of a mid-size pool
        _orth("f32", 8, 1024, 256, True, False, name="orth_tiny_f32"),
        _orth("bf16", 5, 333, 1000, True, True, name="orth_ragged"),
        _orth("bf16", 16, 5632, 1024, True, False, name="orth_16x5632x1024"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """A case of the ranges above: 1 to 65536 tokens (16384 for the loss), widths of 64 to 8192, vocabularies of
    100 to 262144, up to 32 matrices of sides of 16 to 8192."""
    kind = rng.choice(("embed", "loss", "orth"))
    while True:
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if kind == "embed":
            d = 8 * _logint(rng, 8, 1024) if rng.random() < 0.7 else _logint(rng, 64, 8192)
            c = _embed(rng.random() < 0.7, dtype, _logint(rng, 1, 65536), d, _logint(rng, 100, 262144), rng.random() < 0.4)
            if work(c)["bytes"] <= 131072 * 4096 * 2.5:
                return c
        elif kind == "loss":
            d = 128 * _logint(rng, 1, 32) if dtype == "bf16" else 4 * _logint(rng, 16, 512)
            c = _loss(rng.random() < 0.7, dtype, _logint(rng, 1, 16384), d, _logint(rng, 100, 262144), rng.random() < 0.4,
                      rng.random() < 0.4)
            if work(c)["flops"] <= (6.0 * 8192 * 4096 * 131072 if dtype == "bf16" else 2e12):
                return c
        else:
            G = _logint(rng, 1, 32)
            c = _orth(dtype, G, _logint(rng, 16, 8192), _logint(rng, 16, 8192), rng.random() < 0.6, G > 1 and rng.random() < 0.3)
            if work(c)["flops"] <= (3e12 if dtype == "bf16" else 3e11):
                return c


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    f32 = torch.float32

    def normal(*shape, std=1.0, dtype=f32):
        return torch.empty(*shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    def uniform(*shape):
        return torch.empty(*shape, dtype=f32, device="cuda").uniform_(generator=g)

    def tokens(T, V):
        """Ids whose popularity falls as 1 / rank."""
        u = uniform(T).double()
        return (torch.exp(u * math.log(V)) - 1.0).long().clamp_(0, V - 1).to(torch.int32)

    v, dt = {}, _dtype(case)
    if case["kind"] == "embed":
        T, d, V = case["T"], case["d"], case["V"]
        v["ids"] = tokens(T, V)
        if case["padded"]:  # an eighth of the batch behind its sequences' ends
            v["ids"] = torch.where(uniform(T) < 0.125, -1, v["ids"]).to(torch.int32)
        v["w"] = normal(V, d, std=0.02, dtype=dt)
        v["scale"] = math.sqrt(d)
        if case["step"]:
            v["dout"] = normal(T, d, dtype=dt)
    elif case["kind"] == "loss":
        T, d, V = case["T"], case["d"], case["V"]
        v["w"] = normal(V, d, std=0.02, dtype=dt)
        v["target"] = tokens(T, V)
        # half of the tokens lean towards their targets, as those of a model in training do
        lean = torch.where(uniform(T, 1) < 0.5, 8.0 / (0.02 * math.sqrt(d)), 0.0)
        v["h"] = (normal(T, d) + lean * v["w"][v["target"].long()].float()).to(dt)
        if case["masked"]:
            v["target"] = torch.where(uniform(T) < 0.125, -1, v["target"]).to(torch.int32)
        v["weight"] = uniform(T) / T if case["weighted"] else None
    else:
        G, R, C = case["G"], case["rows"], case["cols"]
        # a gradient's few strong directions over a floor of noise
        k = min(16, R, C)
        strong = torch.bmm(normal(G, R, k), normal(G, k, C)) * (3.0 / math.sqrt(k))
        v["g"] = ((normal(G, R, C) + strong) * 1e-3).to(dt)
        v["momentum"] = normal(G, R, C, std=2e-3) if case["momentum"] else None
        v["counts"] = torch.ones(G, dtype=torch.int32, device="cuda") * 17
        if case["skipped"]:
            v["counts"][G // 2] = 0
        v["scale"] = math.sqrt(max(1.0, R / C))
    return v


def prepare(case, seed):
    """The inputs, and the buffers that a program keeps for the results."""
    s = {"case": case, **_inputs(case, seed)}
    dt = _dtype(case)

    def buf(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if case["kind"] == "embed":
        s["out"] = buf(case["T"], case["d"])
        s["dw"] = buf(case["V"], case["d"]) if case["step"] else None
    elif case["kind"] == "loss":
        s["loss"], s["token_loss"] = buf(1, dtype=torch.float32), buf(case["T"], dtype=torch.float32)
        s["dh"] = buf(case["T"], case["d"]) if case["step"] else None
        s["dw"] = buf(case["V"], case["d"]) if case["step"] else None
    else:
        s["out"] = torch.zeros_like(s["g"])
        s["momentum_out"] = torch.zeros_like(s["momentum"]) if case["momentum"] else None
    return s


# --------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2506_02965_gb300 import _lib as L

    c = s["case"]
    dt = L.MOE_BF16 if c["dtype"] == "bf16" else L.MOE_F32

    def room(n):  # kept by the program, as every workspace of the layer is
        if "workspace" not in s:
            s["workspace"] = torch.empty(n(), dtype=torch.uint8, device="cuda")
        return s["workspace"], s["workspace"].numel()

    if c["kind"] == "embed":
        T, d, V = c["T"], c["d"], c["V"]
        L.moe_embed_fwd(T, d, V, dt, s["ids"], s["w"], s["scale"], s["out"])
        if not c["step"]:
            return {"out": s["out"]}
        L.moe_embed_bwd(T, d, V, dt, s["ids"], s["dout"], s["scale"], False, s["dw"], *room(lambda: L.moe_embed_workspace_size(T, d, V)))
        return {"out": s["out"], "dw": s["dw"]}
    if c["kind"] == "loss":
        T, d, V = c["T"], c["d"], c["V"]
        ws = room(lambda: L.moe_vocab_loss_workspace_size(T, d, V, dt, c["step"]))
        L.moe_vocab_loss(T, d, V, dt, s["h"], s["w"], s["target"], s["weight"], s["loss"], s["token_loss"], s["dh"], s["dw"], *ws)
        got = {"loss": s["loss"], "token_loss": s["token_loss"]}
        if c["step"]:
            got.update(dh=s["dh"], dw=s["dw"])
        return got
    G, R, C = c["G"], c["rows"], c["cols"]
    ws = room(lambda: L.moe_orthogonalise_workspace_size(G, R, C, dt))
    L.moe_orthogonalise(G, R, C, dt, s["g"], s["momentum"], BETA, True, s["counts"], STEPS, s["scale"], s["momentum_out"], s["out"], *ws)
    got = {"out": s["out"]}
    if c["momentum"]:
        got["momentum"] = s["momentum_out"]
    return got


# --------------------------------------------------------------------------- plain forms, 32 bits
def _plain_embed(s):
    c, dt = s["case"], _dtype(s["case"])
    ids = s["ids"].long()
    there = ids >= 0
    rows = s["w"][ids.clamp(min=0)].float() * s["scale"]
    got = {"out": torch.where(there[:, None], rows, 0.0).to(dt)}
    if c["step"]:
        # sums of equal ids' rows, in order of the tokens: one more row collects the padding
        order = torch.sort(torch.where(there, ids, c["V"]), stable=True)
        dw = torch.zeros(c["V"] + 1, c["d"], device="cuda")
        dw.index_add_(0, order.values, s["dout"].float()[order.indices])
        got["dw"] = (dw[:-1] * s["scale"]).to(dt)
    return got


def _plain_loss(s):
    c, dt = s["case"], _dtype(s["case"])
    y = s["target"].long()
    there, at = y >= 0, y.clamp(min=0)[:, None]
    h, w = s["h"].float(), s["w"].float()
    z = h @ w.T
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    token = torch.where(there, (torch.log(total) + top - z.gather(1, at))[:, 0], 0.0)
    u = s["weight"] if s["weight"] is not None else torch.ones_like(token) / there.sum().clamp(min=1)
    u = torch.where(there, u, 0.0)
    got = {"loss": (u.double() * token).sum().float().view(1), "token_loss": token}
    if c["step"]:
        dz = e * (u[:, None] / total)
        dz.scatter_add_(1, at, -u[:, None])
        got.update(dh=(dz @ w).to(dt), dw=(dz.T @ h).to(dt))
    return got


def _plain_orth(s):
    c, dt = s["case"], _dtype(s["case"])
    a, b, k = COEF
    called = (s["counts"] > 0)[:, None, None]
    g, got = s["g"].float(), {}
    if c["momentum"]:
        m = BETA * s["momentum"] + g
        g = g + BETA * m
        got["momentum"] = torch.where(called, m, 0.0)
    x = g if c["rows"] <= c["cols"] else g.transpose(1, 2)
    norm = torch.sqrt(x.double().square().sum((1, 2), keepdim=True)).float()
    x = x / torch.where(norm > 0, norm, 1.0)
    for _ in range(STEPS):
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + k * (A @ A)) @ x
    x = x if c["rows"] <= c["cols"] else x.transpose(1, 2)
    return {"out": torch.where(called, s["scale"] * x, 0.0).to(dt).contiguous(), **got}


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "loss": _plain_loss, "orth": _plain_orth}[state["case"]["kind"]](state)


def _distinct(T, V):
    """The ids that T tokens are expected to touch."""
    p = np.diff(np.log(np.arange(1, V + 2, dtype=np.float64))) / math.log(V + 1)
    return float((1.0 - np.exp(T * np.log1p(-np.minimum(p, 1 - 1e-12)))).sum())


def work(case):
    """Every input read once and every result written once; of a symmetric product half."""
    c = case
    b = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "embed":
        T, d, V = c["T"], c["d"], c["V"]
        rows = min(T, V, _distinct(T, V))
        by = 4 * T + rows * d * b + T * d * b
        return {"bytes": by + (4 * T + T * d * b + V * d * b if c["step"] else 0), "flops": 2.0 * T * d}
    if c["kind"] == "loss":
        T, d, V = c["T"], c["d"], c["V"]
        by = (T * d + V * d) * b + 8 * T
        return {"bytes": by * (2 if c["step"] else 1), "flops": (6.0 if c["step"] else 2.0) * T * d * V}
    n, m = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    G = c["G"] - (1 if c["skipped"] else 0)
    each = STEPS * (n * n * m + n * n * n + 2.0 * n * n * m)
    return {"bytes": max(1, G) * n * m * (2 * b + (8 if c["momentum"] else 0)), "flops": max(1, G) * each}


# --------------------------------------------------------------------------- the definitions, 64 bits
def exact(case, seed):
    if work(case)["flops"] > 8e12:  # over half a minute in 64 bits
        return None
    return {"embed": _exact_embed, "loss": _exact_loss, "orth": _exact_orth}[case["kind"]](case, _inputs(case, seed))


def _exact_embed(c, v):
    ids, f64 = v["ids"].long(), torch.float64
    live = torch.nonzero(ids >= 0)[:, 0]
    out = torch.zeros(c["T"], c["d"], dtype=f64, device="cuda")
    out[live] = v["w"].index_select(0, ids[live]).to(f64) * v["scale"]
    if not c["step"]:
        return {"out": out}
    dw = torch.zeros(c["V"], c["d"], dtype=f64, device="cuda")
    if live.numel():  # the rows of each id as differences of a running sum over the sorted tokens, columns at a time
        key, order = torch.sort(ids[live])
        used, n = torch.unique_consecutive(key, return_counts=True)
        ends = torch.cumsum(n, 0)
        for c0 in range(0, c["d"], 512):
            part = torch.cumsum(v["dout"][live[order], c0:c0 + 512].to(f64), 0)[ends - 1]
            part[1:] -= part[:-1].clone()
            dw[used, c0:c0 + 512] = part * v["scale"]
    return {"out": out, "dw": dw}


def _exact_loss(c, v):
    f64, T, V = torch.float64, c["T"], c["V"]
    y, w = v["target"].long(), v["w"].to(f64)
    n = int((y >= 0).sum())
    u = v["weight"].to(f64) if c["weighted"] else torch.full((T,), 1.0 / max(n, 1), dtype=f64, device="cuda")
    token = torch.zeros(T, dtype=f64, device="cuda")
    dh, dw = torch.zeros(T, c["d"], dtype=f64, device="cuda"), torch.zeros_like(w)
    for t0 in range(0, T, 1024):  # tokens at a time, those without a target left out
        rows = t0 + torch.nonzero(y[t0:t0 + 1024] >= 0)[:, 0]
        h = v["h"][rows].to(f64)
        logp = torch.log_softmax(torch.mm(h, w.t()), 1)
        r = torch.arange(rows.numel(), device="cuda")
        token[rows] = -logp[r, y[rows]]
        if c["step"]:
            d = torch.exp(logp)
            d[r, y[rows]] -= 1.0
            d *= u[rows, None]
            dh[rows] = torch.mm(d, w)
            dw.addmm_(d.t(), h)
    got = {"loss": torch.dot(u, token).view(1), "token_loss": token}
    if c["step"]:
        got.update(dh=dh, dw=dw)
    return got


def _exact_orth(c, v):
    a, b, k = COEF
    f64 = torch.float64
    out, mom = torch.zeros(v["g"].shape, dtype=f64, device="cuda"), torch.zeros(v["g"].shape, dtype=f64, device="cuda")
    for i in range(c["G"]):  # each matrix as a tall one, its small square to the right
        if int(v["counts"][i]) <= 0:
            continue
        x = v["g"][i].to(f64)
        if c["momentum"]:
            mom[i] = torch.add(x, v["momentum"][i].to(f64), alpha=BETA)
            x = torch.add(x, mom[i], alpha=BETA)
        x = x if c["rows"] >= c["cols"] else x.t()
        x = x / torch.linalg.matrix_norm(x)
        eye = torch.eye(x.shape[1], dtype=f64, device="cuda")
        for _ in range(STEPS):
            q = torch.mm(x.t(), x)
            x = torch.mm(x, torch.addmm(a * eye, q, torch.add(b * eye, q, alpha=k)))
        out[i] = v["scale"] * (x if c["rows"] >= c["cols"] else x.t())
    return {"out": out, "momentum": mom} if c["momentum"] else {"out": out}
