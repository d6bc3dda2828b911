"""Timed cases of the operators around the MoE expert layer: layer norm, gating rules, 8-bit
activation checkpoints.

A case is one pass of one operator: a forward alone (inference), a forward with its backward
(a training step), or a checkpoint with what the backward makes of it. With ``own`` false,
``run`` computes it in elementary 32-bit torch operations; with ``own`` true it calls the
framework's entry points. Sizes are those of the repository's workloads (``synth``) and the
batches around them: one token, a decode batch, ragged prompts, training batches of both
storage types.

``norm``  h = x + residual, y = LN(h) gamma + beta; the step adds dx, dgamma, dbeta, read from
          the stored h or from its 8-bit checkpoint.
``gate``  scores of the router logits (softmax or sigmoid), picks by score and balance bias
          among the kept expert groups, gate weights, counts; the step adds the logits'
          gradient and the balance bias after its update.
``ckpt``  8-bit blocks of 128 columns with one scale each: the values they stand for
          ("values"), or the SwiGLU activations and gradients made from them ("swiglu").
"""
import math
import random

import torch

own = False

BLOCK, EPS, RATE, AUX = 128, 1e-5, 1e-3, 0.01
TINY = 2.0 ** -100  # a block whose largest magnitude is below this is held as zeros


def _norm(step, dtype, T, d, residual, ckpt, **name):
    return dict(name, kind="norm", step=step, dtype=dtype, T=T, d=d, residual=residual, ckpt=ckpt)


def _gate(step, T, E, k, P=1, score="softmax", groups=1, kept=1, best=1, normalize=False, scale=1.0, bias=False, masked=False, **name):
    return dict(name, kind="gate", step=step, T=T, E=E, k=k, P=P, score=score, groups=groups, kept=kept, best=best,
                normalize=normalize, scale=scale, bias=bias, masked=masked)


def _ckpt(use, dtype, R, C, **name):
    return dict(name, kind="ckpt", use=use, dtype=dtype, R=R, C=C)


def listed():
    wide = dict(score="sigmoid", groups=8, kept=4, best=2, normalize=True, scale=2.5, bias=True)
    return [
        # a decode step of a few users: launch and latency
        _norm(False, "bf16", 4, 4096, True, False, name="norm_fwd_4"),
        # a ragged prompt, whose hidden states are kept in 8 bits
        _norm(False, "bf16", 2999, 2048, True, True, name="norm_fwd_2999"),
        # an fp32 training step with a ragged width, and the largest bf16 one, its backward from 8 bits
        _norm(True, "f32", 1501, 1000, False, False, name="norm_step_ragged_f32"),
        _norm(True, "bf16", 16384, 4096, True, True, name="norm_step_16384"),
        # one token through a fine-grained pool
        _gate(False, 1, 64, 6, name="gate_fwd_1"),
        # a ragged prompt through a wide pool in groups, some experts out of reach of some tokens
        _gate(False, 2999, 256, 8, masked=True, name="gate_fwd_2999", **wide),
        # training steps: a small pool, and a wide one of four parties with a balance bias
        _gate(True, 4096, 16, 2, name="gate_step_4096"),
        _gate(True, 65536, 256, 8, P=4, name="gate_step_65536", **wide),
        # the hidden states of a small batch
        _ckpt("values", "bf16", 33, 4096, name="ckpt_values_33"),
        # expert activations of training steps: ragged fp32, a fine-grained pool, the largest layer
        _ckpt("swiglu", "f32", 4503, 1366, name="ckpt_swiglu_ragged_f32"),
        _ckpt("swiglu", "bf16", 17994, 1408, name="ckpt_swiglu_17994"),
        _ckpt("swiglu", "bf16", 32768, 14336, name="ckpt_swiglu_32768"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """A case of the ranges above: 1 to 65536 tokens, widths of 64 to 8192, pools of 4 to 256
    experts, up to 98304 expert rows of widths up to 14336."""
    kind = rng.choice(("norm", "gate", "ckpt"))
    while True:
        if kind == "norm":
            d = 8 * _logint(rng, 8, 1024) if rng.random() < 0.7 else _logint(rng, 64, 8192)
            c = _norm(rng.random() < 0.6, rng.choice(("bf16", "bf16", "f32")), _logint(rng, 1, 65536), d,
                      rng.random() < 0.5, rng.random() < 0.4)
            most = 16384 * 4096 * 18
        elif kind == "gate":
            groups = rng.choice((1, 1, 2, 4, 8))
            E = groups * _logint(rng, 4, 256 // groups)
            kept = rng.randint(1, groups)
            k = rng.randint(1, min(8, kept * (E // groups)))
            c = _gate(rng.random() < 0.6, _logint(rng, 1, 65536), E, k, P=rng.choice((1, 1, 2, 3, 5)),
                      score=rng.choice(("softmax", "sigmoid")), groups=groups, kept=kept, best=rng.choice((1, 2)),
                      normalize=rng.random() < 0.5, scale=rng.choice((1.0, 2.5)), bias=rng.random() < 0.5,
                      masked=rng.random() < 0.3)
            most = 65536 * 256 * 13
        else:
            C = 8 * _logint(rng, 8, 1792) if rng.random() < 0.7 else _logint(rng, 64, 14336)
            c = _ckpt(rng.choice(("values", "swiglu", "swiglu")), rng.choice(("bf16", "bf16", "f32")),
                      _logint(rng, 1, 98304), C)
            most = 32768 * 14336 * 16
        if work(c)["bytes"] <= most:
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

    v = {}
    if case["kind"] == "norm":
        T, d, dt = case["T"], case["d"], _dtype(case)
        # hidden states with an offset and a few loud channels, as residual streams have them
        loud = torch.where(uniform(d) < 0.01, 20.0, 1.0)
        v["x"] = (normal(T, d) * loud + 0.3).to(dt)
        v["residual"] = normal(T, d, dtype=dt) if case["residual"] else None
        v["gamma"], v["beta"] = 1.0 + normal(d, std=0.1), normal(d, std=0.1)
        if case["step"]:
            v["dy"] = normal(T, d, dtype=dt)
            v["dh"] = normal(T, d, dtype=dt) if case["residual"] else None
    elif case["kind"] == "gate":
        T, E, k, P = (case[n] for n in ("T", "E", "k", "P"))
        v["logits"] = normal(T, E, std=0.9)
        if case["masked"]:  # one expert in four out of a token's reach; now and then all of them
            out = (uniform(T, E) < 0.25) | (uniform(T, 1) < 0.002)
            v["logits"].masked_fill_(out, -math.inf)
        v["bias"] = normal(P, E, std=0.02) if case["bias"] else None
        # parties of unequal size, equal ones where they divide the batch
        cut = [0] + sorted(min(T, T * p // P + ((7 * p) % 11 if T % P else 0)) for p in range(1, P)) + [T]
        v["party_offsets"] = torch.tensor(cut, dtype=torch.int32, device="cuda")
        if case["step"]:
            v["dweights"] = normal(T, k)
            v["aux_coef"] = uniform(P, E) * (AUX * E / max(T, 1))
    else:
        R, C, dt = case["R"], case["C"], _dtype(case)
        v["x"] = normal(R, 2 * C if case["use"] == "swiglu" else C, std=1.3, dtype=dt)
        if case["use"] == "swiglu":
            v["dact"] = normal(R, C, dtype=dt)
    return v


def prepare(case, seed):
    """The inputs, and the buffers that a program keeps for the results."""
    s = {"case": case, **_inputs(case, seed)}
    f32, i32 = torch.float32, torch.int32

    def buf(*shape, dtype=f32):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    if case["kind"] == "norm":
        T, d, dt = case["T"], case["d"], _dtype(case)
        s["y"] = buf(T, d, dtype=dt)
        s["h"] = buf(T, d, dtype=dt) if case["residual"] else None
        s["mean"], s["rstd"] = (buf(T), buf(T)) if case["step"] else (None, None)
        if case["ckpt"]:
            s["q"], s["h_scale"] = buf(T, d, dtype=torch.int8), buf(T, -(-d // BLOCK))
            s["h_held"] = None if case["step"] else buf(T, d, dtype=dt)
        if case["step"]:
            s["dx"], s["dgamma"], s["dbeta"] = buf(T, d, dtype=dt), buf(d), buf(d)
    elif case["kind"] == "gate":
        T, E, k, P = (case[n] for n in ("T", "E", "k", "P"))
        s["topk_idx"], s["topk_w"], s["counts"] = buf(T, k, dtype=i32), buf(T, k), buf(P, E, dtype=i32)
        if case["step"]:
            s["dlogits"], s["bias_next"] = buf(T, E), buf(P, E)
            s["bias"] = torch.zeros(P, E, device="cuda") if s["bias"] is None else s["bias"]
    else:
        R, C, dt = case["R"], case["C"], _dtype(case)
        W = s["x"].shape[1]
        s["q"], s["scale"] = buf(R, W, dtype=torch.int8), buf(R, -(-W // BLOCK))
        if case["use"] == "values":
            s["held"] = buf(R, C, dtype=dt)
        else:
            s["act"], s["dh"] = buf(R, C, dtype=dt), buf(R, 2 * C, dtype=dt)
    return s


# --------------------------------------------------------------------------- the framework's calls
def _own(s):
    from paper_2506_02965_gb300 import _lib as L

    c = s["case"]
    if c["kind"] == "norm":
        T, d = c["T"], c["d"]
        dt = L.MOE_BF16 if c["dtype"] == "bf16" else L.MOE_F32
        q, scale = s.get("q"), s.get("h_scale")
        L.moe_layer_norm_fwd(T, d, dt, s["x"], s["residual"], s["gamma"], s["beta"], EPS, s["h"], s["y"], s["mean"], s["rstd"],
                             q, scale)
        got = {"y": s["y"]}
        if c["residual"]:
            got["h"] = s["h"]
        if c["ckpt"]:
            got["h_scale"] = scale
        if not c["step"]:
            if c["ckpt"]:
                L.moe_ckpt_unpack(T, d, dt, q, scale, s["h_held"])
                got["h_held"] = s["h_held"]
            return got
        if "workspace" not in s:  # kept by the program, as every workspace of the layer is
            s["workspace"] = torch.empty(L.moe_layer_norm_workspace_size(T, d), dtype=torch.uint8, device="cuda")
        h = None if c["ckpt"] else s["h"] if c["residual"] else s["x"]
        L.moe_layer_norm_bwd(T, d, dt, s["dy"], h, q, scale, s["mean"], s["rstd"], s["gamma"], s["dh"], s["dx"], s["dgamma"],
                             s["dbeta"], s["workspace"], s["workspace"].numel())
        got.update(mean=s["mean"], rstd=s["rstd"], dx=s["dx"], dgamma=s["dgamma"], dbeta=s["dbeta"])
        return got
    if c["kind"] == "gate":
        if "cfg" not in s:
            s["cfg"] = L.make_config(c["T"], 128, c["E"], 128, c["k"], c["P"], normalize_topk=c["normalize"])
            score = L.MOE_SCORE_SIGMOID if c["score"] == "sigmoid" else L.MOE_SCORE_SOFTMAX
            s["rule"] = L.make_gate_rule(score, c["groups"], c["kept"], c["best"], c["scale"])
        cfg, rule = s["cfg"], s["rule"]
        po = s["party_offsets"] if c["P"] > 1 else None
        L.moe_gate(cfg, rule, s["logits"], s["bias"], po, None, s["topk_idx"], s["topk_w"], s["counts"])
        got = {"topk_idx": s["topk_idx"], "topk_w": s["topk_w"], "counts": s["counts"]}
        if c["step"]:
            L.moe_gate_bwd(cfg, rule, s["logits"], s["topk_idx"], s["dweights"], s["aux_coef"], po, s["dlogits"])
            L.moe_gate_balance(cfg, s["counts"], RATE, s["bias"], s["bias_next"])
            got.update(dlogits=s["dlogits"], bias=s["bias_next"])
        return got
    dt = L.MOE_BF16 if c["dtype"] == "bf16" else L.MOE_F32
    R, C = c["R"], c["C"]
    L.moe_ckpt_pack(R, s["x"].shape[1], dt, s["x"], s["q"], s["scale"])
    if c["use"] == "values":
        L.moe_ckpt_unpack(R, C, dt, s["q"], s["scale"], s["held"])
        return {"held": s["held"], "scale": s["scale"]}
    L.moe_ckpt_swiglu_bwd(R, C, dt, s["q"], s["scale"], s["dact"], s["act"], s["dh"])
    return {"act": s["act"], "dh": s["dh"], "scale": s["scale"]}


# --------------------------------------------------------------------------- plain forms, 32 bits
def _blocks(x):
    """[R, C] -> [R, blocks, 128], zeros past C."""
    R, C = x.shape
    n = -(-C // BLOCK)
    if n * BLOCK != C:
        x = torch.cat([x, x.new_zeros(R, n * BLOCK - C)], 1)
    return x.view(R, n, BLOCK)


def _held(x):
    """What 8 bits hold of x (32-bit values): the values, and the blocks' scales."""
    b = _blocks(x)
    most = b.abs().amax(2)
    small, top = most < TINY, most.new_full((), 127.0)  # a tensor: each quotient is rounded once
    scale = torch.where(small, 0.0, most / top)
    q = torch.round(b * torch.where(small, 0.0, top / most)[..., None])
    return (q * scale[..., None]).view(x.shape[0], -1)[:, :x.shape[1]], scale


def _plain_norm(s):
    c, dt = s["case"], _dtype(s["case"])
    h = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    stored = h.to(dt)
    mean = h.mean(1)
    rstd = 1.0 / torch.sqrt((h - mean[:, None]).square().mean(1) + EPS)
    y = (h - mean[:, None]) * rstd[:, None] * s["gamma"] + s["beta"]
    got = {"y": y.to(dt)}
    if c["residual"]:
        got["h"] = stored
    kept = stored.float()
    if c["ckpt"]:
        kept, got["h_scale"] = _held(kept)
        if not c["step"]:
            got["h_held"] = kept.to(dt)
    if c["step"]:
        dy = s["dy"].float()
        xh = (kept - mean[:, None]) * rstd[:, None]
        g = dy * s["gamma"]
        dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        got.update(mean=mean, rstd=rstd, dx=dx.to(dt), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
    return got


def _party(s):
    """The party of every token."""
    t = torch.arange(s["case"]["T"], device="cuda", dtype=torch.int32)
    return (t[:, None] >= s["party_offsets"][None, 1:-1]).sum(1)


def _plain_gate(s):
    c = s["case"]
    T, E, k, P, G = c["T"], c["E"], c["k"], c["P"], c["groups"]
    party = _party(s)
    z = torch.where(torch.isnan(s["logits"]), -math.inf, s["logits"])
    if c["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-z))
        key = score
    else:
        top = z.amax(1, keepdim=True)
        score = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
        total = score.sum(1, keepdim=True)
        score = torch.where(total > 0, score / total, 0.0)
        key = z
    if s["bias"] is not None:
        key = key + s["bias"][party]
    key = torch.where(z == -math.inf, -math.inf, key)
    best = torch.sort(key.view(T, G, E // G), dim=2, descending=True, stable=True).values[..., :c["best"]].sum(2)
    order = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["kept"]]
    kept = torch.zeros(T, G, dtype=torch.int32, device="cuda").scatter_(1, order, 1).repeat_interleave(E // G, 1)
    # by key, those of dropped groups after all others, equal ones by expert
    idx = torch.sort(key, dim=1, descending=True, stable=True).indices
    last = torch.sort(kept.gather(1, idx), dim=1, descending=True, stable=True).indices
    idx = idx.gather(1, last)[:, :k]
    pick = score.gather(1, idx)
    total = pick.sum(1, keepdim=True) if c["normalize"] else torch.ones(T, 1, device="cuda")
    w = torch.where(total > 0, c["scale"] * pick / total, 0.0)
    counts = torch.zeros(P * E, dtype=torch.int32, device="cuda")
    counts.index_add_(0, (party[:, None] * E + idx).view(-1), torch.ones(T * k, dtype=torch.int32, device="cuda"))
    got = {"topk_idx": idx.int(), "topk_w": w, "counts": counts.view(P, E)}
    if c["step"]:
        g = s["dweights"]
        if c["normalize"]:
            ds = torch.where(total > 0, (c["scale"] * g - (g * w).sum(1, keepdim=True)) / total, 0.0)
        else:
            ds = c["scale"] * g
        ds = s["aux_coef"][party].scatter_add(1, idx, ds)
        if c["score"] == "sigmoid":
            u = torch.exp(-z.abs())
            got["dlogits"] = torch.where(torch.isinf(z), 0.0, ds * u / ((1.0 + u) * (1.0 + u)))
        else:
            got["dlogits"] = score * (ds - (ds * score).sum(1, keepdim=True))
        n = got["counts"].long()
        got["bias"] = s["bias"] + RATE * torch.sign(n.sum(1, keepdim=True) - E * n).float()
    return got


def _plain_ckpt(s):
    c, dt = s["case"], _dtype(s["case"])
    held, scale = _held(s["x"].float())
    if c["use"] == "values":
        return {"held": held.to(dt), "scale": scale}
    G, U = held[:, :c["C"]], held[:, c["C"]:]
    dact = s["dact"].float()
    sig = 1.0 / (1.0 + torch.exp(-G))
    dh = torch.cat([dact * U * sig * (1.0 + G * (1.0 - sig)), dact * G * sig], 1)
    return {"act": (G * sig * U).to(dt), "dh": dh.to(dt), "scale": scale}


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "gate": _plain_gate, "ckpt": _plain_ckpt}[state["case"]["kind"]](state)


def work(case):
    """Every input read once and every result written once; a backward of its own call reads
    what the forward left for it, and a checkpoint is written and read."""
    c = case
    if c["kind"] == "norm":
        n, b = c["T"] * c["d"], 2 if c["dtype"] == "bf16" else 4
        r, q = int(c["residual"]), 1.0 + 4.0 / BLOCK
        by = n * b * (2 + 2 * r) + (n * q if c["ckpt"] else 0) + 8 * c["d"]
        if c["step"]:  # dy, dh and the stored states read, dx and the weights' gradients written
            return {"bytes": by + n * b * (2 + r) + n * (q if c["ckpt"] else b) + 16 * c["T"] + 12 * c["d"], "flops": 20.0 * n}
        if c["ckpt"]:
            by += n * (q + b)
        return {"bytes": by, "flops": 8.0 * n}
    if c["kind"] == "gate":
        n, m = c["T"] * c["E"], c["T"] * c["k"]
        if c["step"]:
            return {"bytes": 12 * n + 16 * m + 20 * c["P"] * c["E"], "flops": 16.0 * n}
        return {"bytes": 4 * n + 8 * m + 4 * c["P"] * c["E"], "flops": 8.0 * n}
    n, b, q = c["R"] * c["C"], 2 if c["dtype"] == "bf16" else 4, 1.0 + 4.0 / BLOCK
    if c["use"] == "values":
        return {"bytes": n * (2 * b + 2 * q), "flops": 4.0 * n}
    return {"bytes": n * (2 * b + 4 * q + 4 * b), "flops": 30.0 * n}


# --------------------------------------------------------------------------- the definitions, 64 bits
def exact(case, seed):
    return {"norm": _exact_norm, "gate": _exact_gate, "ckpt": _exact_ckpt}[case["kind"]](case, _inputs(case, seed))


def _exact_held(x):
    """x in 64 bits -> what the 8-bit blocks hold, block by block of columns."""
    out, scales = torch.empty_like(x), []
    for c0 in range(0, x.shape[1], BLOCK):
        b = x[:, c0:c0 + BLOCK]
        most = b.abs().max(1, keepdim=True).values
        step = torch.where(most < TINY, torch.zeros_like(most), most / 127)
        out[:, c0:c0 + BLOCK] = torch.round(b / torch.where(step > 0, step, torch.ones_like(step))) * step
        scales.append(step)
    return out, torch.cat(scales, 1)


def _exact_norm(c, v):
    f64, dt = torch.float64, _dtype(c)
    h = v["x"].to(f64)
    if c["residual"]:
        h = h + v["residual"].to(f64)
    var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
    rstd = torch.rsqrt(var + EPS)
    got = {"y": torch.addcmul(v["beta"].to(f64), (h - mean) * rstd, v["gamma"].to(f64))}
    if c["residual"]:
        got["h"] = h
    kept = h.to(dt).to(f64)
    if c["ckpt"]:
        kept, got["h_scale"] = _exact_held(kept)
        if not c["step"]:
            got["h_held"] = kept
    if not c["step"]:
        return got
    # dx = (I - 1 1'/d - xh xh'/d) (dy gamma) rstd, with xh of the kept states
    dy, d = v["dy"].to(f64), c["d"]
    xh = (kept - mean) * rstd
    g = dy * v["gamma"].to(f64)
    dx = (g - g.sum(1, keepdim=True) / d - xh * torch.einsum("td,td->t", g, xh)[:, None] / d) * rstd
    if c["residual"]:
        dx = dx + v["dh"].to(f64)
    got.update(mean=mean[:, 0], rstd=rstd[:, 0], dx=dx, dgamma=torch.einsum("td,td->d", dy, xh), dbeta=dy.sum(0))
    return got


def _exact_gate(c, v):
    """Weights and gradients in 64 bits for the picks, which are decided on the 32-bit keys."""
    T, E, k, f64 = c["T"], c["E"], c["k"], torch.float64
    idx = _plain_gate({"case": dict(c, step=False), **v})["topk_idx"].long()
    z = v["logits"].to(f64)
    gone = torch.isneginf(z)
    if c["score"] == "sigmoid":
        p = torch.sigmoid(z)
    else:
        p = torch.nan_to_num(torch.softmax(z, 1))
    pick = p.gather(1, idx)
    total = pick.sum(1, keepdim=True) if c["normalize"] else torch.ones_like(pick[:, :1])
    w = torch.nan_to_num(c["scale"] * pick / total)
    got = {"topk_idx": None, "topk_w": w, "counts": None}
    if not c["step"]:
        return got
    cut = v["party_offsets"].long()
    rows = torch.repeat_interleave(torch.arange(c["P"], device="cuda"), cut[1:] - cut[:-1])
    dp = v["aux_coef"].to(f64)[rows]
    g = v["dweights"].to(f64)
    if c["normalize"]:  # d(w_i)/d(p_j) = (scale [i = j] - w_i) / sum
        through = torch.nan_to_num((c["scale"] * g - (w * g).sum(1, keepdim=True)) / total, posinf=0.0, neginf=0.0)
    else:
        through = c["scale"] * g
    dp = dp.scatter_add(1, idx, through)
    if c["score"] == "sigmoid":
        dz = dp * p * torch.sigmoid(-z)
    else:
        dz = p * dp - p * (p * dp).sum(1, keepdim=True)
    got.update(dlogits=dz.masked_fill(gone, 0.0), bias=None)
    return got


def _exact_ckpt(c, v):
    x, C = v["x"], c["C"]
    act, dh, scales, held = [], [], [], []
    for r in range(0, c["R"], 4096):  # rows at a time: the largest case's 64-bit temporaries
        h, scale = _exact_held(x[r:r + 4096].double())
        scales.append(scale)
        if c["use"] == "values":
            held.append(h)
            continue
        g, u = h[:, :C], h[:, C:]
        da, sig = v["dact"][r:r + 4096].double(), torch.sigmoid(g)
        act.append(g * sig * u)
        dh.append(torch.cat([da * u * (sig + g * sig * torch.sigmoid(-g)), da * g * sig], 1))
    if c["use"] == "values":
        return {"held": torch.cat(held), "scale": torch.cat(scales)}
    return {"act": torch.cat(act), "dh": torch.cat(dh), "scale": torch.cat(scales)}
