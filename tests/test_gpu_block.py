"""A stack of pre-norm MoE blocks trained from 8-bit checkpoints (block.PreNormMoE) against a plain
64-bit implementation that holds the same activations in 8 bits, and moe_expert_ffn_bwd_ckpt
against moe_expert_ffn_bwd.

Bounds. fp32: both sides quantise the same values but for a few that lie within fp32 rounding of a step's
middle (a share of about 1e-4 after several matrix products); one such value moves by a step, 1/127 of its
block's largest, so that a gradient's norm is off by at most about 1e-4 of itself per checkpoint: 2e-3.
bf16: the operands of every product are rounded to 2^-8 relative, independently; a gradient passes
about ten such products per block: 5e-2 of its norm over two blocks (checked by norms, not by element)."""
import pytest
import torch

from synth import moe_inputs as mi
from tests.gpu_util import need_gpu, status

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def L():
    return need_gpu()


def held(x, dt):
    """What a checkpoint of x (rounded to dt) holds, unrounded."""
    x = x.to(dt).double()
    R, C = x.shape
    n = -(-C // 128)
    b = torch.nn.functional.pad(x, (0, n * 128 - C)).view(R, n, 128)
    a = b.abs().amax(2, keepdim=True)
    step = torch.where(a > 0, a / 127, torch.ones_like(a))
    return (torch.round(b / step) * step).view(R, -1)[:, :C]


def build(shape, n, rule, seed):
    from paper_2506_02965_gb300.block import PreNormMoE
    g = torch.Generator(device="cuda").manual_seed(seed)
    net = PreNormMoE(shape, n, rule)
    for b in net.blocks:
        b.gamma.normal_(1.0, 0.1, generator=g)
        b.beta.normal_(0.0, 0.1, generator=g)
        b.w_router.normal_(0.0, 0.1, generator=g)
        b.w1.normal_(0.0, 0.1, generator=g)
        b.w2.normal_(0.0, 0.1, generator=g)
        b.balance_bias.normal_(0.0, 0.05, generator=g)
    net.gamma.normal_(1.0, 0.1, generator=g)
    net.beta.normal_(0.0, 0.1, generator=g)
    x = torch.empty(shape.T, shape.d_model, device="cuda").normal_(generator=g).to(net.out.dtype)
    dout = torch.empty(shape.T, shape.d_model, device="cuda").normal_(generator=g).to(net.out.dtype)
    return net, x, dout


def norm(h, gamma, beta):
    v, m = torch.var_mean(h, dim=1, correction=0, keepdim=True)
    return (h - m) / torch.sqrt(v + EPS) * gamma.double() + beta.double(), m, 1 / torch.sqrt(v + EPS)


def norm_bwd(dy, kept, m, rs, gamma):
    xh = (kept - m) * rs
    g = dy * gamma.double()
    return rs * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)), (dy * xh).sum(0), dy.sum(0)


def plain(net, sh, picks, x, dout, scale, dt, cut):
    """Output and gradients in 64 bits with the network's picks, from the checkpoints' values."""
    E, k, F = sh.n_experts, sh.top_k, sh.d_ff
    saved, h, m = [], x.double(), None
    for b, idx in zip(net.blocks, picks):
        h = h if m is None else (h + m)
        y, mean, rs = norm(h, b.gamma, b.beta)
        hk = held(h, dt)
        z = torch.cat([y[cut[p]:cut[p + 1]] @ b.w_router[p].double().T for p in range(sh.n_parties)])
        s = torch.sigmoid(z)
        pick = s.gather(1, idx)
        w = scale * pick / pick.sum(1, keepdim=True)
        out = torch.zeros_like(h)
        per = []
        for e in range(E):
            t, j = (idx == e).nonzero(as_tuple=True)
            gu = y[t] @ b.w1[e].double().T
            G, U = gu.chunk(2, 1)
            ye = (G * torch.sigmoid(G) * U) @ b.w2[e].double().T
            out.index_add_(0, t, w[t, j, None] * ye)
            per.append((t, j, held(gu, dt) if len(t) else gu, held(ye, dt) if len(t) else ye))
        saved.append((hk, mean, rs, z, s, w, per))
        m = out
    h = h + m
    final, mean, rs = norm(h, net.gamma, net.beta)
    dh, dg, db = norm_bwd(dout.double(), held(h, dt), mean, rs, net.gamma)
    got = {"out": final, "gamma": dg, "beta": db}
    for i in reversed(range(len(net.blocks))):
        b, idx = net.blocks[i], picks[i]
        hk, mean, rs, z, s, w, per = saved[i]
        y = norm(hk, b.gamma, b.beta)[0]
        dy, dw = torch.zeros_like(hk), torch.zeros_like(w)
        dw1, dw2 = torch.zeros(E, 2 * F, sh.d_model, dtype=torch.float64, device="cuda"), torch.zeros(E, sh.d_model, F, dtype=torch.float64, device="cuda")
        for e in range(E):
            t, j, gu, ye = per[e]
            if not len(t):
                continue
            G, U = gu.chunk(2, 1)
            sg = torch.sigmoid(G)
            dw[t, j] = (dh[t] * ye).sum(1)
            de = w[t, j, None] * dh[t]
            dA = de @ b.w2[e].double()
            dgu = torch.cat([dA * U * sg * (1 + G * (1 - sg)), dA * G * sg], 1)
            dw2[e], dw1[e] = de.T @ (G * sg * U), dgu.T @ y[t]
            dy.index_add_(0, t, dgu @ b.w1[e].double())
        S = s.gather(1, idx).sum(1, keepdim=True)
        ds = torch.zeros_like(s).scatter_(1, idx, (scale * dw - (dw * w).sum(1, keepdim=True)) / S)
        dz = ds * s * (1 - s)
        dwr = torch.stack([dz[cut[p]:cut[p + 1]].T @ y[cut[p]:cut[p + 1]] for p in range(sh.n_parties)])
        dy += torch.cat([dz[cut[p]:cut[p + 1]] @ b.w_router[p].double() for p in range(sh.n_parties)])
        dx, dg, db = norm_bwd(dy, hk, mean, rs, b.gamma)
        dh = dh + dx
        got[i] = {"gamma": dg, "beta": db, "w_router": dwr, "w1": dw1, "w2": dw2}
    got["dx"] = dh
    return got


def near(name, got, ref, tol):
    off = float((got.double() - ref).norm() / ref.norm().clamp_min(1e-30))
    assert off <= tol, (name, off)


@pytest.mark.parametrize("dtype,T,d,E,F,k,P,n,tol", [
    ("f32", 150, 64, 6, 50, 2, 1, 1, 2e-3), ("f32", 203, 96, 8, 72, 3, 3, 3, 2e-3), ("f32", 1, 64, 4, 32, 2, 1, 2, 2e-3),
    ("bf16", 300, 256, 8, 256, 2, 1, 2, 5e-2), ("bf16", 257, 128, 16, 384, 4, 2, 2, 5e-2)])
def test_stack_against_plain(L, dtype, T, d, E, F, k, P, n, tol):
    sh = mi.MoEShape("b", T, d, E, F, k, dtype, n_parties=P, normalize_topk=1)
    rule = L.make_gate_rule(L.MOE_SCORE_SIGMOID, 2, 2 if E == 4 else 1 if E == 6 else 2, 1, 1.5)
    net, x, dout = build(sh, n, rule, T + d)
    cut = [0] + [T * p // P for p in range(1, P)] + [T]
    net.layer.party_offsets.copy_(torch.tensor(cut, dtype=torch.int32))
    bias0 = [b.balance_bias.clone() for b in net.blocks]
    out = net.forward(x).clone()
    dx = net.backward(dout).clone()
    net.check_status()
    picks = [b.topk_idx.long() for b in net.blocks]
    ref = plain(net, sh, picks, x, dout, 1.5, net.out.dtype, cut)
    near("out", out, ref["out"], tol)
    near("dx", dx, ref["dx"], tol)
    near("gamma", net.dgamma, ref["gamma"], tol)
    near("beta", net.dbeta, ref["beta"], tol)
    for i, b in enumerate(net.blocks):
        for name, g in b.grads().items():
            near((i, name), g, ref[i][name], tol)
        c = b.counts.long()
        assert torch.equal(b.balance_bias, bias0[i] + 1e-3 * torch.sign(c.sum(1, keepdim=True) - E * c).float())
        assert int(c.sum()) == T * k
    # the same batch again, with the first one's balance bias: the same bits
    for b, v in zip(net.blocks, bias0):
        b.balance_bias.copy_(v)
    first = {i: {m: g.clone() for m, g in b.grads().items()} for i, b in enumerate(net.blocks)}
    assert torch.equal(net.forward(x), out) and torch.equal(net.backward(dout), dx)
    assert all(torch.equal(g, first[i][m]) for i, b in enumerate(net.blocks) for m, g in b.grads().items())
    full = sum(t.numel() for t in (x,)) * net.out.element_size() + T * k * (3 * F + d) * net.out.element_size()
    if T > 100:  # a half of what 16 bits take, a quarter of 32 bits, and the tables
        assert net.kept_bytes() < n * (0.62 if dtype == "bf16" else 0.34) * full + n * T * (E + 2 * k + 2) * 4 + 2 * T * d


@pytest.mark.parametrize("dtype,T,d,E,F,k,S,P", [("bf16", 500, 256, 8, 384, 2, 1, 1), ("bf16", 700, 512, 4, 256, 2, 0, 2),
                                              ("f32", 120, 60, 5, 50, 2, 2, 1), ("bf16", 0, 128, 4, 128, 1, 1, 1)])
def test_expert_backward_from_a_checkpoint(L, dtype, T, d, E, F, k, S, P):
    """Against the 16- or 32-bit backward on the values that the checkpoint holds: the two differ by dA's rounding
    (bf16: 2^-8) and summation order."""
    from paper_2506_02965_gb300.layer import MoELayer
    sh = mi.MoEShape("c", T, d, E, F, k, dtype, n_parties=P, n_shared=S, d_ff_shared=128 if S else 0)
    lay = MoELayer(sh)
    g = torch.Generator(device="cuda").manual_seed(T + d)
    for t, std in ((lay.x, 1.0), (lay.dout, 1.0), (lay.w_router, 0.1), (lay.w1, 0.1), (lay.w2, 0.1), (lay.ws1, 0.1), (lay.ws2, 0.1)):
        if t is not None:
            t.normal_(0.0, std, generator=g)
    lay.party_offsets.copy_(torch.tensor([0] + [T * p // P for p in range(1, P)] + [T], dtype=torch.int32))
    lay.forward()
    mt = L.MOE_BF16 if dtype == "bf16" else L.MOE_F32
    TK = T * k
    q = torch.empty(TK, 2 * F, dtype=torch.int8, device="cuda")
    sc = torch.empty(TK, L.ckpt_blocks(2 * F), device="cuda")
    L.moe_ckpt_pack(TK, 2 * F, mt, lay.h_gu, q, sc)
    L.moe_combine_bwd(lay.cfg, lay.dout, lay.y_perm, lay.topk_w, lay.slot_of, lay.dy_perm, lay.dtopk_w)
    names = ["dx_perm", "dw1", "dw2"] + (["dx_sh", "dws1", "dws2"] if S else [])
    dact, act = torch.empty(TK, F, dtype=lay.dt, device="cuda"), torch.empty(TK, F, dtype=lay.dt, device="cuda")
    L.moe_expert_ffn_bwd_ckpt(lay.cfg, lay.x_perm, lay.offsets, lay.w1, lay.w2, q, sc, lay.dy_perm, dact, act, lay.dh, lay.dx_perm,
                              lay.dw1, lay.dw2, lay.x, lay.dout, lay.ws1, lay.ws2, lay.h_gu_sh, lay.act_sh, lay.dh_sh, lay.dx_sh,
                              lay.dws1, lay.dws2, group_expert=lay.group_expert)
    got = {m: getattr(lay, m).clone() for m in names}
    held_gu = (q.float() * sc.repeat_interleave(128, 1)[:, :2 * F])
    lay.h_gu.copy_(held_gu)
    G, U = lay.h_gu.float().chunk(2, 1)
    lay.act.copy_(G * torch.sigmoid(G) * U)
    lay.ffn_bwd(torch.cuda.current_stream())
    assert status(L) == 0
    for m in names:
        ref = getattr(lay, m).double()
        if ref.numel():
            near(m, got[m], ref, 1.5e-2 if dtype == "bf16" else 1e-5)


def test_bad_stacks_are_refused(L):
    from paper_2506_02965_gb300.block import PreNormMoE
    with pytest.raises(ValueError, match="shared"):
        PreNormMoE(mi.MoEShape("b", 8, 128, 4, 128, 2, "bf16", n_shared=1, d_ff_shared=128), 1)
    with pytest.raises(ValueError, match="n_blocks"):
        PreNormMoE(mi.MoEShape("b", 8, 128, 4, 128, 2, "bf16"), 0)


def test_no_tokens(L):
    """A batch without tokens: weight gradients of zero, the bias as it was."""
    sh = mi.MoEShape("b", 0, 128, 4, 128, 2, "bf16")
    net, x, dout = build(sh, 2, L.make_gate_rule(L.MOE_SCORE_SIGMOID), 3)
    bias = [b.balance_bias.clone() for b in net.blocks]
    for b in net.blocks:
        for g in b.grads().values():
            g.fill_(3.0)
    assert net.forward(x).numel() == 0 and net.backward(dout).numel() == 0
    net.check_status()
    for b, v in zip(net.blocks, bias):
        assert all(float(g.float().abs().max()) == 0 for g in b.grads().values()) and torch.equal(b.balance_bias, v)


@pytest.mark.parametrize("which", ["x", "out"])
@pytest.mark.parametrize("n", [1, 2, 3])
def test_input_in_the_layers_own_buffers(L, n, which):
    """x may lie in the input or the output buffer of the stack's layer: the same bits as from a buffer of its own, and x as it was."""
    sh = mi.MoEShape("b", 130, 128, 8, 128, 2, "bf16", normalize_topk=1)
    net, x, dout = build(sh, n, L.make_gate_rule(L.MOE_SCORE_SIGMOID), 17)
    bias = [b.balance_bias.clone() for b in net.blocks]
    out, dx = net.forward(x).clone(), net.backward(dout).clone()
    grads = [{m: g.clone() for m, g in b.grads().items()} for b in net.blocks]
    for b, v in zip(net.blocks, bias):
        b.balance_bias.copy_(v)
    buf = getattr(net.layer, which)
    buf.copy_(x)
    assert torch.equal(net.forward(buf), out) and torch.equal(net.backward(dout), dx)
    net.check_status()
    assert all(torch.equal(g, grads[i][m]) for i, b in enumerate(net.blocks) for m, g in b.grads().items())
    assert torch.equal(buf, x)


def test_the_layers_own_weights_are_not_the_blocks(L):
    """A pass lends the layer the blocks' weights and tables and takes them back: what a caller puts into the layer between two
    passes does not reach a block."""
    sh = mi.MoEShape("b", 40, 128, 8, 128, 2, "bf16", normalize_topk=1)
    net, x, dout = build(sh, 2, L.make_gate_rule(L.MOE_SCORE_SIGMOID), 18)
    want = [{m: p.clone() for m, p in b.params().items()} for b in net.blocks]
    for step in (lambda: net.forward(x), lambda: net.backward(dout)):
        step()
        for t in (net.layer.w_router, net.layer.w1, net.layer.w2, net.layer.dw1, net.layer.dw2):
            t.fill_(3.0)
        for b, v in zip(net.blocks, want):
            assert all(torch.equal(p, v[m]) for m, p in b.params().items())
    assert all(float((g.float() - 3).abs().max()) > 0 for b in net.blocks for g in b.grads().values())


def test_buffers_of_the_expert_backward(L):
    """Buffers with room to spare give the same bits; too small, strided or of another type are refused before any of them is
    written, and so is a workspace smaller than its bytes."""
    T, d, E, F, k = 200, 128, 4, 256, 2
    cfg, TK, bf = L.make_config(T, d, E, F, k), T * k, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(3)

    def normal(*s, std=1.0):
        return torch.empty(*s, device="cuda").normal_(0.0, std, generator=g).to(bf)

    q, sc = torch.empty(TK, 2 * F, dtype=torch.int8, device="cuda"), torch.empty(TK, L.ckpt_blocks(2 * F), device="cuda")
    L.moe_ckpt_pack(TK, 2 * F, L.MOE_BF16, normal(TK, 2 * F), q, sc)
    a = {"x_perm": normal(TK, d), "offsets": torch.tensor([0, 70, 70, 250, TK], dtype=torch.int32, device="cuda"),
         "w1": normal(E, 2 * F, d, std=0.1), "w2": normal(E, d, F, std=0.1), "gu_q": q, "gu_scale": sc, "dy_perm": normal(TK, d)}
    outs = {"dact": TK * F, "act": TK * F, "dh": TK * 2 * F, "dx_perm": TK * d, "dw1": E * 2 * F * d, "dw2": E * d * F}
    exact = {m: torch.zeros(n, dtype=bf, device="cuda") for m, n in outs.items()}
    room = {m: torch.zeros(n + 64, dtype=bf, device="cuda") for m, n in outs.items()}
    L.moe_expert_ffn_bwd_ckpt(cfg, **a, **exact)
    L.moe_expert_ffn_bwd_ckpt(cfg, **{m: torch.cat([t.flatten(), t.flatten()[:64]]) for m, t in a.items()}, **room)
    assert status(L) == 0
    for m, n in outs.items():
        assert torch.equal(room[m][:n], exact[m]) and float(room[m][n:].abs().max()) == 0 and float(exact[m].abs().max()) > 0
        assert torch.isfinite(exact[m].float()).all()
    for m in [*a, *outs]:
        t = {**a, **exact}[m]
        for bad in (t.flatten()[:-1], t.flatten()[::2], t.double()):
            with pytest.raises(L.MoEError, match=f"{m}: expected a dense GPU tensor"):
                L.moe_expert_ffn_bwd_ckpt(cfg, **{**a, **room, m: bad})
    n = L.moe_layer_norm_workspace_size(T, d)
    rows = [normal(T, d), normal(T, d), None, None, *(torch.zeros(s, device="cuda") for s in (T, T, d)), None, normal(T, d),
            torch.zeros(d, device="cuda"), None]
    for bad in (torch.empty(n - 1, dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.uint8),
                torch.empty(2 * n, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(L.MoEError, match="workspace"):
            L.moe_layer_norm_bwd(T, d, L.MOE_BF16, *rows, bad, n)
    L.moe_layer_norm_bwd(T, d, L.MOE_BF16, *rows, torch.empty(-(-n // 4), device="cuda"), n)
    assert status(L) == 0
