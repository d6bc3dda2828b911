"""The operators around the layer on buffers off a 16-byte boundary, each argument by itself, and past 32-bit offsets.

Bounds are those of the operators' own tests (layer norm: 256 u of the output's size, 512 u of the gradients'; gating: 64 u of a weight, 256 u
of a gradient's size; SwiGLU: 32 u, or 2^-19 of bf16; half a spacing of bf16, at most 2^-8; u = 2^-24), twice where two calls
are compared that may add in another order. Whole numbers and 8-bit values are equal."""
import pytest
import torch

from tests.gpu_util import need_gpu, status

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def L():
    return need_gpu()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def off(t, by):
    """A copy of t that starts `by` elements past a 16-byte boundary; the elements before it are NaN or -1 (canaries)."""
    if t is None or not by:
        return t
    whole = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
    whole[:by] = float("nan") if t.is_floating_point() else -1
    whole[by:] = t.flatten()
    return whole[by:].view(t.shape)


def canary(t, by):
    """The elements before t are as `off` left them."""
    before = torch.as_strided(t, (by,), (1,), t.storage_offset() - by)
    return bool(torch.isnan(before).all()) if t.is_floating_point() else bool((before == -1).all())


def within(what, got, ref, bound):
    d = (got.double() - ref.double()).abs()
    assert not (d > bound).any(), (what, float(d.max()))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", [(40, 512), (37, 333), (3, 16384)])
@pytest.mark.parametrize("residual", [False, True])
def test_norm(L, R, d, name, residual):
    dt, mt = (torch.bfloat16, L.MOE_BF16) if name == "bf16" else (torch.float32, L.MOE_F32)
    half = 2.0 ** -8 if name == "bf16" else 0.0
    g = gen(R + d)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")

    a = {"x": (normal(R, d) + 0.5).to(dt), "residual": normal(R, d).to(dt) if residual else None, "gamma": 1 + 0.2 * normal(d),
         "beta": 0.2 * normal(d)}
    o = {"h": torch.zeros(R, d, dtype=dt, device="cuda") if residual else None, "y": torch.zeros(R, d, dtype=dt, device="cuda"),
         "mean": torch.zeros(R, device="cuda"), "rstd": torch.zeros(R, device="cuda"),
         "h_q": torch.zeros(R, d, dtype=torch.int8, device="cuda"), "h_scale": torch.zeros(R, -(-d // 128), device="cuda")}

    def forward(a, o):
        L.moe_layer_norm_fwd(R, d, mt, a["x"], a["residual"], a["gamma"], a["beta"], EPS, o["h"], o["y"], o["mean"], o["rstd"], o["h_q"],
                             o["h_scale"])

    forward(a, o)
    top = (a["x"].double() + (a["residual"].double() if residual else 0)).abs().amax(1, keepdim=True)
    rs = o["rstd"].double()[:, None]
    tol = 512 * U * (a["gamma"].double().abs() * top * rs + a["beta"].double().abs()) + 2 * half * o["y"].double().abs()
    for by in (1, 2):
        for which in [n for n, t in {**a, **o}.items() if t is not None]:
            a2 = {n: off(t, by if n == which else 0) for n, t in a.items()}
            o2 = {n: off(torch.zeros_like(t), by if n == which else 0) if t is not None else None for n, t in o.items()}
            forward(a2, o2)
            assert status(L) == 0
            within(which, o2["y"], o["y"], tol)
            assert torch.equal(o2["h_q"], o["h_q"]) and torch.equal(o2["h_scale"], o["h_scale"]), which
            assert not residual or torch.equal(o2["h"], o["h"]), which
            within(which, o2["mean"], o["mean"], 512 * U * top[:, 0])
            within(which, o2["rstd"], o["rstd"], 1024 * U * (1 + (top[:, 0] * rs[:, 0]) ** 2) * rs[:, 0])
            assert canary({**a2, **o2}[which], by), which

    h = o["h"] if residual else a["x"]
    held = o["h_q"].float() * o["h_scale"].repeat_interleave(128, 1)[:, :d]
    b = {"dy": normal(R, d).to(dt), "h": h, "h_q": o["h_q"], "h_scale": o["h_scale"], "mean": o["mean"], "rstd": o["rstd"],
         "gamma": a["gamma"], "dh": normal(R, d).to(dt)}
    n = L.moe_layer_norm_workspace_size(R, d)
    outs = {"dx": torch.zeros(R, d, dtype=dt, device="cuda"), "dgamma": torch.zeros(d, device="cuda"), "dbeta": torch.zeros(d, device="cuda"),
            "workspace": torch.zeros(n // 4, device="cuda")}

    def backward(b, outs, q):
        L.moe_layer_norm_bwd(R, d, mt, b["dy"], None if q else b["h"], b["h_q"] if q else None, b["h_scale"] if q else None, b["mean"],
                             b["rstd"], b["gamma"], b["dh"], outs["dx"], outs["dgamma"], outs["dbeta"], outs["workspace"], n)

    for q in (False, True):
        backward(b, outs, q)
        xh = ((held if q else h).double() - o["mean"].double()[:, None]) * rs
        dy = b["dy"].double()
        gg = dy * a["gamma"].double()
        tol = 1024 * U * rs * gg.abs().amax(1, keepdim=True) * (1 + xh.abs().amax(1, keepdim=True) ** 2) \
            + 8 * U * b["dh"].double().abs() + 2 * half * outs["dx"].double().abs()
        size = (dy * xh).abs().sum(0) + dy.abs().sum(0) * (top.amax() * rs.amax())
        for by in (1, 2):
            for which in [m for m in [*b, *outs] if m not in (("h",) if q else ("h_q", "h_scale"))]:
                b2 = {m: off(t, by if m == which else 0) for m, t in b.items()}
                o2 = {m: off(torch.zeros_like(t), by if m == which else 0) for m, t in outs.items()}
                backward(b2, o2, q)
                assert status(L) == 0
                within((q, which), o2["dx"], outs["dx"], tol)
                within((q, which), o2["dgamma"], outs["dgamma"], 1024 * U * size)
                within((q, which), o2["dbeta"], outs["dbeta"], 1024 * U * dy.abs().sum(0))
                assert canary({**b2, **o2}[which], by), which


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("T,E,k,G,top,best", [(300, 256, 8, 8, 4, 2), (257, 64, 6, 1, 1, 1), (300, 128, 2, 4, 2, 1), (9000, 256, 8, 4, 2, 2)])
def test_gate(L, T, E, k, G, top, best, sigmoid):
    g = gen(T + E)
    P, scale = 2, 1.5
    cfg = L.make_config(T, 128, E, 128, k, P, normalize_topk=1)
    r = L.make_gate_rule(L.MOE_SCORE_SIGMOID if sigmoid else L.MOE_SCORE_SOFTMAX, G, top, best, scale)
    z = torch.randn(T, E, generator=g, device="cuda")
    z[torch.rand(T, E, generator=g, device="cuda") < 0.05] = -float("inf")
    a = {"logits": z, "bias": 0.1 * torch.randn(P, E, generator=g, device="cuda"),
         "po": torch.tensor([0, T // 3, T], dtype=torch.int32, device="cuda")}
    o = {"scores": torch.zeros(T, E, device="cuda"), "idx": torch.zeros(T, k, dtype=torch.int32, device="cuda"),
         "w": torch.zeros(T, k, device="cuda"), "counts": torch.zeros(P, E, dtype=torch.int32, device="cuda")}

    def forward(a, o):
        L.moe_gate(cfg, r, a["logits"], a["bias"], a["po"], o["scores"], o["idx"], o["w"], o["counts"])

    forward(a, o)
    b = {"logits": z, "idx": o["idx"], "g": torch.randn(T, k, generator=g, device="cuda"),
         "aux": 0.1 * torch.rand(P, E, generator=g, device="cuda"), "po": a["po"]}
    outs = {"dlogits": torch.zeros(T, E, device="cuda")}

    def backward(b, outs):
        L.moe_gate_bwd(cfg, r, b["logits"], b["idx"], b["g"], b["aux"], b["po"], outs["dlogits"])

    backward(b, outs)
    S = o["scores"].gather(1, o["idx"].long()).double().sum(1, keepdim=True)
    size = scale * b["g"].double().abs().amax(1, keepdim=True) * torch.where(S > 0, 2 / S, 0.0) + 0.1
    for by in (1, 2, 3):
        for which in [*a, *o]:
            a2 = {n: off(t, by if n == which else 0) for n, t in a.items()}
            o2 = {n: off(torch.zeros_like(t), by if n == which else 0) for n, t in o.items()}
            forward(a2, o2)
            assert status(L) == 0 and torch.equal(o2["idx"], o["idx"]) and torch.equal(o2["counts"], o["counts"]), which
            within(which, o2["w"], o["w"], 128 * U * o["w"].double() + 2.0 ** -125)
            within(which, o2["scores"], o["scores"], 128 * U * o["scores"].double() + 2.0 ** -125)
            assert canary({**a2, **o2}[which], by), which
        for which in [*b, *outs]:
            b2 = {n: off(t, by if n == which else 0) for n, t in b.items()}
            o2 = {n: off(torch.zeros_like(t), by if n == which else 0) for n, t in outs.items()}
            backward(b2, o2)
            assert status(L) == 0
            within(which, o2["dlogits"], outs["dlogits"], 512 * U * size)
            assert canary({**b2, **o2}[which], by), which


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,F", [(33, 256), (20, 136), (40, 100)])
def test_swiglu(L, R, F, dt):
    g = gen(R + F)
    mt = L.MOE_BF16 if dt == torch.bfloat16 else L.MOE_F32
    q, scale = torch.empty(R, 2 * F, dtype=torch.int8, device="cuda"), torch.empty(R, -(-2 * F // 128), device="cuda")
    L.moe_ckpt_pack(R, 2 * F, mt, (1.5 * torch.randn(R, 2 * F, generator=g, device="cuda")).to(dt), q, scale)
    a = {"q": q, "scale": scale, "dact": torch.randn(R, F, generator=g, device="cuda").to(dt)}
    o = {"act": torch.zeros(R, F, dtype=dt, device="cuda"), "dh": torch.zeros(R, 2 * F, dtype=dt, device="cuda")}
    held = (q.float() * scale.repeat_interleave(128, 1)[:, :2 * F]).double()
    G, V, da = held[:, :F], held[:, F:], a["dact"].double()
    sg = torch.sigmoid(G)
    ref = {"act": G * sg * V, "dh": torch.cat([da * V * sg * (1 + G * torch.sigmoid(-G)), da * G * sg], 1)}
    mag = {"act": V.abs() * (1 + G.abs()), "dh": torch.cat([(da * V).abs() * (1 + G.abs()), da.abs() * (1 + G.abs())], 1)}
    rel, half = (2.0 ** -19, 2.0 ** -8) if dt == torch.bfloat16 else (32 * U, 0.0)
    for which in [*a, *o]:
        for by in (1, 2, 3, 4):
            a2 = {n: off(t, by if n == which else 0) for n, t in a.items()}
            o2 = {n: off(torch.zeros_like(t), by if n == which else 0) for n, t in o.items()}
            L.moe_ckpt_swiglu_bwd(R, F, mt, a2["q"], a2["scale"], a2["dact"], o2["act"], o2["dh"])
            assert status(L) == 0
            for n in ref:
                within((which, n), o2[n], ref[n], rel * mag[n] + half * ref[n].abs() + 2.0 ** -120)
            assert canary({**a2, **o2}[which], by), which


@pytest.mark.parametrize("sigmoid", [False, True])
def test_gate_past_2_31_logits(L, sigmoid):
    """The first and last tokens of 8.6 GB of logits: the picks of a small call, its weights and gradients."""
    T, E, k, n = 8_400_007, 256, 8, 100
    assert T * E > 1 << 31
    z = torch.empty(T, E, device="cuda").normal_(generator=gen(1))
    z[T - n:] = z[:n]
    gr, aux = torch.randn(n, k, generator=gen(2), device="cuda"), 0.1 * torch.rand(1, E, generator=gen(3), device="cuda")
    r = L.make_gate_rule(L.MOE_SCORE_SIGMOID if sigmoid else L.MOE_SCORE_SOFTMAX, 8, 4, 2, 1.5)
    res = []
    for m in (n, T):
        cfg = L.make_config(m, 128, E, 128, k, normalize_topk=1)
        idx, w = torch.empty(m, k, dtype=torch.int32, device="cuda"), torch.empty(m, k, device="cuda")
        counts, sc, dz = torch.empty(1, E, dtype=torch.int32, device="cuda"), torch.empty(m, E, device="cuda"), torch.empty(m, E, device="cuda")
        g = torch.zeros(m, k, device="cuda")
        g[:n], g[m - n:] = gr, gr
        L.moe_gate(cfg, r, z[:m], None, None, sc, idx, w, counts)
        L.moe_gate_bwd(cfg, r, z[:m], idx, g, aux, None, dz)
        assert status(L) == 0 and int(counts.sum()) == m * k
        res.append((idx, w, sc, dz))
    (i0, w0, s0, d0), (i1, w1, s1, d1) = res
    size = 1.5 * gr.double().abs().amax(1, keepdim=True) * 2 / s0.gather(1, i0.long()).double().sum(1, keepdim=True) + 0.1
    for part in (slice(0, n), slice(T - n, T)):
        assert torch.equal(i1[part], i0)
        within("w", w1[part], w0, 128 * U * w0.double())
        within("scores", s1[part], s0, 128 * U * s0.double())
        within("dlogits", d1[part], d0, 512 * U * size)
    del z, res, i1, w1, s1, d1, idx, w, sc, dz, g
    torch.cuda.empty_cache()


@pytest.mark.parametrize("R,F", [(1_000_003, 1080), ((1 << 30) + 5, 1)])
def test_swiglu_past_2_31_elements(L, R, F):
    """The first and last rows of more than 2^31 values, and of more rows than one launch counts: those of a small call."""
    assert R * 2 * F > 1 << 31
    n, bf = 5, torch.bfloat16
    gu, da = torch.randn(n, 2 * F, generator=gen(4), device="cuda").to(bf), torch.randn(n, F, generator=gen(5), device="cuda").to(bf)
    x = torch.zeros(R, 2 * F, dtype=bf, device="cuda")
    x[:n], x[-n:] = gu, gu
    dact = torch.zeros(R, F, dtype=bf, device="cuda")
    dact[:n], dact[-n:] = da, da
    got = []
    for m, h, d in ((n, gu, da), (R, x, dact)):
        q, s = torch.empty(m, 2 * F, dtype=torch.int8, device="cuda"), torch.empty(m, -(-2 * F // 128), device="cuda")
        L.moe_ckpt_pack(m, 2 * F, L.MOE_BF16, h, q, s)
        act, dh = torch.empty(m, F, dtype=bf, device="cuda"), torch.empty(m, 2 * F, dtype=bf, device="cuda")
        L.moe_ckpt_swiglu_bwd(m, F, L.MOE_BF16, q, s, d, act, dh)
        L.moe_ckpt_unpack(m, 2 * F, L.MOE_BF16, q, s, h)
        assert status(L) == 0
        got.append((q, s, act, dh, h))
    for small, large in zip(*got):
        assert torch.equal(large[:n], small) and torch.equal(large[-n:], small)
        assert not large[n:-n].any()
    del got, x, dact, q, s, act, dh, h, d, small, large
    torch.cuda.empty_cache()
