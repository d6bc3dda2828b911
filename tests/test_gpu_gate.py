"""Gating rules (moe_gate, moe_route_gate, moe_gate_bwd, moe_gate_balance) against a plain 64-bit
implementation, token by token.

Picks are compared wherever the decision is not within the keys' own rounding: a key or a sum of two is
off by at most 8 u of a magnitude below 8 (u = 2^-24), so a token is decided when the distinct 64-bit keys it
compares are 4e-6 apart; equal inputs give equal keys and are decided by the lower id. Weights: the
exponentials are off by 12 u (argument and function), the sum of 256 by 13 u more, the quotients and
products by 8 u: within 64 u of the weight. dlogits: within 256 u of scale max|g| (2 / sum) + max|aux|, or of
scale max|g| + max|aux| without renormalisation."""
import numpy as np
import pytest
import torch

from tests.gpu_util import need_gpu, status

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
GAP = 4e-6


@pytest.fixture(scope="module")
def L():
    return need_gpu()


def scores(z, sigmoid):
    z = np.where(np.isnan(z), -np.inf, z)
    with np.errstate(all="ignore"):
        if sigmoid:
            return z, 1 / (1 + np.exp(-z))
        m = z.max()
        e = np.exp(z - (0 if m == -np.inf else m))
        return z, e / e.sum() if e.sum() > 0 else e * 0


def order(v, n):
    """Indices by descending value, equal ones by index; and whether the n + 1 largest, which decide the
    first n, are apart wherever they are finite and differ."""
    o = sorted(range(len(v)), key=lambda i: (-v[i], i))
    f = v[o[:n + 1]]
    d = -np.diff(f[np.isfinite(f)])
    return o, bool(((d == 0) | (d > GAP)).all())


def token(z, b, k, sigmoid, G, top, best, normalize, scale):
    E = len(z)
    z, s = scores(z, sigmoid)
    key = np.where(z == -np.inf, -np.inf, (s if sigmoid else z) + b)
    gs = E // G
    group = np.array([np.sort(key[g * gs:(g + 1) * gs])[::-1][:best].sum() for g in range(G)])
    go, sure1 = order(group, top)
    kept = sorted(go[:top])
    ids = [e for g in kept for e in range(g * gs, (g + 1) * gs)]
    o, sure2 = order(key[ids], k)
    I = [ids[i] for i in o[:k]]
    S = s[I].sum() if normalize else 1.0
    w = scale * s[I] / S if S > 0 else np.zeros(k)
    return I, w, s, (sure1 or top == G) and sure2


def rule(L, sigmoid, G, top, best, scale):
    return L.make_gate_rule(L.MOE_SCORE_SIGMOID if sigmoid else L.MOE_SCORE_SOFTMAX, G, top, best, scale)


def run(L, T, E, k, z, bias, sigmoid, G=1, top=1, best=1, normalize=0, scale=1.0, po=None, want_scores=False):
    P = len(po) - 1 if po else 1
    cfg = L.make_config(T, 128, E, 128, k, P, normalize_topk=normalize)
    idx, w = torch.full((T, k), -5, dtype=torch.int32, device="cuda"), torch.full((T, k), 9.0, device="cuda")
    counts = torch.full((P, E), 33, dtype=torch.int32, device="cuda")
    sc = torch.full((T, E), 9.0, device="cuda") if want_scores else None
    pod = torch.tensor(po, dtype=torch.int32, device="cuda") if po else None
    r = rule(L, sigmoid, G, top, best, scale)
    L.moe_gate(cfg, r, z, bias, pod, sc, idx, w, counts)
    assert status(L) == 0
    return cfg, r, pod, idx, w, counts, sc


def gradient(z, I, s, g, aux, sigmoid, normalize, scale):
    """dlogits of a token in 64 bits."""
    z = np.where(np.isnan(z), -np.inf, z)
    ds = aux.astype(np.float64).copy()
    S = s[I].sum()
    if normalize:
        w = scale * s[I] / S if S > 0 else np.zeros(len(I))
        add = (scale * g - (g * w).sum()) / S if S > 0 else np.zeros(len(I))
    else:
        add = scale * g
    ds[I] += add
    if sigmoid:
        with np.errstate(all="ignore"):
            return ds * s * (1 / (1 + np.exp(z)))
    return s * (ds - (ds * s).sum())


CASES = [
    # T, E, k, sigmoid, G, top, best, normalize, scale, bias, parties
    (1, 1, 1, False, 1, 1, 1, 0, 1.0, False, None),
    (3, 2, 2, True, 1, 1, 1, 1, 1.0, True, None),
    (70, 5, 3, True, 1, 1, 2, 1, 2.5, True, [0, 10, 70]),
    (33, 16, 2, False, 1, 1, 1, 0, 1.0, False, None),
    (40, 64, 6, False, 1, 1, 1, 1, 1.0, True, None),
    (64, 12, 4, True, 3, 2, 2, 0, 1.0, True, None),
    (50, 63, 7, True, 7, 3, 2, 1, 2.5, True, [0, 0, 20, 50]),
    (45, 96, 8, False, 32, 5, 2, 1, 1.5, True, None),
    (30, 128, 8, True, 8, 3, 1, 1, 2.5, False, None),
    (129, 176, 7, True, 8, 6, 1, 0, 2.5, True, None),
    (61, 256, 8, True, 8, 4, 2, 1, 2.5, True, [0, 30, 61]),
    (25, 255, 8, True, 3, 1, 2, 1, 1.0, True, None),
    (20, 250, 5, False, 5, 2, 1, 0, 1.0, True, None),
    (21, 248, 8, False, 31, 1, 2, 1, 1.0, False, None),
    (2500, 20, 3, True, 4, 2, 2, 1, 1.0, True, [0, 1, 700, 2500]),
]


@pytest.mark.parametrize("T,E,k,sigmoid,G,top,best,normalize,scale,bias,po", CASES)
@pytest.mark.parametrize("masked", [False, True])
def test_rule_and_backward(L, T, E, k, sigmoid, G, top, best, normalize, scale, bias, po, masked):
    gen = torch.Generator(device="cuda").manual_seed(T + 3 * E + k)
    z = torch.randn(T, E, generator=gen, device="cuda")
    P = len(po) - 1 if po else 1
    b = 0.1 * torch.randn(P, E, generator=gen, device="cuda") if bias else None
    if E > 3:  # equal keys: the lower id first
        z[:, E - 1] = z[:, 1]
        if bias:
            b[:, E - 1] = b[:, 1]
    if masked:
        z[torch.rand(T, E, generator=gen, device="cuda") < 0.4] = -float("inf")
        z[torch.rand(T, E, generator=gen, device="cuda") < 0.05] = float("nan")
        z[::5] = -float("inf")  # whole rows
        z[1::7, 0] = torch.finfo(torch.float32).min
    cfg, r, pod, idx, w, counts, sc = run(L, T, E, k, z, b, sigmoid, G, top, best, normalize, scale, po, want_scores=True)
    g, aux = torch.randn(T, k, generator=gen, device="cuda"), 0.1 * torch.rand(P, E, generator=gen, device="cuda")
    dz = torch.full((T, E), 9.0, device="cuda")
    L.moe_gate_bwd(cfg, r, z, idx, g, aux, pod, dz)
    assert status(L) == 0
    zh, bh = z.double().cpu().numpy(), b.double().cpu().numpy() if bias else np.zeros((P, E))
    ih, wh, sh, dzh, gh, ah = (t.double().cpu().numpy() for t in (idx, w, sc, dz, g, aux))
    cut = po or [0, T]
    decided = 0
    for t in range(T):
        p = max(i for i in range(P) if cut[i] <= t and (t < cut[i + 1]))
        I, wr, s, sure = token(zh[t], bh[p], k, sigmoid, G, top, best, normalize, scale)
        got = ih[t].astype(int).tolist()
        assert len(set(got)) == k and all(0 <= e < E for e in got)
        if sure:
            decided += 1
            assert got == I, (t, got, I)
        S = s[got].sum() if normalize else 1.0
        wr = scale * s[got] / S if S > 0 else np.zeros(k)
        assert (np.abs(wh[t] - wr) <= 64 * U * np.abs(wr) + 2.0 ** -126).all()
        assert (np.abs(sh[t] - s) <= 64 * U * s + 2.0 ** -126).all()
        ref = gradient(zh[t], got, s, gh[t], ah[p], sigmoid, normalize, scale)
        size = scale * np.abs(gh[t]).max() * (2 / S if normalize and S > 0 else 1) + np.abs(ah[p]).max()
        assert (np.abs(dzh[t] - ref) <= 256 * U * size).all(), (t, np.abs(dzh[t] - ref).max(), size)
    assert decided >= 0.95 * T - 1
    for p in range(P):
        n = np.bincount(ih[cut[p]:cut[p + 1]].astype(int).ravel(), minlength=E)
        assert (n == counts[p].cpu().numpy()).all()


def test_softmax_rule_is_the_plain_gating(L):
    """Softmax, one group, no bias, scale 1: the picks and counts of moe_route_from_logits, its weights and
    the dlogits of moe_route_bwd within rounding."""
    T, E, k, d = 1500, 60, 4, 128
    gen = torch.Generator(device="cuda").manual_seed(8)
    z = torch.randn(T, E, generator=gen, device="cuda")
    z[:, 40] = z[:, 3]
    for normalize in (0, 1):
        cfg, r, _, idx, w, counts, sc = run(L, T, E, k, z, None, False, normalize=normalize, want_scores=True)
        probs, i2, w2, c2 = torch.empty_like(z), torch.empty_like(idx), torch.empty_like(w), torch.empty_like(counts)
        L.moe_route_from_logits(cfg, z, None, probs, i2, w2, c2)
        assert torch.equal(idx, i2) and torch.equal(counts, c2)
        torch.testing.assert_close(w, w2, rtol=64 * U, atol=0)
        torch.testing.assert_close(sc, probs, rtol=64 * U, atol=0)
        x, wr = torch.randn(T, d, generator=gen, device="cuda").bfloat16(), torch.randn(1, E, d, generator=gen, device="cuda").bfloat16()
        g, aux = torch.randn(T, k, generator=gen, device="cuda"), torch.rand(1, E, generator=gen, device="cuda")
        ws = torch.empty(L.moe_workspace_size(cfg), dtype=torch.uint8, device="cuda")
        outs = []
        for _ in range(2):
            outs.append([torch.empty_like(z), torch.empty_like(wr), torch.empty(1, E, device="cuda"), torch.empty_like(x)])
        dz, dw, db, dx = outs[0]
        L.moe_gate_bwd(cfg, r, z, idx, g, aux, None, dz, x, wr, dw, db, dx, ws, ws.numel())
        dz2, dw2, db2, dx2 = outs[1]
        L.moe_route_bwd(cfg, x, wr, probs, idx, w2, g, aux, None, dz2, dw2, db2, dx2, ws, ws.numel())
        assert status(L) == 0
        size = float(g.abs().max()) * (float((2 / probs.gather(1, idx.long()).sum(1)).max()) if normalize else 1) + 1
        assert (dz - dz2).abs().max() <= 512 * U * size
        # the same products of dlogits that differ in their last bits: half a spacing of bf16 on each of
        # dlogits and the result, over the sums' magnitudes
        for a, b, mag in ((dw[0], dw2[0], dz.abs().T @ x.float().abs()), (dx, dx2, dz.abs() @ wr[0].float().abs())):
            assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * mag + 1e-6).all()
        assert ((db - db2).abs() <= 1e-5 * dz.abs().sum(0) + 1e-6).all()


@pytest.mark.parametrize("dtype,d,E,P", [("bf16", 256, 24, 1), ("bf16", 128, 130, 2), ("f32", 100, 9, 3)])
def test_router_products(L, dtype, d, E, P):
    """moe_route_gate takes moe_route's logits; moe_gate_bwd's products are those of its dlogits (bf16: rounded
    to bf16 as operands, 2^-8 of the sum of magnitudes)."""
    T, k = 333, 3
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(d + E)
    cfg = L.make_config(T, d, E, 128, k, P, normalize_topk=1, dtype=L.MOE_BF16 if dtype == "bf16" else L.MOE_F32)
    r = rule(L, True, 1, 1, 1, 2.0)
    x = torch.randn(T, d, generator=gen, device="cuda").to(dt)
    wr = (0.05 * torch.randn(P, E, d, generator=gen, device="cuda")).to(dt)
    rb, bb = 0.1 * torch.randn(P, E, generator=gen, device="cuda"), 0.1 * torch.randn(P, E, generator=gen, device="cuda")
    cut = [0] + [T * p // P for p in range(1, P)] + [T]
    po = torch.tensor(cut, dtype=torch.int32, device="cuda") if P > 1 else None
    f = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    i = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    z0, pr, i0, w0, c0 = f(T, E), f(T, E), i(T, k), f(T, k), i(P, E)
    L.moe_route(cfg, x, wr, rb, po, z0, pr, i0, w0, c0)
    z, sc, idx, w, counts = f(T, E), f(T, E), i(T, k), f(T, k), i(P, E)
    L.moe_route_gate(cfg, r, x, wr, rb, bb, po, z, sc, idx, w, counts)
    assert torch.equal(z, z0)
    idx2, w2, counts2 = i(T, k), f(T, k), i(P, E)
    L.moe_gate(cfg, r, z, bb, po, None, idx2, w2, counts2)
    assert torch.equal(idx, idx2) and torch.equal(w, w2) and torch.equal(counts, counts2)
    g = torch.randn(T, k, generator=gen, device="cuda")
    ws = torch.empty(L.moe_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    dz, dw, db, dx = f(T, E), torch.empty_like(wr), f(P, E), torch.empty_like(x)
    L.moe_gate_bwd(cfg, r, z, idx, g, None, po, dz, x, wr, dw, db, dx, ws, ws.numel())
    alone = f(T, E)
    L.moe_gate_bwd(cfg, r, z, idx, g, None, po, alone)
    assert status(L) == 0 and torch.equal(dz, alone)
    rel = 2.0 ** -7 if dtype == "bf16" else 1e-5
    for p in range(P):
        s = slice(cut[p], cut[p + 1])
        D, X, W = dz[s].double(), x[s].double(), wr[p].double()
        assert ((dw[p].double() - D.T @ X).abs() <= rel * (D.abs().T @ X.abs())).all()
        assert ((dx[s].double() - D @ W).abs() <= rel * (D.abs() @ W.abs())).all()
        assert ((db[p].double() - D.sum(0)).abs() <= 1e-5 * D.abs().sum(0) + 1e-9).all()


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("normalize", [0, 1])
def test_gradient_against_differences(L, sigmoid, normalize):
    """dlogits against central differences of the 64-bit weights at fixed picks: a step of 2^-12 leaves
    (2^-24 / 6) times a third derivative below 64."""
    T, E, k, step = 6, 10, 3, 2.0 ** -12
    gen = torch.Generator(device="cuda").manual_seed(21)
    z, g, aux = (torch.randn(*s, generator=gen, device="cuda") for s in ((T, E), (T, k), (1, E)))
    cfg, r, _, idx, w, _, _ = run(L, T, E, k, z, None, sigmoid, normalize=normalize, scale=1.5)
    dz = torch.empty_like(z)
    L.moe_gate_bwd(cfg, r, z, idx, g, aux, None, dz)
    ix, gd = idx.long(), g.double()

    def loss(z):
        s = torch.sigmoid(z) if sigmoid else torch.softmax(z, 1)
        p = s.gather(1, ix)
        w = 1.5 * p / p.sum(1, keepdim=True) if normalize else 1.5 * p
        return (w * gd).sum(1) + (s * aux.double()).sum(1)

    for e in range(E):
        h = torch.zeros(T, E, dtype=torch.float64, device="cuda")
        h[:, e] = step
        diff = (loss(z.double() + h) - loss(z.double() - h)) / (2 * step)
        assert (diff - dz[:, e].double()).abs().max() < 1e-4


def test_saturated_and_extreme_logits(L):
    """Large logits: sigmoid scores of exactly 1 tie by id; the type's lowest value is a score of 0 within reach,
    before one of -inf."""
    z = torch.zeros(3, 8, device="cuda")
    z[0] = torch.tensor([90., 95., float("inf"), -1., 90., 20., 200., 0.])
    z[1] = -float("inf")
    z[1, 6] = torch.finfo(torch.float32).min
    z[1, 2] = -120.0
    z[2] = torch.finfo(torch.float32).min
    _, _, _, idx, w, _, _ = run(L, 3, 8, 4, z, None, True)
    assert idx.tolist() == [[0, 1, 2, 4], [2, 6, 0, 1], [0, 1, 2, 3]]
    assert w[0].tolist() == [1.0] * 4 and w[1, 1:].tolist() == [0.0] * 3 and w[2].tolist() == [0.0] * 4
    _, _, _, idx, w, _, _ = run(L, 3, 8, 2, z, None, False, normalize=1)
    assert idx[1:].tolist() == [[2, 6], [0, 1]] and w[1].tolist() == [1.0, 0.0]
    assert torch.allclose(w[2], torch.full((2,), 0.5, device="cuda"))


def test_pick_out_of_range_is_recorded(L):
    z, g = torch.randn(4, 8, device="cuda"), torch.ones(4, 2, device="cuda")
    cfg, r, _, idx, _, _, _ = run(L, 4, 8, 2, z, None, True)
    good = torch.empty_like(z)
    L.moe_gate_bwd(cfg, r, z, idx, g, None, None, good)
    idx[2, 1] = 8
    dz = torch.empty_like(z)
    L.moe_gate_bwd(cfg, r, z, idx, g, None, None, dz)
    assert status(L) == L.MOE_ERR_DEVICE_CHECK and status(L) == 0
    assert torch.equal(dz[[0, 1, 3]], good[[0, 1, 3]]) and torch.isfinite(dz).all()


@pytest.mark.parametrize("P,E", [(1, 1), (2, 60), (3, 256)])
def test_balance(L, P, E):
    cfg = L.make_config(10, 128, E, 128, 1, P)
    gen = torch.Generator(device="cuda").manual_seed(E)
    counts = torch.randint(0, 9, (P, E), generator=gen, device="cuda", dtype=torch.int32)
    counts[0] = 2 ** 30  # equal loads, a sum past 32 bits
    b = torch.randn(P, E, generator=gen, device="cuda")
    out = torch.empty_like(b)
    L.moe_gate_balance(cfg, counts, 0.25, b, out)
    n = counts.long()
    assert torch.equal(out, b + 0.25 * torch.sign(n.sum(1, keepdim=True) - E * n).float())
    assert torch.equal(out[0], b[0])
    L.moe_gate_balance(cfg, counts, 0.25, b, b)
    assert torch.equal(b, out) and status(L) == 0


def test_no_tokens(L):
    counts = torch.full((2, 7), 3, dtype=torch.int32, device="cuda")
    cfg = L.make_config(0, 128, 7, 128, 2, 2)
    po = torch.zeros(3, dtype=torch.int32, device="cuda")
    L.moe_gate(cfg, L.make_gate_rule(), None, None, po, None, None, None, counts)
    assert status(L) == 0 and int(counts.abs().max()) == 0
    L.moe_gate_bwd(cfg, L.make_gate_rule(), None, None, None, None, po, None)
    assert status(L) == 0


def exact_by_sorting(L, z, b, k, sigmoid, G=1, top=1, best=1):
    """Picks from exact 32-bit keys by stable sorts (the scores in torch's 32-bit arithmetic)."""
    T, E = z.shape
    z = torch.where(torch.isnan(z), -float("inf"), z)
    key = 1.0 / (1.0 + torch.exp(-z)) if sigmoid else z
    key = torch.where(z == -float("inf"), z, key + b if b is not None else key)
    g = torch.sort(key.view(T, G, E // G), dim=2, descending=True, stable=True).values[..., :best].sum(2)
    order = torch.sort(g, dim=1, descending=True, stable=True).indices[:, :top]
    kept = torch.zeros(T, G, dtype=torch.int32, device="cuda").scatter_(1, order, 1).repeat_interleave(E // G, 1)
    idx = torch.sort(key, dim=1, descending=True, stable=True).indices
    last = torch.sort(kept.gather(1, idx), dim=1, descending=True, stable=True).indices
    return idx.gather(1, last)[:, :k].int()


@pytest.mark.parametrize("E,k,G,top,best", [(256, 8, 8, 4, 2), (256, 8, 1, 1, 1), (128, 2, 1, 1, 1), (64, 6, 4, 2, 1), (16, 2, 1, 1, 1),
                                            (96, 8, 3, 2, 2), (248, 5, 31, 7, 2), (30, 4, 5, 3, 1)])
@pytest.mark.parametrize("T", [37, 20011])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_picks_of_close_equal_and_crowded_keys(L, E, k, G, top, best, T, sigmoid):
    """Keys that the networks' approximate keys cannot tell apart (some units of the last place apart), equal ones
    few and many, all picks in one lane's experts, ranges past the sort keys', -inf in the bias: exact picks."""
    gen = torch.Generator(device="cuda").manual_seed(E + k + T)
    z = torch.randn(T, E, generator=gen, device="cuda")
    b = 0.05 * torch.randn(1, E, generator=gen, device="cuda")
    kind = torch.arange(T, device="cuda") % 9
    base = torch.randn(T, 1, generator=gen, device="cuda")
    near = (base * (1 + torch.randint(-6, 7, (T, E), generator=gen, device="cuda") * 2.0 ** -23))  # units of the last place
    z = torch.where((kind == 1)[:, None], near, z)
    z = torch.where((kind == 2)[:, None], base.expand(T, E), z)                    # all equal
    z = torch.where((kind == 3)[:, None] & (torch.rand(T, E, generator=gen, device="cuda") < 0.1), 40.0, z)  # saturated
    first = torch.zeros(T, E, device="cuda")
    first[:, :16] = 6.0
    z = torch.where((kind == 4)[:, None], z + first, z)                            # neighbours
    first.zero_()
    first[:, ::16] = 6.0
    z = torch.where((kind == 5)[:, None], z + first, z)                            # 16 apart
    z = torch.where((kind == 6)[:, None], 30 * z, z)                               # past 16 below the largest
    z = torch.where((kind == 7)[:, None] & (torch.arange(E, device="cuda") > 1), -float("inf"), z)  # two within reach
    z = torch.where((kind == 8)[:, None], torch.round(4 * z) / 4, z)               # many equal ones
    for bias in (None, b, torch.where(torch.rand(1, E, generator=gen, device="cuda") < 0.2, -float("inf"), 3 * b), 40 * b):
        _, _, _, idx, w, counts, _ = run(L, T, E, k, z, bias, sigmoid, G, top, best)
        want = exact_by_sorting(L, z, bias, k, sigmoid, G, top, best)
        bad = (idx != want).any(1)
        assert not bad.any(), (int(bad.sum()), sorted(set(kind[bad].tolist())), idx[bad][:2].tolist(), want[bad][:2].tolist())
        assert torch.equal(torch.bincount(idx.flatten().long(), minlength=E), counts[0].long())


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("E,k,G,top,best", [(256, 8, 8, 4, 2), (64, 6, 1, 1, 1), (32, 2, 4, 2, 2)])
def test_picks_under_large_biases_and_logits(L, E, k, G, top, best, sigmoid):
    """Keys whose own spacing is coarser than the networks' units: a bias of 5 to 3000 (scores rounded to 5e-7 to 2e-4 in the
    sum, many equal), logits of thousands (sums of two rounded again): exact picks all the same."""
    T = 4001
    gen = torch.Generator(device="cuda").manual_seed(E + k)
    z = torch.randn(T, E, generator=gen, device="cuda")
    for size in (5.0, 9.0, 40.0, 3000.0):
        for sign in (1, -1):
            b = sign * size + 0.01 * torch.randn(1, E, generator=gen, device="cuda")
            zz = z if sigmoid else (z * size * 0.3 + sign * size)
            _, _, _, idx, _, _, _ = run(L, T, E, k, zz, b, sigmoid, G, top, best)
            want = exact_by_sorting(L, zz, b, k, sigmoid, G, top, best)
            assert torch.equal(idx, want), (size, sign, int((idx != want).any(1).sum()))


@pytest.mark.parametrize("T", [1, 7, 8, 9, 31, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513])
@pytest.mark.parametrize("E,k,P", [(256, 8, 1), (256, 8, 4), (64, 6, 2), (16, 2, 64), (20, 3, 3), (250, 4, 5)])
def test_counts_of_every_batch_size(L, T, E, k, P):
    """One CTA or several, one party or several: the counts of each party, over buffers that held something else."""
    gen = torch.Generator(device="cuda").manual_seed(T * 7 + E + P)
    z, b = torch.randn(T, E, generator=gen, device="cuda"), 0.1 * torch.randn(P, E, generator=gen, device="cuda")
    cut = sorted([0, T] + [int(v) for v in torch.randint(0, T + 1, (P - 1,), generator=torch.Generator().manual_seed(T))])
    _, _, _, idx, w, counts, _ = run(L, T, E, k, z, b, True, normalize=1, po=cut if P > 1 else None)
    rows = torch.cat([torch.full((cut[p + 1] - cut[p],), p, device="cuda") for p in range(P)]).long()
    key = 1.0 / (1.0 + torch.exp(-z)) + b[rows]
    want = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :k].int()
    assert torch.equal(idx, want)
    n = torch.zeros(P * E, dtype=torch.int64, device="cuda").index_add_(0, (rows[:, None] * E + idx).flatten(), torch.ones(T * k, dtype=torch.int64, device="cuda"))
    assert torch.equal(counts.flatten().long(), n)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("scale", [1.0, 2.5])
def test_one_renormalised_pick_has_no_gradient(L, sigmoid, scale):
    """k = 1: the weight is the scale whatever the score, so its gradient is exactly 0."""
    T, E = 3000, 40
    gen = torch.Generator(device="cuda").manual_seed(5)
    z, g = torch.randn(T, E, generator=gen, device="cuda"), torch.randn(T, 1, generator=gen, device="cuda")
    cfg, r, _, idx, w, _, _ = run(L, T, E, 1, z, None, sigmoid, normalize=1, scale=scale)
    dz = torch.full_like(z, 7.0)
    L.moe_gate_bwd(cfg, r, z, idx, g, None, None, dz)
    assert status(L) == 0 and float((w - scale).abs().max()) <= scale * 2.0**-22 and float(dz.abs().max()) == 0


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("normalize", [0, 1])
@pytest.mark.parametrize("E,k", [(24, 4), (25, 8), (40, 3), (250, 8), (256, 2), (8, 8)])
def test_equal_picks_add_up(L, sigmoid, normalize, E, k):
    """Picks that a caller brings may name an expert several times: its logit's gradient is that of their sum, and so are the
    router's products. k equal picks add k terms of the bound of one; the products' operands are rounded to bf16."""
    T, d, scale = 333, 128, 1.5
    gen = torch.Generator(device="cuda").manual_seed(E + k)
    z, g = torch.randn(T, E, generator=gen, device="cuda"), torch.randn(T, k, generator=gen, device="cuda")
    z[torch.rand(T, E, generator=gen, device="cuda") < 0.1] = -float("inf")
    aux = 0.1 * torch.rand(1, E, generator=gen, device="cuda")
    idx = torch.randint(0, E, (T, k), generator=gen, device="cuda", dtype=torch.int32)
    idx[::2] = idx[::2] % 3  # few experts, so that most of these picks are equal ones
    idx[::5] = idx[::5, :1]  # all of a token
    cfg = L.make_config(T, d, E, 128, k, normalize_topk=normalize)
    r = rule(L, sigmoid, 1, 1, 1, scale)
    dz = torch.full((T, E), 9.0, device="cuda")
    L.moe_gate_bwd(cfg, r, z, idx, g, aux, None, dz)
    assert status(L) == 0
    zh, gh, ah, ih, dzh = (t.double().cpu().numpy() for t in (z, g, aux[0], idx, dz))
    for t in range(T):
        I = ih[t].astype(int)
        zt, s = scores(zh[t], sigmoid)
        S = s[I].sum() if normalize else 1.0
        add = scale * gh[t]
        if normalize:
            w = scale * s[I] / S if S > 0 else np.zeros(k)
            add = (add - (gh[t] * w).sum()) / S if S > 0 else np.zeros(k)
        ds = ah.copy()
        np.add.at(ds, I, add)
        with np.errstate(all="ignore"):
            ref = ds * s / (1 + np.exp(zt)) if sigmoid else s * (ds - (ds * s).sum())
        size = scale * np.abs(gh[t]).max() * (2 / S if normalize and S > 0 else 1) + np.abs(ah).max()
        assert (np.abs(dzh[t] - ref) <= 256 * k * U * size).all(), (t, I, np.abs(dzh[t] - ref).max(), size)
    x, wr = torch.randn(T, d, generator=gen, device="cuda").bfloat16(), torch.randn(1, E, d, generator=gen, device="cuda").bfloat16()
    ws = torch.empty(L.moe_workspace_size(cfg), dtype=torch.uint8, device="cuda")
    dz2, dw, db, dx = torch.empty_like(dz), torch.empty_like(wr), torch.empty(1, E, device="cuda"), torch.empty_like(x)
    L.moe_gate_bwd(cfg, r, z, idx, g, aux, None, dz2, x, wr, dw, db, dx, ws, ws.numel())
    assert status(L) == 0 and torch.equal(dz2, dz)
    D, X, W = dz.double(), x.double(), wr[0].double()
    assert ((dw[0].double() - D.T @ X).abs() <= 2.0 ** -7 * (D.abs().T @ X.abs())).all()
    assert ((dx.double() - D @ W).abs() <= 2.0 ** -7 * (D.abs() @ W.abs())).all()
    assert ((db[0].double() - D.sum(0)).abs() <= 1e-5 * D.abs().sum(0) + 1e-9).all()
