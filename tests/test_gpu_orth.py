"""Orthogonalised updates against a plain form in 64 bits.

Tolerances. The steps amplify what is rounded in small singular directions by up to 3.4445^5, so a bound for the worst case
says little; what the roundings make is what the same roundings make elsewhere: the plain form is run once more in fp32 with
X, A and b A + c A A + t I rounded to fp16 where the kernels round them (X's residual to 3 bits more), and the kernels may be off
64 bits by 1.3 times what that is off, in the norm, and in any element by 14 times its root mean square (a
normal variable passes 7 once in 10^11; rows differ in scale by less than 2) - plus half a step of the storage type.
fp32 matrices: the same with plain fp32 products, and twice their error (another order of the sums).
"""
import pytest
import torch

from paper_2506_02965_gb300 import _lib as L

pytestmark = pytest.mark.gpu
DT = {"f32": (L.MOE_F32, torch.float32), "bf16": (L.MOE_BF16, torch.bfloat16)}
COEF = (3.4445, -4.7750, 2.0315)


def make(G, R, C, kind, seed, strong=3.0, size=1e-3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = min(8, R, C)
    x = torch.randn(G, R, C, generator=g, device="cuda")
    x += torch.bmm(torch.randn(G, R, k, generator=g, device="cuda"), torch.randn(G, k, C, generator=g, device="cuda")) * strong / k ** 0.5
    return (x * size).to(DT[kind][1]), torch.randn(G, R, C, generator=g, device="cuda") * 2 * size


def update_of(dw, mom, beta, nesterov):
    g = dw.double()
    if mom is None:
        return g, None
    m = beta * mom.double() + g
    return (g + beta * m if nesterov else m), m


def steps64(u, steps):
    a, b, c = COEF
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2) if tall else u
    n = x.flatten(1).norm(dim=1)[:, None, None]
    x = x / torch.where(n > 0, n, 1.0)
    for _ in range(steps):
        A = x @ x.transpose(1, 2)
        x = a * x + (b * A + c * (A @ A)) @ x
    return x.transpose(1, 2) if tall else x


def steps_rounded(u, steps, kind):
    """fp32, rounded where the kernels round."""
    a, b, c = COEF
    f16 = (lambda t, s: (t * s).half().float() / s) if kind == "bf16" else (lambda t, s: t)
    tall = u.shape[1] > u.shape[2]
    x = (u.transpose(1, 2) if tall else u)
    x = (x / x.flatten(1).norm(dim=1)[:, None, None].clamp(min=1e-300)).float()
    eye = torch.eye(x.shape[1], device="cuda")
    for it in range(steps):
        t = (0.0, 0.0, 1.25, 2.25, 2.5)[min(it, 4)] if kind == "bf16" else 0.0
        h = f16(x, 256.0)
        r = ((x - h) * 256 * 4096).to(torch.float8_e5m2).float() / (256 * 4096) if kind == "bf16" else 0.0
        A = f16(h @ h.transpose(1, 2), 4096.0)
        x = (a - t) * (h + r) + f16(b * A + c * (A @ A) + t * eye, 4096.0) @ h
    return x.transpose(1, 2) if tall else x


def run(dw, mom, beta=0.95, nesterov=1, counts=None, steps=5, scale=1.0, out=None, mom_out=None, ws=None, stream=None):
    G, R, C = dw.shape
    dt = L.MOE_F32 if dw.dtype == torch.float32 else L.MOE_BF16
    out = torch.full_like(dw, 7.0) if out is None else out
    if mom is not None and mom_out is None:
        mom_out = torch.full_like(mom, 7.0)
    if ws is None:
        ws = torch.full((L.moe_orthogonalise_workspace_size(G, R, C, dt),), 255, dtype=torch.uint8, device="cuda")
    L.moe_orthogonalise(G, R, C, dt, dw, mom, beta, nesterov, counts, steps, scale, mom_out, out, ws, ws.numel(), stream=stream)
    return out, mom_out


def check(out, mom_out, dw, mom, kind, beta=0.95, nesterov=1, counts=None, steps=5, scale=1.0):
    called = torch.ones(dw.shape[0], dtype=torch.bool, device="cuda") if counts is None else counts > 0
    u, m = update_of(dw, mom, beta, nesterov)
    if m is not None:
        err = (mom_out[called].double() - m[called]).abs()
        over = (err - 2.0 ** -22 * ((beta * mom[called].double()).abs() + dw[called].double().abs()) - 2.0 ** -149).max().item()
        assert over <= 0
        left = (mom_out[~called] == 7.0).all().item()
        assert left
    left = (out[~called] == 7.0).all().item()
    assert left
    ref, emu = steps64(u, steps) * scale, steps_rounded(u, steps, kind).double() * scale
    half = torch.finfo(DT[kind][1]).eps / 2
    for i in torch.nonzero(called)[:, 0].tolist():
        own = (emu[i] - ref[i])
        floor = 2.0 ** -20 if kind == "f32" else 2.0 ** -12  # of the result: what one element's few roundings come to
        most = 1.3 if kind == "bf16" else 2.0
        rms = own.norm() / own.numel() ** 0.5 + floor * ref[i].norm() / own.numel() ** 0.5
        err = out[i].double() - ref[i]
        assert torch.isfinite(out[i]).all()
        rounding = half * ref[i].norm()
        assert err.norm() <= most * rms * own.numel() ** 0.5 + rounding, (i, (err.norm() / ref[i].norm()).item(), (own.norm() / ref[i].norm()).item())
        assert (err.abs() <= 14 * rms + half * ref[i].abs() * 1.01).all(), (i, (err.abs() / rms).max())


SIZES = [(1, 1, 1), (1, 1, 5), (2, 5, 1), (1, 16, 16), (3, 100, 33), (3, 33, 100), (2, 64, 257), (2, 333, 1000), (2, 1000, 333), (1, 512, 512),
         (5, 257, 255), (2, 300, 700), (1, 130, 2000), (17, 40, 24),
         (3, 44, 6748), (2, 4501, 83), (1, 3000, 130)]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("G,R,C", SIZES)
def test_sizes(kind, G, R, C):
    dw, mom = make(G, R, C, kind, G + R + C)
    scale = max(1.0, R / C) ** 0.5
    out, mo = run(dw, mom, scale=scale)
    check(out, mo, dw, mom, kind, scale=scale)
    again, _ = run(dw, mom, scale=scale)
    assert torch.equal(out, again) and L.moe_device_status() == 0


@pytest.mark.parametrize("G,R,C", [(2, 1024, 2816), (3, 1408, 640), (1, 2048, 2048)])
def test_large(G, R, C):
    dw, mom = make(G, R, C, "bf16", 3)
    out, mo = run(dw, mom)
    check(out, mo, dw, mom, "bf16")


@pytest.mark.parametrize("G,R,C,left", [(26, 300, 4000, 0), (26, 300, 4000, 1), (26, 4001, 301, 20), (13, 520, 4100, 0), (13, 4099, 519, 1), (13, 4099, 520, 12)])
def test_a_last_round_in_parts(G, R, C, left):
    """One tile or a few more than run at once (and, with matrices left out, about as many or a few in all)."""
    dw, mom = make(G, R, C, "bf16", R)
    counts = torch.ones(G, dtype=torch.int32, device="cuda")
    counts[:left] = 0
    out, mo = run(dw, mom, counts=counts)
    check(out, mo, dw, mom, "bf16", counts=counts)
    again, _ = run(dw, mom, counts=counts)
    assert torch.equal(out, again) and L.moe_device_status() == 0


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("nesterov,beta,momentum,steps", [(0, 0.9, True, 5), (1, 0.0, True, 5), (0, 0.5, False, 5), (1, 0.95, True, 1), (1, 0.95, True, 2),
                                                           (1, 0.95, True, 8)])
def test_forms(kind, nesterov, beta, momentum, steps):
    dw, mom = make(3, 96, 200, kind, 4)
    mom = mom if momentum else None
    out, mo = run(dw, mom, beta=beta, nesterov=nesterov, steps=steps, scale=-0.2)
    check(out, mo, dw, mom, kind, beta=beta, nesterov=nesterov, steps=steps, scale=-0.2)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("R,C", [(200, 96), (65, 130)])
def test_matrices_left_out(kind, R, C):
    dw, mom = make(6, R, C, kind, 5)
    counts = torch.tensor([3, 0, 1, -2, 0, 9], dtype=torch.int32, device="cuda")
    dw[1] = float("nan")
    out, mo = run(dw, mom, counts=counts)
    dw[1] = 0
    check(out, mo, dw, mom, kind, counts=counts)
    none = torch.zeros_like(counts)
    out, mo = run(dw, mom, counts=none)
    assert (out == 7).all() and (mo == 7).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_in_place(kind):
    dw, mom = make(2, 120, 72, kind, 6)
    ref, mo = run(dw, mom)
    d2, m2 = dw.clone(), mom.clone()
    run(d2, m2, out=d2, mom_out=m2)
    assert torch.equal(d2, ref) and torch.equal(m2, mo)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e-40, 1e-36, 1e-25, 1e-12, 1e12, 1e25, 1e36, 1.5e37])
def test_range_of_the_gradient(kind, size):
    dw, _ = make(2, 64, 100, kind, 7, size=size)
    out, _ = run(dw, None)
    check(out, None, dw, None, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_zeros_and_bad_values_stay_in_their_matrix(kind):
    dw, mom = make(4, 90, 150, kind, 8)
    dw[0], mom[0] = 0, 0
    dw[2, 5, 7] = float("nan")
    dw[3, 1, 1] = float("inf")
    out, _ = run(dw, mom)
    assert not out[0].any() and torch.isnan(out[2]).all() and torch.isnan(out[3]).all()
    ref, _ = run(dw[1:2].clone(), mom[1:2].clone())
    assert torch.equal(out[1:2], ref)


@pytest.mark.parametrize("strong", [30.0, 100.0])
def test_a_few_directions_that_outweigh_the_rest(strong):
    dw, mom = make(2, 512, 768, "bf16", 9, strong=strong)
    mom = mom * 0
    out, mo = run(dw, mom)
    check(out, mo, dw, mom, "bf16")


def test_rank_one():
    """One direction only: u v^T comes out as s u v^T with s the steps' value at 1."""
    g = torch.Generator(device="cuda").manual_seed(1)
    a, b = torch.randn(300, generator=g, device="cuda"), torch.randn(200, generator=g, device="cuda")
    a, b = a / a.norm(), b / b.norm()
    dw = torch.outer(a, b)[None].contiguous()
    out, _ = run(dw, None)
    s = 1.0
    for _ in range(5):
        s = COEF[0] * s + COEF[1] * s ** 3 + COEF[2] * s ** 5
    assert (out[0] - s * torch.outer(a, b)).norm() <= 1e-4 * abs(s)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_singular_values(kind):
    dw, _ = make(1, 256, 1024, kind, 10, strong=0.0)
    s = torch.linalg.svdvals(run(dw, None)[0][0].double())
    assert s.min() > 0.65 and s.max() < 1.25


def test_stream_and_graphs_on_one_workspace():
    a, b = make(3, 200, 300, "bf16", 11), make(3, 200, 300, "bf16", 12)
    ws = torch.empty(L.moe_orthogonalise_workspace_size(3, 200, 300, L.MOE_BF16), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [run(*a, ws=ws), run(*b, ws=ws)]
    s.synchronize()
    check(*got[0], *a, "bf16")
    check(*got[1], *b, "bf16")
    graphs, results = [], []
    for x in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(run(*x, ws=ws))
        graphs.append(g)
    for g in (graphs[1], graphs[0], graphs[1]):
        g.replay()
    torch.cuda.synchronize()
    for r, e in zip(results, got):
        assert torch.equal(r[0], e[0]) and torch.equal(r[1], e[1])


def test_many_matrices():
    dw, mom = make(256, 24, 40, "bf16", 13)
    out, mo = run(dw, mom)
    check(out[::37], mo[::37], dw[::37], mom[::37], "bf16")
