"""Layer norm (moe_layer_norm_fwd, _bwd) against 64-bit arithmetic on the same inputs.

Bounds. u = 2^-24. A sum of a row runs through at most 16 * 4 additions of a thread, 5 of a warp
and 32 of the warps, so a row's mean is off by at most 101 u mean|h|, its variance by about as much of
itself; y = (h - mean) rstd gamma + beta is then off by 256 u (|gamma| max|h| rstd + |beta|) at most,
and by half a spacing of bf16 (at most 2^-8 relative) after rounding. The backward's two row sums carry
the same 101 u, so dx is within 512 u rstd max|g| (1 + max|xh|^2). dgamma and dbeta add at most 128
terms in a row on any path (33 rows of a CTA at these sizes, 38 partials of a slice, 16 slices), with terms off by
256 u: within 512 u sum|dy xh| (sum|dy|)."""
import pytest
import torch

from tests.gpu_util import need_gpu, status

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def L():
    return need_gpu()


def dtype_of(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def rounding(name):
    return 2.0 ** -8 if name == "bf16" else 0.0


def case(R, d, name, seed, residual=True, loud=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = dtype_of(name)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")

    x = normal(R, d) + 0.5
    if loud and d > 2:
        x[:, d // 2] *= 40.0
    return {"x": x.to(dt), "r": normal(R, d).to(dt) if residual else None, "gamma": 1 + 0.2 * normal(d), "beta": 0.2 * normal(d),
            "dy": normal(R, d).to(dt), "dh": normal(R, d).to(dt)}


def forward(L, c, R, d, name, stats=True, ckpt=False, beta=True):
    dt, dev = dtype_of(name), "cuda"
    mt = L.MOE_BF16 if name == "bf16" else L.MOE_F32
    o = {"y": torch.empty(R, d, dtype=dt, device=dev), "h": torch.empty(R, d, dtype=dt, device=dev) if c["r"] is not None else None,
         "mean": torch.empty(R, device=dev) if stats else None, "rstd": torch.empty(R, device=dev) if stats else None,
         "q": torch.empty(R, d, dtype=torch.int8, device=dev) if ckpt else None,
         "scale": torch.empty(R, -(-d // 128), device=dev) if ckpt else None}
    L.moe_layer_norm_fwd(R, d, mt, c["x"], c["r"], c["gamma"], c["beta"] if beta else None, EPS, o["h"], o["y"], o["mean"], o["rstd"],
                         o["q"], o["scale"])
    assert status(L) == 0
    return o


def backward(L, R, d, name, dy, h, q, scale, mean, rstd, gamma, dh, dbeta=True):
    mt, dev = (L.MOE_BF16 if name == "bf16" else L.MOE_F32), "cuda"
    ws = torch.empty(L.moe_layer_norm_workspace_size(R, d), dtype=torch.uint8, device=dev)
    dx, dg = torch.empty(R, d, dtype=dtype_of(name), device=dev), torch.empty(d, device=dev)
    db = torch.empty(d, device=dev) if dbeta else None
    L.moe_layer_norm_bwd(R, d, mt, dy, h, q, scale, mean, rstd, gamma, dh, dx, dg, db, ws, ws.numel())
    assert status(L) == 0
    return dx, dg, db


def within(name, got, ref, bound):
    bad = (got.double() - ref).abs() > bound
    assert not bad.any(), (name, int(bad.sum()), float((got.double() - ref).abs().max()))


# one row to many; widths of every team size and of both access widths, ragged ends among them
SHAPES = [(1, 1), (3, 2), (5, 7), (9, 64), (33, 96), (17, 250), (4, 255), (130, 256), (65, 257), (40, 512), (7, 1000), (12, 1023),
          (64, 1024), (11, 1366), (5, 2048), (3, 2049), (300, 2056), (4, 4096), (3, 4104), (2, 5001), (3, 8192), (2, 8191), (2, 9000),
          (2, 16384), (2, 16383), (1301, 384)]


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", SHAPES)
def test_forward_and_backward(L, R, d, name):
    c = case(R, d, name, 7 * R + d)
    h64 = c["x"].double() + c["r"].double()
    o = forward(L, c, R, d, name, ckpt=True)
    var, mean = torch.var_mean(h64, dim=1, correction=0)
    rstd = 1 / torch.sqrt(var + EPS)
    top = h64.abs().amax(1, keepdim=True)
    # d = 1 and 2: rstd is the largest amplification of the mean's error
    bound = 256 * U * (c["gamma"].double().abs() * top * rstd[:, None] + c["beta"].double().abs())
    ref = (h64 - mean[:, None]) * rstd[:, None] * c["gamma"].double() + c["beta"].double()
    within("y", o["y"], ref, bound + rounding(name) * ref.abs())
    assert torch.equal(o["h"], (c["x"].float() + c["r"].float()).to(o["h"].dtype))
    within("mean", o["mean"], mean, 128 * U * h64.abs().mean(1) + U * mean.abs())
    within("rstd", o["rstd"], rstd, (256 * U * (1 + (top[:, 0] * rstd) ** 2)) * rstd)
    # the checkpoint is that of the stored h
    q, scale = torch.empty_like(o["q"]), torch.empty_like(o["scale"])
    mt = L.MOE_BF16 if name == "bf16" else L.MOE_F32
    L.moe_ckpt_pack(R, d, mt, o["h"], q, scale)
    assert torch.equal(q, o["q"]) and torch.equal(scale, o["scale"])

    held = o["q"].double() * o["scale"].double().repeat_interleave(128, 1)[:, :d]
    for h, kept in ((o["h"], o["h"].double()), (None, held)):
        for dh in (None, c["dh"]):
            dx, dg, db = backward(L, R, d, name, c["dy"], h, None if h is not None else o["q"], None if h is not None else o["scale"],
                                  o["mean"], o["rstd"], c["gamma"], dh, dbeta=dh is not None)
            rs = o["rstd"].double()[:, None]
            dy = c["dy"].double()
            xh = (kept - o["mean"].double()[:, None]) * rs
            g = dy * c["gamma"].double()
            ref = rs * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
            b = 512 * U * rs * g.abs().amax(1, keepdim=True) * (1 + xh.abs().amax(1, keepdim=True) ** 2)
            if dh is not None:
                ref = ref + dh.double()
                b = b + 4 * U * dh.double().abs()
            within("dx", dx, ref, b + rounding(name) * ref.abs())
            size = (dy * xh).abs().sum(0) + dy.abs().sum(0) * (kept.abs().amax() * rs.amax())
            within("dgamma", dg, (dy * xh).sum(0), 512 * U * size)
            if db is not None:
                within("dbeta", db, dy.sum(0), 512 * U * dy.abs().sum(0))


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_many_rows_and_repeats(L, name):
    """More rows than CTAs of the backward, several per team; the same bits on every call."""
    R, d = 5003, 136
    c = case(R, d, name, 3, residual=False)
    o = forward(L, c, R, d, name, beta=False)
    x = c["x"].double()
    ref = torch.nn.functional.layer_norm(x, (d,), c["gamma"].double(), None, EPS)
    within("y", o["y"], ref, 256 * U * (x.abs().amax() * o["rstd"].double()[:, None] * c["gamma"].double().abs()) + rounding(name) * ref.abs())
    a = backward(L, R, d, name, c["dy"], c["x"], None, None, o["mean"], o["rstd"], c["gamma"], None)
    b = backward(L, R, d, name, c["dy"], c["x"], None, None, o["mean"], o["rstd"], c["gamma"], None)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    dy, rs = c["dy"].double(), o["rstd"].double()[:, None]
    xh = (x - o["mean"].double()[:, None]) * rs
    within("dgamma", a[1], (dy * xh).sum(0), 512 * U * ((dy * xh).abs().sum(0) + (dy.abs() * rs * x.abs().amax()).sum(0)))
    within("dbeta", a[2], dy.sum(0), 512 * U * dy.abs().sum(0))


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", [(3001, 333), (6007, 77), (2500, 1003), (1001, 4099), (700, 7001), (9001, 13), (40000, 6)])
def test_many_rows_of_odd_widths(L, R, d, name):
    """Rows that start at every element of a 16-byte span, many per team (bounds as above; a column's sum runs through
    R / 152 rows of a CTA at most, 10 partials of a slice and 16 slices: below 512 additions)."""
    c = case(R, d, name, R)
    h64 = c["x"].double() + c["r"].double()
    o = forward(L, c, R, d, name, ckpt=True)
    var, mean = torch.var_mean(h64, dim=1, correction=0, keepdim=True)
    rstd = 1 / torch.sqrt(var + EPS)
    ref = (h64 - mean) * rstd * c["gamma"].double() + c["beta"].double()
    top = h64.abs().amax(1, keepdim=True)
    within("y", o["y"], ref, 256 * U * (c["gamma"].double().abs() * top * rstd + c["beta"].double().abs()) + rounding(name) * ref.abs())
    held = o["q"].double() * o["scale"].double().repeat_interleave(128, 1)[:, :d]
    rs, dy = o["rstd"].double()[:, None], c["dy"].double()
    for h, kept in ((o["h"], o["h"].double()), (None, held)):
        dx, dg, db = backward(L, R, d, name, c["dy"], h, None if h is not None else o["q"], None if h is not None else o["scale"],
                              o["mean"], o["rstd"], c["gamma"], c["dh"])
        xh = (kept - o["mean"].double()[:, None]) * rs
        g = dy * c["gamma"].double()
        ref = c["dh"].double() + rs * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        b = 512 * U * rs * g.abs().amax(1, keepdim=True) * (1 + xh.abs().amax(1, keepdim=True) ** 2) + 4 * U * c["dh"].double().abs()
        within("dx", dx, ref, b + rounding(name) * ref.abs())
        size = (dy * xh).abs().sum(0) + (dy.abs() * rs * kept.abs().amax(1, keepdim=True)).sum(0)
        within("dgamma", dg, (dy * xh).sum(0), 1024 * U * size)
        within("dbeta", db, dy.sum(0), 1024 * U * dy.abs().sum(0))


@pytest.mark.parametrize("off", [1, 2, 4])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_unaligned_buffers_equal_aligned_sizes(L, name, off):
    """Buffers that start `off` elements past a 16-byte boundary, and rows of an odd width behind them."""
    for R, d in ((6, 512), (5, 333)):
        c = case(R, d, name, off + d, residual=False)
        whole = torch.zeros(R * d + off, dtype=dtype_of(name), device="cuda")
        shifted = whole[off:].view(R, d)
        shifted.copy_(c["x"])
        a, b = forward(L, c, R, d, name, ckpt=True), forward(L, {**c, "x": shifted}, R, d, name, ckpt=True)
        assert torch.equal(a["q"], b["q"]) and torch.equal(a["scale"], b["scale"])
        tol = 512 * U * float(c["x"].float().abs().max() * a["rstd"].max() * c["gamma"].abs().max() + 1)
        within("y", b["y"], a["y"].double(), tol + 2 * rounding(name) * a["y"].double().abs())
        ga = backward(L, R, d, name, c["dy"], c["x"], None, None, a["mean"], a["rstd"], c["gamma"], c["dh"])
        gb = backward(L, R, d, name, c["dy"], shifted, None, None, a["mean"], a["rstd"], c["gamma"], c["dh"])
        xh = float((c["x"].float().abs().max() + 1) * a["rstd"].max())
        within("dx", gb[0], ga[0].double(), 1024 * U * float(a["rstd"].max()) * float((c["dy"].float() * c["gamma"]).abs().max()) * (1 + xh * xh)
               + 2 * rounding(name) * ga[0].double().abs() + 8 * U * c["dh"].double().abs())
        assert whole[:off].abs().max() == 0


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_rows_that_are_not_finite_stay_alone(L, name):
    """An infinity or a NaN spoils its own row only (and the weights' gradients), a constant row gives beta."""
    R, d = 6, 264
    c = case(R, d, name, 5, residual=False)
    c["x"][1, 3], c["x"][2, 200], c["x"][4] = float("inf"), float("nan"), 7.0
    o = forward(L, c, R, d, name)
    fine = [0, 3, 5]
    assert torch.isfinite(o["y"][fine].float()).all() and torch.isnan(o["y"][[1, 2]].float()).any(1).all()
    assert torch.equal(o["y"][4], c["beta"].to(o["y"].dtype))
    dx, dg, _ = backward(L, R, d, name, c["dy"], c["x"], None, None, o["mean"], o["rstd"], c["gamma"], None)
    assert torch.isfinite(dx[fine + [4]].float()).all() and not torch.isfinite(dg).all()


def test_gradients_against_differences(L):
    """dx, dgamma and dbeta against central differences of the 64-bit forward. With a step of 2^-12 the
    difference's own error is (2^-24 / 6) times a third derivative below 64 at these inputs, and the
    fp32 kernel's 512 u of the largest term is below that."""
    R, d, step = 3, 24, 2.0 ** -12
    c = case(R, d, "f32", 11, residual=False, loud=False)
    o = forward(L, c, R, d, "f32")
    dx, dg, db = backward(L, R, d, "f32", c["dy"], c["x"], None, None, o["mean"], o["rstd"], c["gamma"], None)
    dy = c["dy"].double()

    def loss(x, gamma, beta):
        return (torch.nn.functional.layer_norm(x, (d,), gamma, beta, EPS) * dy).sum()

    args = [c["x"].double(), c["gamma"].double(), c["beta"].double()]
    for i, got in enumerate((dx, dg, db)):
        flat = args[i].view(-1)
        for j in range(flat.numel()):
            keep = flat[j].item()
            flat[j] = keep + step
            up = loss(*args)
            flat[j] = keep - step
            down = loss(*args)
            flat[j] = keep
            assert abs(float(up - down) / (2 * step) - float(got.view(-1)[j])) < 1e-4, (i, j)


def test_no_rows(L):
    d = 200
    dg, db = torch.full((d,), 3.0, device="cuda"), torch.full((d,), 3.0, device="cuda")
    L.moe_layer_norm_fwd(0, d, L.MOE_F32, None, None, None, None, EPS, None, None)
    L.moe_layer_norm_bwd(0, d, L.MOE_F32, None, None, None, None, None, None, None, None, None, dg, db, None, 0)
    assert status(L) == 0 and dg.abs().max() == 0 and db.abs().max() == 0


def test_other_stream(L):
    """The calls run on the stream they are given, in its order."""
    R, d = 2000, 1024
    c = case(R, d, "bf16", 2, residual=False)
    s = torch.cuda.Stream()
    y, x = torch.zeros(R, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(R, d, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            x.zero_()
        x.copy_(c["x"])
    L.moe_layer_norm_fwd(R, d, L.MOE_BF16, x, None, c["gamma"], c["beta"], EPS, None, y, stream=s)
    s.synchronize()
    assert torch.equal(y, forward(L, c, R, d, "bf16", stats=False)["y"])


def test_more_than_2_31_elements(L):
    """Offsets past 32 bits, forward and backward: the first and last rows are those of a small call."""
    R, d = 523_907, 4104
    assert R * d > 1 << 31
    n = 8
    c = case(n, d, "bf16", 6, residual=False)
    x = torch.zeros(R, d, dtype=torch.bfloat16, device="cuda")
    x[:n], x[-n:] = c["x"], c["x"]
    y, mean, rstd = torch.empty_like(x), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    L.moe_layer_norm_fwd(R, d, L.MOE_BF16, x, None, c["gamma"], c["beta"], EPS, None, y, mean, rstd)
    o = forward(L, c, n, d, "bf16")
    for part in (slice(0, n), slice(R - n, R)):
        assert torch.equal(y[part], o["y"]) and torch.equal(mean[part], o["mean"]) and torch.equal(rstd[part], o["rstd"])
    assert torch.equal(y[n:n + 1], c["beta"].bfloat16()[None]) and torch.equal(y[n], y[R - n - 1])
    y.zero_()
    y[:n], y[-n:] = c["dy"], c["dy"]
    ws = torch.empty(L.moe_layer_norm_workspace_size(R, d), dtype=torch.uint8, device="cuda")
    dg, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    L.moe_layer_norm_bwd(R, d, L.MOE_BF16, y, x, None, None, mean, rstd, c["gamma"], None, y, dg, db, ws, ws.numel())  # in place
    dx, dg1, db1 = backward(L, n, d, "bf16", c["dy"], c["x"], None, None, o["mean"], o["rstd"], c["gamma"], None)
    assert torch.equal(y[:n], dx) and torch.equal(y[-n:], dx) and float(y[n:-n].abs().max()) == 0
    # each row counts twice; the sums run in another order
    assert ((dg - 2 * dg1).abs() <= 64 * U * 2 * c["dy"].float().abs().sum(0) * 64).all()
    assert ((db - 2 * db1).abs() <= 64 * U * 2 * c["dy"].float().abs().sum(0)).all()
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", [(700, 512), (601, 333)])
def test_in_place(L, R, d, name):
    """h over x, y over the residual, dx over dh and over dy give what separate buffers give."""
    c = case(R, d, name, 12)
    o = forward(L, c, R, d, name)
    mt = L.MOE_BF16 if name == "bf16" else L.MOE_F32
    x, r = c["x"].clone(), c["r"].clone()
    L.moe_layer_norm_fwd(R, d, mt, x, r, c["gamma"], c["beta"], EPS, x, r, o["mean"].clone(), o["rstd"].clone())
    assert torch.equal(x, o["h"]) and torch.equal(r, o["y"])
    dx, dg, db = backward(L, R, d, name, c["dy"], o["h"], None, None, o["mean"], o["rstd"], c["gamma"], c["dh"])
    ws = torch.empty(L.moe_layer_norm_workspace_size(R, d), dtype=torch.uint8, device="cuda")
    for over in ("dh", "dy"):
        b = {m: c[m].clone() for m in ("dh", "dy")}
        g, e = torch.empty_like(dg), torch.empty_like(db)
        L.moe_layer_norm_bwd(R, d, mt, b["dy"], o["h"], None, None, o["mean"], o["rstd"], c["gamma"], b["dh"], b[over], g, e, ws, ws.numel())
        assert status(L) == 0 and torch.equal(b[over], dx) and torch.equal(g, dg) and torch.equal(e, db)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("R,d", [(700, 512), (601, 333), (60, 130), (2, 16383)])
@pytest.mark.parametrize("off", ["", "x", "q"])
def test_checkpoint_of_x_when_y_lies_over_it(L, R, d, name, off):
    """Without a residual the stored h is x: its checkpoint and y are the same bits whether y is another buffer or x's own,
    at widths of whole 16-byte spans and others, with x or h_q off their alignment or not."""
    c = case(R, d, name, 5 * R + d, residual=False)
    mt = L.MOE_BF16 if name == "bf16" else L.MOE_F32
    q, scale = torch.empty(R, d, dtype=torch.int8, device="cuda"), torch.empty(R, -(-d // 128), device="cuda")
    L.moe_ckpt_pack(R, d, mt, c["x"], q, scale)

    def shifted(dt, by):
        return torch.zeros(R * d + by, dtype=dt, device="cuda")[by:].view(R, d)

    got = []
    for over in (False, True):
        x = shifted(dtype_of(name), 1 if off == "x" else 0)
        x.copy_(c["x"])
        y = x if over else torch.empty_like(c["x"])
        qq, ss = shifted(torch.int8, 1 if off == "q" else 0), torch.zeros_like(scale)
        mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
        L.moe_layer_norm_fwd(R, d, mt, x, None, c["gamma"], c["beta"], EPS, None, y, mean, rstd, qq, ss)
        assert status(L) == 0 and torch.equal(qq, q) and torch.equal(ss, scale), over
        got.append((y, mean, rstd))
    assert all(torch.equal(a, b) for a, b in zip(*got))
