"""The cross entropy over a vocabulary and its gradients against a plain form in 64 bits.

Tolerances, from the arithmetic, element by element. Logits: fp32 accumulators that may truncate, one step of 2^-23 of the
terms' magnitudes per 16 of them and a few for what follows: tau = (d / 16 + 8) 2^-23 sum |h w|, the largest of a row. lse is
off by tau, its sum's and its functions' roundings (2^-18 of 1 bounds a sum of 2^18 terms whose parts are
joined pairwise or by shares of at most 512, and the exponentials' 2^-20); a token's loss by twice tau and those.
dz = u (p - onehot): half a step of the storage type, and p's own error (2 tau and the same 2^-18; in bf16
also fp16's half step 2^-11, and 2^-25 of the row's largest p). The gradients: those of dz through the product, the
product's own (K / 16 + 80) 2^-23 of the terms' magnitudes (80: splits, pieces), half a step of the result.
"""
import pytest
import torch

from paper_2506_02965_gb300 import _lib as L

pytestmark = pytest.mark.gpu
DT = {"f32": (L.MOE_F32, torch.float32), "bf16": (L.MOE_BF16, torch.bfloat16)}


def make(T, d, V, kind, seed, peaked=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[kind][1]
    w = (torch.randn(V, d, generator=g, device="cuda") * 0.05).to(dt)
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    lean = (torch.rand(T, 1, generator=g, device="cuda") < 0.5).float() * (8 / (0.05 * d ** 0.5) if peaked else 0.0)
    h = (torch.randn(T, d, generator=g, device="cuda") + lean * w[y.long()].float()).to(dt)
    return h, w, y, torch.rand(T, generator=g, device="cuda")


class Result:
    pass


def run(h, w, y, weight, kind, grads=True, token=True, stream=None, ws=None):
    (T, d), V, dt = h.shape, w.shape[0], DT[kind][1]
    r = Result()
    r.loss = torch.full((1,), float("nan"), device="cuda")
    r.token = torch.full((T,), float("nan"), device="cuda") if token else None
    r.dh = torch.full((T, d), float("nan"), dtype=dt, device="cuda") if grads else None
    r.dw = torch.full((V, d), float("nan"), dtype=dt, device="cuda") if grads else None
    if ws is None:
        ws = torch.full((L.moe_vocab_loss_workspace_size(T, d, V, DT[kind][0], grads),), 255, dtype=torch.uint8, device="cuda")
    L.moe_vocab_loss(T, d, V, DT[kind][0], h, w, y, weight, r.loss, r.token, r.dh, r.dw, ws, ws.numel(), stream=stream)
    return r


def check(r, h, w, y, weight, kind):
    (T, d), V, dt = h.shape, w.shape[0], DT[kind][1]
    half, f64 = torch.finfo(dt).eps / 2, torch.float64
    live = (y >= 0) & (y < V)
    h64, w64 = torch.where(live[:, None], h.double(), 0.0), w.double()
    at = y.long().clamp(0, V - 1)
    z = h64 @ w64.T
    tau = (d / 16 + 8) * 2.0 ** -23 * (h64.abs() @ w64.abs().T).amax(1)
    lse = torch.logsumexp(z, 1)
    token = torch.where(live, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    u = weight.double() if weight is not None else torch.full((T,), 1.0 / max(int(live.sum()), 1), dtype=f64, device="cuda")
    u = torch.where(live, u, 0.0)
    off = torch.where(live, 2 * tau + 2.0 ** -18 + 2.0 ** -23 * (lse.abs() + z.abs().amax(1)), 0.0)
    if r.token is not None:
        assert ((r.token.double() - token).abs() <= off).all(), ((r.token.double() - token).abs() - off).max()
    bound = (u.abs() * (off + 2.0 ** -23 * token.abs())).sum() + 2.0 ** -23 * (u * token).sum().abs()
    assert (r.loss.double() - (u * token).sum()).abs() <= bound
    if r.dh is None:
        return
    p = torch.exp(z - lse[:, None])
    one = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    dz = u[:, None] * (p - one)
    edz = p * (2 * tau[:, None] + 2.0 ** -18) + half * (p - one).abs()
    if kind == "bf16":
        edz = edz + 2.0 ** -11 * p + 2.0 ** -25 * p.amax(1, keepdim=True)
    else:
        edz = edz + 2.0 ** -22
    edz = u.abs()[:, None] * edz * (1 + 2.0 ** -7)
    for got, a, ea, b in ((r.dh, dz, edz, w64), (r.dw, dz.T, edz.T, h64)):
        ref = a @ b
        lim = ea @ b.abs() + (a.shape[1] / 16 + 80) * 2.0 ** -23 * (a.abs() @ b.abs()) + half * ref.abs() * 1.01 + 1e-38
        err = (got.double() - ref).abs()
        assert torch.isfinite(got).all() and (err <= lim).all(), (err / lim).max()


SIZES = [(1, 128, 1), (1, 128, 2), (2, 256, 100), (7, 128, 65), (64, 128, 5003), (128, 256, 256), (129, 128, 257), (300, 384, 1000),
         (257, 1152, 511), (1003, 1152, 5003), (2100, 1024, 130), (33, 2048, 9000)]


@pytest.mark.parametrize("T,d,V", SIZES)
@pytest.mark.parametrize("weighted", [False, True])
def test_bf16(T, d, V, weighted):
    h, w, y, u = make(T, d, V, "bf16", T + V)
    if weighted:
        y[1::4] = -1 - y[1::4]
        u[2::4] = 0.0
        u[3::4] *= -3.0
    r = run(h, w, y, u if weighted else None, "bf16")
    check(r, h, w, y, u if weighted else None, "bf16")
    again = run(h, w, y, u if weighted else None, "bf16")
    for a, b in ((r.loss, again.loss), (r.token, again.token), (r.dh, again.dh), (r.dw, again.dw)):
        assert torch.equal(a, b)
    f = run(h, w, y, u if weighted else None, "bf16", grads=False)
    check(f, h, w, y, u if weighted else None, "bf16")
    assert L.moe_device_status() == 0


@pytest.mark.parametrize("T,d,V", [(1, 4, 1), (3, 64, 7), (129, 20, 1000), (501, 256, 5003), (64, 1000, 513), (300, 132, 12000)])
@pytest.mark.parametrize("weighted", [False, True])
def test_f32(T, d, V, weighted):
    h, w, y, u = make(T, d, V, "f32", T + V)
    if weighted:
        y[1::4] = -1 - y[1::4]
        u[2::4] = 0.0
    r = run(h, w, y, u if weighted else None, "f32")
    check(r, h, w, y, u if weighted else None, "f32")
    check(run(h, w, y, u if weighted else None, "f32", grads=False), h, w, y, u if weighted else None, "f32")
    assert torch.equal(r.dw, run(h, w, y, u if weighted else None, "f32").dw) and L.moe_device_status() == 0


@pytest.mark.parametrize("kind,T,d,V", [("bf16", 4097, 128, 300), ("bf16", 9000, 128, 301), ("bf16", 12289, 256, 77),
                                        ("bf16", 4100, 128, 70001), ("bf16", 8300, 128, 70001), ("f32", 1100, 16, 262144)])
def test_pieces_of_the_batch(kind, T, d, V):
    h, w, y, u = make(T, d, V, kind, 5)
    y[::3] = -1
    check(run(h, w, y, u, kind), h, w, y, u, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_large_vocabulary_few_tokens(kind):
    h, w, y, _ = make(5, 128, 100003, kind, 9)
    y[0], y[1] = 0, 100002
    check(run(h, w, y, None, kind), h, w, y, None, kind)


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_no_token_has_a_target(kind):
    h, w, _, u = make(70, 128, 300, kind, 1)
    y = torch.full((70,), -100, dtype=torch.int32, device="cuda")
    for weight in (None, u):
        r = run(h, w, y, weight, kind)
        assert r.loss.item() == 0 and not r.token.any() and not r.dh.any() and not r.dw.any()
    r = run(h, w, torch.zeros_like(y), torch.zeros_like(u), kind)  # targets that weigh nothing
    assert r.loss.item() == 0 and not r.dh.any() and not r.dw.any() and (r.token > 0).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_states_of_masked_tokens_do_not_count(kind, bad):
    h, w, y, u = make(300, 128, 500, kind, 2)
    y[10:40] = -1
    h[10:40:3] = bad
    u[10:40] = float("nan")
    r = run(h, w, y, u, kind)
    check(r, torch.where(torch.isfinite(h), h, 0.0), w, y, torch.where(torch.isnan(u), 0.0, u), kind)


def test_a_bad_state_stays_in_its_row():
    h, w, y, _ = make(200, 128, 500, "bf16", 3)
    h[17, 5] = float("nan")
    r = run(h, w, y, None, "bf16")
    ok = torch.arange(200, device="cuda") != 17
    assert torch.isnan(r.token[17]) and torch.isfinite(r.token[ok]).all() and torch.isfinite(r.dh[ok]).all() and torch.isnan(r.dh[17]).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_peaked_and_flat_rows(kind):
    """Logits of +-300 (probabilities that underflow), and all alike."""
    h, w, y, _ = make(128, 128, 777, kind, 4)
    h = (h.float() * 40).to(h.dtype)
    h[::4] = 0
    check(run(h, w, y, None, kind), h, w, y, None, kind)


@pytest.mark.parametrize("size", [1e-42, 1e-36, 1e34])
@pytest.mark.parametrize("T", [20, 300])
def test_weights_of_any_size(size, T):
    h, w, y, u = make(T, 128, 300, "bf16", 13)
    y[::5] = -1
    u = u * size
    r = run(h, w, y, u, "bf16")
    if size > 1:
        check(r, h, w, y, u, "bf16")
    else:  # below bf16's normal numbers a step is 2^-133 (and 2^-149 in fp32): next to that, the sums of as many terms
        live = (y >= 0).double()
        p = torch.softmax(h.double() @ w.double().T, 1)
        dz = (u.double() * live)[:, None] * (p - torch.zeros_like(p).scatter_(1, y.long().clamp(min=0)[:, None], 1.0))
        for got, ref, n in ((r.dh, dz @ w.double(), 300), (r.dw, dz.T @ h.double(), T)):
            mag = 2.0 ** -133 * n * 40 + ref.abs().max() * 2.0 ** -6
            assert torch.isfinite(got).all() and ((got.double() - ref).abs() <= mag).all()


@pytest.mark.slow
def test_a_last_piece_of_one_token():
    """Pieces of 4096 tokens and one of a single token, with gradients."""
    T, d, V = 17 * 4096 + 1, 128, 65600
    h, w, y, _ = make(T, d, V, "bf16", 15)
    r = run(h, w, y, None, "bf16")
    z = h[-1].double() @ w.double().T
    lse = torch.logsumexp(z, 0)
    assert abs(r.token[-1].item() - (lse - z[y[-1].long()]).item()) <= 1e-4
    dz = torch.exp(z - lse)
    dz[y[-1].long()] -= 1
    ref = dz @ w.double() / T
    assert (r.dh[-1].double() - ref).norm() <= 1e-2 * ref.norm()
    assert torch.isfinite(r.dw).all() and torch.isfinite(r.dh).all()


def test_targets_out_of_range_are_recorded():
    h, w, y, _ = make(50, 128, 300, "bf16", 6)
    y[7], y[9] = 300, 2 ** 31 - 1
    check(run(h, w, y, None, "bf16"), h, w, y, None, "bf16")
    assert L.moe_device_status() == L.MOE_ERR_DEVICE_CHECK and L.moe_device_status() == 0


def test_no_tokens():
    loss, dw = torch.ones(1, device="cuda"), torch.ones(20, 128, dtype=torch.bfloat16, device="cuda")
    L.moe_vocab_loss(0, 128, 20, L.MOE_BF16, None, None, None, None, loss, None, None, dw, None, 0)
    assert loss.item() == 0 and not dw.any()


def test_without_the_tokens_losses():
    h, w, y, _ = make(100, 128, 300, "bf16", 7)
    a, b = run(h, w, y, None, "bf16"), run(h, w, y, None, "bf16", token=False)
    assert torch.equal(a.loss, b.loss) and torch.equal(a.dw, b.dw)


def test_gradients_against_differences():
    """The loss along a direction of h and of w, central differences of the call's own losses in fp32."""
    h, w, y, u = make(40, 32, 60, "f32", 8, peaked=False)
    y[::7] = -1
    r = run(h, w, y, u, "f32")
    g = torch.Generator(device="cuda").manual_seed(1)
    for x, grad, other in ((h, r.dh, lambda t: run(t, w, y, u, "f32", grads=False)), (w, r.dw, lambda t: run(h, t, y, u, "f32", grads=False))):
        v = torch.randn(x.shape, generator=g, device="cuda")
        step = 1e-2
        hi, lo = other(x + step * v), other(x - step * v)
        num = (u.double() * (hi.token.double() - lo.token.double())).sum() / (2 * step)
        ana = (grad.double() * v.double()).sum()
        # third derivatives of lse are at most |z'|^3, here z' = <v, w> or <h, v> of about 0.3 and 6, weights of 0.5 in sum 20;
        # rounding: 40 tokens' 2^-20 over the step
        size = (v.double().norm(dim=1).max() * (w if x is h else h).double().norm(dim=1).max()) ** 3
        assert (num - ana).abs() <= step ** 2 / 6 * size * u.sum() + 40 * 2.0 ** -20 / step


def test_stream_graph_and_shared_workspace():
    T, d, V = 600, 256, 3000
    h, w, y, u = make(T, d, V, "bf16", 11)
    ws = torch.empty(L.moe_vocab_loss_workspace_size(T, d, V, L.MOE_BF16, True), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        r = run(h, w, y, u, "bf16", ws=ws)
    s.synchronize()
    check(r, h, w, y, u, "bf16")
    h2, w2, y2, u2 = make(T, d, V, "bf16", 12)
    graphs, results = [], []
    for args in ((h, w, y, u), (h2, w2, y2, None)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(run(*args, "bf16", ws=ws))
        graphs.append(g)
    for r in results:
        r.dw.zero_(), r.dh.zero_()
    for g in graphs + graphs[::-1]:  # one after the other on one workspace
        g.replay()
    torch.cuda.synchronize()
    check(results[0], h, w, y, u, "bf16")
    check(results[1], h2, w2, y2, None, "bf16")


@pytest.mark.slow
def test_offsets_past_32_bits():
    """More than 2^31 elements of W, and of the stored probabilities."""
    T, d, V = 300, 128, 17_000_000
    w = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    w[-3:, 0] = torch.tensor([1.0, 2.0, 3.0], device="cuda")
    h = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 8.0
    y = torch.full((T,), V - 1, dtype=torch.int32, device="cuda")
    r = run(h, w, y, None, "bf16")
    e = torch.exp(torch.tensor([0.0, 8.0, 16.0, 24.0], dtype=torch.float64))
    total = (V - 3) * e[0] + e[1] + e[2] + e[3]
    assert abs(r.token[-1].item() - (torch.log(total) - 24).item()) < 1e-4
    p = (e / total).cuda()
    assert (r.dw[-2, 0].double() - p[2] * 8).abs() <= p[2] * 8 * 2.0 ** -7
    assert (r.dw[-1, 0].double() - (p[3] - 1) * 8).abs() <= (1 - p[3]) * 8 * 2.0 ** -7 + 2.0 ** -17
    assert (r.dh[:, 0].double() - (p[1] + 2 * p[2] + 3 * (p[3] - 1)) / T).abs().max() <= 2.0 ** -7 / T
