"""The vocabulary loss of tokens that are sure of their target, whose loss and gradient are far below a step of their logits.

Every logit is h0 - h1 gap_v, products of a few bits whose sum is exact in fp32, so that no error of a product covers for one
of the softmax. Tolerances, from the arithmetic, with r a row's largest logit, s = sum_v exp(z - r) (1 and what the others add),
q = (s - 1) / s: a share's sum is V additions in sequence at most, those of shares 13 more, each half a step 2^-24 of s; the exponentials are
off by 2^-20 of themselves, log by 2^-22 of itself, r - z_y (0 or an exact difference) by none. So the loss is off by
ls = (V + 16) 2^-24 + 2^-20 (s - 1) + 2^-22 l. dz at the target is -q: (s - 1)'s errors again, ls, and 3 roundings of
1 / s, f and the product, 3 2^-24; at the others p to ls + 2^-20 relative; in bf16 also fp16's half step 2^-11 and 2^-25 for p, and bf16's
half step for dz. The products' own terms and the result's rounding as in test_gpu_vocab_loss.
"""
import pytest
import torch

from tests.test_gpu_vocab_loss import DT, check, run
from tests.test_gpu_vocab_loss import make as make_plain

pytestmark = pytest.mark.gpu

BASES = (0.0, 50.0, 100.0, 200.0, 300.0, -100.0, -300.0)


def make(T, d, V, kind):
    """Logits h0 - h1 gap_v: word 1 (0 of a single one) has gap 0, the others 10 to 17.5 in steps of 1/8."""
    dt = DT[kind][1]
    i, v = torch.arange(T, device="cuda"), torch.arange(V, device="cuda")
    h, w = torch.zeros(T, d, device="cuda"), torch.zeros(V, d, device="cuda")
    h[:, 0] = torch.tensor(BASES, device="cuda")[i % len(BASES)]
    h[:, 1] = 1.0 + 0.25 * ((i // len(BASES)) % 2)
    w[:, 0] = 1.0
    w[:, 1] = -(10.0 + (v * 7 % 61) / 8.0)
    top = min(1, V - 1)
    w[top, 1] = 0.0
    y = torch.full((T,), top, dtype=torch.int32, device="cuda")
    if V > 2:
        y[::11] = V - 1  # and a token in eleven that is sure of another word
    return h.to(dt), w.to(dt), y


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("T,V", [(1, 1), (1, 2), (14, 2), (33, 3), (29, 8), (300, 8), (300, 40)])
@pytest.mark.parametrize("kind,d", [("f32", 4), ("f32", 64), ("bf16", 128)])
def test_a_small_loss_of_large_logits(kind, d, T, V, weighted):
    h, w, y = make(T, d, V, kind)
    u = torch.rand(T, generator=torch.Generator(device="cuda").manual_seed(T), device="cuda") + 0.5 if weighted else None
    r = run(h, w, y, u, kind)
    f = run(h, w, y, u, kind, grads=False)
    h64, w64, at = h.double(), w.double(), y.long()[:, None]
    z = h64 @ w64.T
    assert torch.equal(z.float().double(), z)
    e = torch.exp(z - z.amax(1, keepdim=True))
    rest = e.sum(1) - 1.0  # (exact to 2^-52)
    l = (z.amax(1) - z.gather(1, at)[:, 0]) + torch.log1p(rest)
    ls = (V + 16) * 2.0 ** -24 + 2.0 ** -20 * rest + 2.0 ** -22 * l
    for got in (r, f):
        assert ((got.token.double() - l).abs() <= ls).all(), ((got.token.double() - l).abs() / ls).max()
    live = torch.full((T,), 1.0 / T, dtype=torch.float64, device="cuda") if u is None else u.double()
    assert abs(r.loss.item() - (live * l).sum().item()) <= ((live * ls).sum() + 2.0 ** -23 * (live * l).sum()).item()
    p = e / e.sum(1, keepdim=True)
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    others = (p * (1 - one)).sum(1, keepdim=True)
    dz = live[:, None] * torch.where(one > 0, -others, p)
    half = torch.finfo(DT[kind][1]).eps / 2
    ep = p * (ls[:, None] + 2.0 ** -20) + 3 * 2.0 ** -24 * torch.where(one > 0, 1.0, p)
    if kind == "bf16":  # (fp16 holds the 1 of a largest logit exactly)
        ep = ep + torch.where(e == 1.0, 0.0, 2.0 ** -11 * p + 2.0 ** -25)
    edz = (live[:, None] * ep + half * dz.abs()) * (1 + 2.0 ** -7) + live[:, None] * 2.0 ** -24 * p
    for got, a, ea, b in ((r.dh, dz, edz, w64), (r.dw, dz.T, edz.T, h64)):
        ref = a @ b
        lim = ea @ b.abs() + (a.shape[1] / 16 + 80) * 2.0 ** -23 * (a.abs() @ b.abs()) + half * ref.abs() * 1.01 + 1e-38
        err = (got.double() - ref).abs()
        assert (err <= lim).all(), (err / lim).max()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_single_word_costs_nothing(kind):
    """V = 1: a softmax of 1, a loss of 0 and no gradient, whatever the logit."""
    g = torch.Generator(device="cuda").manual_seed(3)
    dt = DT[kind][1]
    h, w = torch.randn(70, 128, generator=g, device="cuda").mul(30).to(dt), torch.randn(1, 128, generator=g, device="cuda").to(dt)
    r = run(h, w, torch.zeros(70, dtype=torch.int32, device="cuda"), None, kind)
    assert r.loss.item() == 0 and not r.token.any() and not r.dh.any() and not r.dw.any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(20, 1), (20, 300), (300, 2), (300, 300)])
@pytest.mark.parametrize("size", [1e5, 1e9, 1e13])
def test_logits_without_digits(kind, T, V, size):
    """Logits whose fp32 step is above 1: losses within the products' error, gradients of probabilities near 0 and 1, all finite."""
    h, w, y, _ = make_plain(T, 256, V, kind, 17)
    h = (h.float() * size).to(h.dtype)
    r = run(h, w, y, None, kind)
    check(r, h, w, y, None, kind)
    assert torch.isfinite(r.token).all() and (V > 1 or not r.token.any())
