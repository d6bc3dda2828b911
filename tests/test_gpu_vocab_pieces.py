"""The vocabulary loss of batches that are taken in pieces, and of weights far below 1. Tolerances as in test_gpu_vocab_loss."""
import pytest
import torch

from paper_2506_02965_gb300 import _lib as L
from tests.test_gpu_vocab_loss import DT, check, make, run

pytestmark = pytest.mark.gpu

# With gradients a piece has up to max(4096, 2 d, 2^28 / V) tokens (rounded up to 256) in bf16 and 2^28 / V in fp32; without, 65536
# in bf16 and 2^28 / V in fp32.


@pytest.mark.parametrize("kind,T,d,V,grads,pieces", [
    ("bf16", 4500, 128, 65537, True, 2), ("bf16", 8449, 128, 66000, True, 3), ("bf16", 9100, 128, 50021, True, 2),
    ("bf16", 4400, 2176, 70001, True, 2), ("f32", 300, 4, 1500001, True, 3), ("bf16", 65537, 128, 50, False, 2),
    ("bf16", 140000, 256, 301, False, 3), ("f32", 1100, 16, 262144, False, 2), ("f32", 300, 4, 1500001, False, 3)])
def test_pieces(kind, T, d, V, grads, pieces):
    most = (max(4096, 2 * d, 2 ** 28 // V) if grads else 65536) if kind == "bf16" else max(128, 2 ** 28 // V // 128 * 128)
    assert -(-T // most) == pieces
    h, w, y, u = make(T, d, V, kind, 5)
    y[::3] = -1
    check(run(h, w, y, u, kind, grads=grads), h, w, y, u, kind)
    assert L.moe_device_status() == 0


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("size", [1e-25, 1e-31, 1e-33, 1e-36, 1e-42])
def test_small_weights(kind, T, size):
    """Loss and gradients scale with the weights down to what the types hold. In check()'s bounds stands 1e-38 beside the
    roundings relative to the values; here, half a step of a subnormal number in its place: of dz in its type times the other
    operand's magnitudes, of the result, and of the products' fp32 terms."""
    V, dt = 300, DT[kind][1]
    h, w, y, u = make(T, 128, V, kind, 13)
    y[::5] = -1
    u = (u + 0.25) * size
    r = run(h, w, y, u, kind)
    h64, w64, u64 = h.double(), w.double(), u.double() * (y >= 0)
    at = y.long().clamp(min=0)[:, None]
    z = h64 @ w64.T
    tau = (128 / 16 + 8) * 2.0 ** -23 * (h64.abs() @ w64.abs().T).amax(1)
    lse = torch.logsumexp(z, 1)
    token = torch.where(y >= 0, lse - z.gather(1, at)[:, 0], 0.0)
    off = torch.where(y >= 0, 2 * tau + 2.0 ** -18 + 2.0 ** -23 * (lse.abs() + z.abs().amax(1)), 0.0)
    assert ((r.token.double() - token).abs() <= off).all()
    total = (u64 * token).sum()
    assert total > 0 and (r.loss.double() - total).abs() <= (u64 * (off + 2.0 ** -23 * token)).sum() + 2.0 ** -23 * total + 2.0 ** -150
    half, tiny = torch.finfo(dt).eps / 2, 2.0 ** -134 if kind == "bf16" else 2.0 ** -150
    p = torch.exp(z - lse[:, None])
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    dz = u64[:, None] * (p - one)
    edz = p * (2 * tau[:, None] + 2.0 ** -18) + half * (p - one).abs()
    edz = edz + (2.0 ** -11 * p + 2.0 ** -25 * p.amax(1, keepdim=True) if kind == "bf16" else 2.0 ** -22)
    edz = u64[:, None] * edz * (1 + 2.0 ** -7) + tiny + 2.0 ** -149
    for got, a, ea, b in ((r.dh, dz, edz, w64), (r.dw, dz.T, edz.T, h64)):
        ref, k = a @ b, a.shape[1]
        lim = ea @ b.abs() + (k / 16 + 80) * 2.0 ** -23 * (a.abs() @ b.abs()) + half * ref.abs() * 1.01 + tiny + (k + 80) * 2.0 ** -149
        assert ((got.double() - ref).abs() <= lim).all(), ((got.double() - ref).abs() / lim).max()
        if size >= 1e-33:  # zeros, or another size's values, are far outside
            assert ref.norm() >= 10 * lim.norm(), (ref.norm() / lim.norm())


@pytest.mark.slow
def test_the_largest_vocabulary():
    """One token against 2^31 - 1 - 2^18 words (35 GB of W and of dW): logits of 0 but for the last three words'. A lane of the statistics
    adds up 2^17 shares of 512 equal terms, each half a step off: 2^17 2^-25 of its sum, a 32nd of V exp(-24) = 0.081, in 32 lanes."""
    T, d, V = 1, 4, 2 ** 31 - 1 - 2 ** 18
    w = torch.zeros(V, d, device="cuda")
    w[-3:, 0] = torch.tensor([1.0, 2.0, 3.0], device="cuda")
    h = torch.tensor([[8.0, 0.0, 0.0, 0.0]], device="cuda")
    y = torch.tensor([V - 1], dtype=torch.int32, device="cuda")
    r = run(h, w, y, None, "f32")
    e = torch.exp(torch.tensor([-24.0, -16.0, -8.0, 0.0], dtype=torch.float64))
    total = ((V - 3) * e[0] + e[1] + e[2] + e[3]).item()
    p = [x.item() / total for x in e]
    off = 2.0 ** 17 * 2.0 ** -25 * V * e[0].item() / total + 2.0 ** -20  # relative, of s and so of every probability
    assert abs(r.token.item() - torch.log(torch.tensor(total, dtype=torch.float64)).item()) <= off and torch.equal(r.loss, r.token)
    rest = r.dw[:-3, 0]
    for extreme in (rest.amin(), rest.amax()):  # the first rows, those past 2^30 and the last ones alike
        assert abs(extreme.item() - 8 * p[0]) <= 8 * p[0] * (off + 2.0 ** -20)
    for i, want in ((-3, p[1]), (-2, p[2]), (-1, p[3] - 1.0)):
        assert abs(r.dw[i, 0].item() - 8 * want) <= 8 * (p[3] * off + 2.0 ** -20)
    assert r.dw[:, 1:].amax().item() == 0 and r.dw[:, 1:].amin().item() == 0
    assert abs(r.dh[0, 0].item() - (p[1] + 2 * p[2] + 3 * (p[3] - 1.0))) <= 3 * off + 2.0 ** -18 and not r.dh[0, 1:].any()
    assert L.moe_device_status() == 0
