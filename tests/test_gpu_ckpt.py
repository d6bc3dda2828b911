"""8-bit activation checkpoints: packing bit for bit against the same 32-bit arithmetic on the host,
and the SwiGLU backward from a checkpoint against 64 bits.

Bounds. u = 2^-24. G and U are the same 32-bit products on both sides. The sigmoid of fp32
results is off by 4 u (exponential 2, sum, quotient), that of bf16 ones by 2^-21 (fast exponential: 2 + 1.2 |G|
units for |G| < 11, where it counts; beyond, s is 0 or 1 to that accuracy), the products after it by 4 u:
within 32 u (2^-19 for bf16) of |dA U| (1 + |G|), plus half a spacing of bf16, at most 2^-8 of the result."""
import numpy as np
import pytest
import torch

from tests.gpu_util import need_gpu, status

pytestmark = pytest.mark.gpu
B = 128


@pytest.fixture(scope="module")
def L():
    return need_gpu()


def host_pack(x):
    """q, scale of float32 values, in float32 arithmetic."""
    R, C = x.shape
    n = -(-C // B)
    b = np.zeros((R, n * B), np.float32)
    b[:, :C] = x
    b = b.reshape(R, n, B)
    with np.errstate(all="ignore"):
        a = np.abs(b).max(2)
        bad = ~np.isfinite(b).all(2)
        zero = ~bad & (a < np.float32(2.0 ** -100))
        one = np.float32(1)
        safe = np.where(zero | bad, one, a)
        scale = np.where(zero, np.float32(0), np.where(bad, np.float32(np.nan), safe / np.float32(127)))
        inv = np.where(zero | bad, np.float32(0), np.float32(127) / safe)
        q = np.rint(b * inv[..., None])
    return q.reshape(R, -1)[:, :C], scale.astype(np.float32), np.repeat(bad, B, 1)[:, :C]


def pack(L, x):
    R, C = x.shape
    mt = L.MOE_BF16 if x.dtype == torch.bfloat16 else L.MOE_F32
    q = torch.full((R, C), 77, dtype=torch.int8, device="cuda")
    s = torch.full((R, -(-C // B)), 5.0, device="cuda")
    L.moe_ckpt_pack(R, C, mt, x, q, s)
    assert status(L) == 0
    return q, s


def check(L, x):
    R, C = x.shape
    mt = L.MOE_BF16 if x.dtype == torch.bfloat16 else L.MOE_F32
    q, s = pack(L, x)
    hq, hs, bad = host_pack(x.float().cpu().numpy())
    np.testing.assert_array_equal(s.cpu().numpy(), hs)
    np.testing.assert_array_equal(q.cpu().numpy()[~bad], hq[~bad])
    back = torch.empty_like(x)
    L.moe_ckpt_unpack(R, C, mt, q, s, back)
    held = (q.float() * s.repeat_interleave(B, 1)[:, :C]).to(x.dtype)
    assert torch.equal(back[~torch.isnan(held)], held[~torch.isnan(held)])
    assert torch.equal(torch.isnan(back), torch.isnan(held))
    assert np.array_equal(torch.isnan(held).cpu().numpy(), bad)
    return q, s


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", [(1, 1), (2, 5), (3, 127), (3, 128), (5, 129), (4, 136), (7, 256), (9, 1000), (65, 1366), (33, 4096),
                                 (257, 72), (1, 14336), (1031, 264)])
def test_pack_and_unpack_bit_for_bit(L, R, C, dt):
    g = torch.Generator(device="cuda").manual_seed(R * 31 + C)
    check(L, (torch.randn(R, C, generator=g, device="cuda") * torch.exp(3 * torch.randn(R, 1, generator=g, device="cuda"))).to(dt))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("C", [384, 383])
def test_blocks_of_odd_values(L, dt, C):
    """Zeros, magnitudes around the smallest that is scaled, the largest finite one, infinities and NaN in
    one block of a row: the other blocks of the row are not touched by them."""
    top = torch.finfo(dt).max
    x = torch.randn(12, C, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dt)
    x[0] = 0
    x[1, :128] = 0
    x[2] = x[2] * 2.0 ** -102
    x[3] = 2.0 ** -100
    x[4] = 2.0 ** -101
    x[5, 130] = top
    x[6, 3] = -top
    x[7, 140] = float("inf")
    x[8, 5] = -float("inf")
    x[9, 260] = float("nan")
    x[10, 128:256] = -0.0
    x[11, 0], x[11, 1] = float("nan"), float("inf")
    q, s = check(L, x)
    assert (q[0] == 0).all() and (s[0] == 0).all() and (q[3] == 127).all()
    assert torch.isnan(s[7, 1]) and torch.isfinite(s[7, [0, 2]]).all()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_unaligned_buffers(L, dt):
    R, C = 9, 512
    x = torch.randn(R, C, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(dt)
    q, s = pack(L, x)
    whole, qw = torch.zeros(R * C + 3, dtype=dt, device="cuda"), torch.zeros(R * C + 3, dtype=torch.int8, device="cuda")
    xs, qs = whole[3:].view(R, C), qw[3:].view(R, C)
    xs.copy_(x)
    mt = L.MOE_BF16 if dt == torch.bfloat16 else L.MOE_F32
    s2 = torch.empty_like(s)
    L.moe_ckpt_pack(R, C, mt, xs, qs, s2)
    assert torch.equal(q, qs) and torch.equal(s, s2) and qw[:3].abs().max() == 0
    back = torch.empty_like(x)
    L.moe_ckpt_unpack(R, C, mt, q, s, back)
    L.moe_ckpt_unpack(R, C, mt, qs, s2, xs)
    assert torch.equal(back, xs) and status(L) == 0


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,F", [(1, 1), (3, 5), (2, 64), (5, 100), (17, 128), (9, 136), (130, 1366), (33, 1408), (4, 14336), (1000, 72),
                                 (70, 511)])
def test_swiglu_backward(L, R, F, dt):
    g = torch.Generator(device="cuda").manual_seed(R + 5 * F)
    gu = (1.5 * torch.randn(R, 2 * F, generator=g, device="cuda")).to(dt)
    gu[0, 0] = 60.0  # saturated gates
    gu[-1, F - 1] = -60.0
    da = torch.randn(R, F, generator=g, device="cuda").to(dt)
    q, s = pack(L, gu)
    act, dh = torch.empty(R, F, dtype=dt, device="cuda"), torch.empty(R, 2 * F, dtype=dt, device="cuda")
    mt = L.MOE_BF16 if dt == torch.bfloat16 else L.MOE_F32
    L.moe_ckpt_swiglu_bwd(R, F, mt, q, s, da, act, dh)
    assert status(L) == 0
    held = (q.float() * s.repeat_interleave(B, 1)[:, :2 * F]).double()
    G, U, d = held[:, :F], held[:, F:], da.double()
    sg = torch.sigmoid(G)
    rel, half = (2.0 ** -19, 2.0 ** -8) if dt == torch.bfloat16 else (32 * 2.0 ** -24, 0.0)
    size = (1 + G.abs())
    for got, ref, mag in ((act, G * sg * U, U.abs() * size), (dh[:, :F], d * U * sg * (1 + G * torch.sigmoid(-G)), (d * U).abs() * size),
                          (dh[:, F:], d * G * sg, d.abs() * size)):
        bad = (got.double() - ref).abs() > rel * mag + half * ref.abs() + 2.0 ** -120
        assert not bad.any(), int(bad.sum())


def test_swiglu_gradient_against_differences(L):
    """[dG|dU] against central differences of the 64-bit activation at the held values: a step of 2^-12 leaves
    (2^-24 / 6) times a third derivative below 8."""
    R, F, step = 4, 40, 2.0 ** -12
    g = torch.Generator(device="cuda").manual_seed(9)
    gu, da = torch.randn(R, 2 * F, generator=g, device="cuda"), torch.randn(R, F, generator=g, device="cuda")
    q, s = pack(L, gu)
    act, dh = torch.empty(R, F, device="cuda"), torch.empty(R, 2 * F, device="cuda")
    L.moe_ckpt_swiglu_bwd(R, F, L.MOE_F32, q, s, da, act, dh)
    held = (q.float() * s.repeat_interleave(B, 1)[:, :2 * F]).double()

    def loss(G, U):  # per element: each output depends on its own pair alone
        return da.double() * G * torch.sigmoid(G) * U

    G, U = held[:, :F], held[:, F:]
    dG = (loss(G + step, U) - loss(G - step, U)) / (2 * step)
    dU = (loss(G, U + step) - loss(G, U - step)) / (2 * step)
    assert (dh.double() - torch.cat([dG, dU], 1)).abs().max() < 1e-5


def test_more_than_2_31_elements(L):
    """Offsets past 32 bits: the first and the last rows of 4.3 GB hold what a small call gives them."""
    R, C = 2_101_003, 1032
    assert R * C > 1 << 31
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(5, C, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    x[:5], x[-5:] = tail, tail
    q, s = pack(L, x)
    qt, st = pack(L, tail)
    for part in (slice(0, 5), slice(R - 5, R)):
        assert torch.equal(q[part], qt) and torch.equal(s[part], st)
    assert int(q[5:-5].abs().max()) == 0
    x.fill_(1.0)
    L.moe_ckpt_unpack(R, C, L.MOE_BF16, q, s, x)
    assert torch.equal(x[:5], x[-5:]) and float(x[5:-5].abs().max()) == 0
    del x, q, s
    torch.cuda.empty_cache()


def test_nothing_to_do(L):
    L.moe_ckpt_pack(0, 8, L.MOE_F32, None, None, None)
    L.moe_ckpt_unpack(0, 8, L.MOE_BF16, None, None, None)
    L.moe_ckpt_swiglu_bwd(0, 8, L.MOE_BF16, None, None, None, None, None)
    assert status(L) == 0


@pytest.mark.parametrize("C", [2 ** 31 - 1, 2 ** 31 - 120])
def test_the_widest_rows(L, C):
    """A row of nearly 2^31 columns: its first and last blocks are those of short rows, all others zeros."""
    n = 300
    x = torch.zeros(1, C, dtype=torch.bfloat16, device="cuda")
    head = torch.randn(1, n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    cut = C // B * B - B  # the last whole block and the one after it
    x[:, :n], x[:, cut:] = head, head[:, :C - cut]
    q, s = pack(L, x)
    qh, sh = pack(L, head)
    qt, st = pack(L, head[:, :C - cut].contiguous())
    assert torch.equal(q[:, :n], qh) and torch.equal(s[:, :3], sh) and torch.equal(q[:, cut:], qt) and torch.equal(s[:, -2:], st)
    assert int(q[:, n:cut].abs().max()) == 0 and float(s[:, 3:-2].abs().max()) == 0
    x.fill_(1.0)
    L.moe_ckpt_unpack(1, C, L.MOE_BF16, q, s, x)
    held = torch.empty_like(head)
    L.moe_ckpt_unpack(1, n, L.MOE_BF16, qh, sh, held)
    assert status(L) == 0 and torch.equal(x[:, :n], held) and float(x[:, n:cut].abs().max()) == 0
    back = torch.empty(1, C - cut, dtype=torch.bfloat16, device="cuda")
    L.moe_ckpt_unpack(1, C - cut, L.MOE_BF16, qt, st, back)
    assert torch.equal(x[:, cut:], back)
    del x, q, s
    torch.cuda.empty_cache()
