"""A stack from token ids to its loss (lm.TokenMoE), and the orthogonalised update of its matrices (lm.Muon), against plain
64-bit forms.

Bounds. The states and gradients of the stack are those of test_gpu_block (fp32 2e-3, bf16 5e-2 of their norms, over one and
two blocks); the loss is a mean of log-sums of logits of about 1 that inherit the states' error: the same, of log(V).
"""
import math

import pytest
import torch

from synth import moe_inputs as mi
from tests.gpu_util import need_gpu, status
from tests.test_gpu_block import near, plain
from tests.test_gpu_orth import steps64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    return need_gpu()


def build(sh, V, n, rule, tied, seed):
    from paper_2506_02965_gb300.lm import TokenMoE
    g = torch.Generator(device="cuda").manual_seed(seed)
    lm = TokenMoE(sh, V, n, rule, tied=tied)
    for b in lm.net.blocks:
        for t, m, std in ((b.gamma, 1.0, 0.1), (b.beta, 0.0, 0.1), (b.w_router, 0.0, 0.1), (b.w1, 0.0, 0.1), (b.w2, 0.0, 0.1),
                          (b.balance_bias, 0.0, 0.05)):
            t.normal_(m, std, generator=g)
    lm.w_in.normal_(0.0, 1.0 / math.sqrt(sh.d_model), generator=g)
    if not tied:
        lm.w_out.normal_(0.0, 0.1, generator=g)
    ids = torch.randint(0, V, (sh.T,), generator=g, device="cuda", dtype=torch.int32)
    target = torch.randint(0, V, (sh.T,), generator=g, device="cuda", dtype=torch.int32)
    return lm, ids, target


@pytest.mark.parametrize("dtype,T,d,E,F,k,n,V,tied,tol", [
    ("f32", 150, 64, 6, 50, 2, 1, 301, True, 2e-3), ("f32", 97, 96, 8, 72, 3, 2, 1000, False, 2e-3),
    ("bf16", 300, 256, 8, 256, 2, 1, 777, True, 5e-2), ("bf16", 257, 128, 16, 384, 4, 2, 2050, False, 5e-2)])
def test_from_ids_to_gradients(L, dtype, T, d, E, F, k, n, V, tied, tol):
    sh = mi.MoEShape("lm", T, d, E, F, k, dtype, normalize_topk=1)
    rule = L.make_gate_rule(L.MOE_SCORE_SIGMOID, 2, 2 if E == 4 else 1 if E == 6 else 2, 1, 1.5)
    lm, ids, target = build(sh, V, n, rule, tied, T + V)
    ids[T // 3:T // 2] = ids[0]     # a token that comes often
    ids[-T // 8:], target[-T // 8:] = -1, -1   # padding behind the sequence
    target[::7] = -100
    loss = lm.step(ids, target).clone()
    lm.check_status()
    net = lm.net
    bias = [b.balance_bias.clone() for b in net.blocks]
    picks = [b.topk_idx.long() for b in net.blocks]
    live, counts = ids >= 0, target >= 0
    x = torch.where(live[:, None], lm.w_in.double()[ids.long().clamp(min=0)] * lm.scale, 0.0).to(lm.x.dtype)
    assert (lm.x.double() - x.double()).abs().max() <= 2 * torch.finfo(x.dtype).eps * x.double().abs().max()
    h = plain(net, sh, picks, x, torch.zeros_like(x), 1.5, x.dtype, [0, T])["out"]
    w = lm.w_out.double()
    z = h @ w.T
    at = target.long().clamp(min=0)
    lse = torch.logsumexp(z, 1)
    u = counts.double() / counts.sum()
    ref_loss = (u * (lse - z.gather(1, at[:, None])[:, 0])).sum()
    assert abs(loss.item() - ref_loss.item()) <= tol * math.log(V)
    dz = u[:, None] * (torch.exp(z - lse[:, None]) - torch.zeros_like(z).scatter_(1, at[:, None], 1.0))
    dh = dz @ w
    near("dh", lm.dh, dh, tol)
    ref = plain(net, sh, picks, x, dh.to(x.dtype), 1.5, x.dtype, [0, T])
    for i, b in enumerate(net.blocks):
        for name, g in b.grads().items():
            near((i, name), g, ref[i][name], tol)
    dw_out = dz.T @ h
    dw_in = torch.zeros(V + 1, d, dtype=torch.float64, device="cuda").index_add_(0, torch.where(live, ids, V).long(), ref["dx"])[:V] * lm.scale
    if tied:
        near("dw", lm.grads()["w_in"], dw_in + dw_out, tol)
    else:
        near("dw_in", lm.grads()["w_in"], dw_in, tol)
        near("dw_out", lm.grads()["w_out"], dw_out, tol)
    # the loss alone, on the same weights and biases, is the same number; a second step gives the same bits
    for b, v in zip(net.blocks, bias):
        b.balance_bias.copy_(v)
    first = {m: g.clone() for m, g in lm.grads().items()}
    one = lm.evaluate(ids, target).clone()
    lm.step(ids, target)
    for b, v in zip(net.blocks, bias):
        b.balance_bias.copy_(v)
    two = {m: g.clone() for m, g in lm.grads().items()}
    assert torch.equal(lm.step(ids, target), one)
    assert all(torch.equal(g, two[m]) for m, g in lm.grads().items()) and set(first) == set(two)


def test_a_run_of_updates(L):
    """Steps of the whole model: embedding and loss, the blocks, the experts by orthogonalised updates, the rest by SGD. Every
    update is what its definition makes of the gradients of the step before it."""
    from paper_2506_02965_gb300.lm import Muon
    sh = mi.MoEShape("lm", 200, 128, 8, 128, 2, "bf16", normalize_topk=1)
    lm, ids, target = build(sh, 500, 2, L.make_gate_rule(L.MOE_SCORE_SIGMOID, 2, 2, 1, 1.5), True, 3)
    muons = [(Muon(b.w1), Muon(b.w2)) for b in lm.net.blocks]
    masters = [(b.w1.float(), b.w2.float()) for b in lm.net.blocks]
    for it in range(3):
        lm.step(ids, target)
        for b, mu, ma in zip(lm.net.blocks, muons, masters):
            counts = b.counts.view(-1)
            for m, master, w, dw in zip(mu, ma, (b.w1, b.w2), (b.dw1, b.dw2)):
                before, mom = master.double(), m.momentum.double()
                m.update(w, dw, 0.02, counts, master)
                called = counts > 0
                mom = torch.where(called[:, None, None], 0.95 * mom + dw.double(), mom)
                u = dw.double() + 0.95 * mom
                want = before - 0.02 * m.scale * torch.where(called[:, None, None], steps64(u, 5), 0.0)
                # the update is off by 2e-2 of its norm at most (bf16 rounding 2^-9 rms, the products' a few times that)
                off = (master.double() - want).flatten(1).norm(dim=1)
                assert (off <= 2e-2 * (want - before).flatten(1).norm(dim=1) + 1e-6 * before.flatten(1).norm(dim=1)).all()
                assert torch.equal(w, master.to(w.dtype))
        for name, w in lm.params().items():
            L.moe_sgd_update(w, lm.grads()[name], 1, w.numel(), None, 0.1, L.MOE_BF16)
        for b in lm.net.blocks:
            L.moe_sgd_update(b.w_router, b.dw_router, 1, b.w_router.numel(), None, 0.1, L.MOE_BF16)
    assert status(L) == 0 and math.isfinite(lm.loss.item())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_trainer_with_orthogonalised_updates(L, dtype):
    """RoundRobinTrainer(update="muon"): called experts move by the orthogonalised momentum, uncalled ones and their momentum stay,
    and the routers move as with SGD."""
    from paper_2506_02965_gb300.train import RoundRobinTrainer
    sh = mi.MoEShape("t", 40, 128, 16, 128, 2, dtype)
    tr = RoundRobinTrainer(sh, 2, lr=0.05, update="muon")
    sgd = RoundRobinTrainer(sh, 2, lr=0.05)
    init = mi.train_init(sh, 2, seed=1)
    tr.load(init), sgd.load(init)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(40, 128, generator=g, device="cuda")
    x = (x[:1] + 0.05 * x).to(dt)   # alike: few experts are called
    y = torch.randn(40, 128, generator=g, device="cuda").to(dt)
    before = tr.w1.double().clone()
    tr.step(1, x, y), sgd.step(1, x, y)
    assert torch.equal(tr.w_router, sgd.w_router)
    called = tr.layer.counts.view(-1) > 0
    assert 0 < int(called.sum()) < 16
    want = 0.05 * tr.muon[0].scale * steps64((1 + 0.95) * tr.layer.dw1.double(), 5)
    move = before - (tr.m1 if tr.master else tr.w1).double()
    err = (move - want)[called].flatten(1).norm(dim=1) / want[called].flatten(1).norm(dim=1)
    assert (err <= (2e-2 if dtype == "bf16" else 1e-3)).all(), err
    assert torch.equal(tr.w1[~called], sgd.w1[~called]) and not tr.muon[0].momentum[~called].any()
    assert status(L) == 0


def test_refusals(L):
    from paper_2506_02965_gb300.lm import TokenMoE
    from paper_2506_02965_gb300.train import RoundRobinTrainer
    sh = mi.MoEShape("t", 8, 128, 4, 128, 2, "bf16")
    with pytest.raises(ValueError, match="vocab"):
        TokenMoE(sh, 0, 1)
    with pytest.raises(ValueError, match="update"):
        RoundRobinTrainer(sh, 1, lr=0.1, update="adam")
    lm = TokenMoE(sh, 10, 1)
    ids = torch.zeros(8, dtype=torch.int64, device="cuda")
    with pytest.raises(L.MoEError, match="ids: expected"):
        lm.step(ids, ids.int())
    with pytest.raises(L.MoEError, match="target: expected"):
        lm.evaluate(ids.int(), ids[:5].int())
