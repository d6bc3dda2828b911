"""Waits that run out in the products of the vocabulary loss and of the orthogonalised updates: reported, and the same call is
right afterwards (as test_gpu_failure has it for the layer's GEMMs: a limit of 1 ns and contractions of well over
the 40 us that a wait may sleep before it looks at its limit)."""
import pytest
import torch

from tests.gpu_util import need_gpu, status

pytestmark = pytest.mark.gpu


def _loss(L, T, d, V):
    gen = torch.Generator(device="cuda").manual_seed(T)
    h = torch.randn(T, d, generator=gen, device="cuda").bfloat16()
    w = (torch.randn(V, d, generator=gen, device="cuda") * 0.02).bfloat16()
    y = torch.randint(0, V, (T,), generator=gen, device="cuda", dtype=torch.int32)
    loss, token = torch.empty(1, device="cuda"), torch.empty(T, device="cuda")
    ws = torch.empty(L.moe_vocab_loss_workspace_size(T, d, V, L.MOE_BF16, False), dtype=torch.uint8, device="cuda")
    L.moe_vocab_loss(T, d, V, L.MOE_BF16, h, w, y, None, loss, token, None, None, ws, ws.numel())
    z = h.double() @ w.double().T
    # logits: d / 16 steps that each truncate by up to 2^-23 of a partial sum of at most the terms' magnitudes
    tol = 2 * d / 16 * 2.0 ** -23 * (h.double().abs() @ w.double().abs().T).max().item()
    return token.double(), torch.logsumexp(z, 1) - z.gather(1, y[:, None].long())[:, 0], tol


def _update(L, G, R, C):
    from tests.test_gpu_orth import run, steps64
    gen = torch.Generator(device="cuda").manual_seed(G)
    dw = torch.randn(G, R, C, generator=gen, device="cuda").bfloat16()
    out = run(dw, None)[0]
    some = [0, G // 2, G - 1]
    ref = steps64(dw[some].double(), 5)
    return out[some].double(), ref, 0.03 * ref.abs().max().item()


@pytest.mark.parametrize("call,args", [
    (_loss, (8, 65536, 600)),       # 32 rows of A
    (_loss, (100, 65536, 600)),     # single CTAs
    (_loss, (4096, 8192, 4096)),    # pairs
    (_update, (64, 300, 16384))])
def test_waits_give_up_and_the_call_recovers(call, args):
    L = need_gpu()
    assert status(L) == 0
    L.moe_set_wait_limit_ns(1)
    try:
        call(L, *args)
        code = status(L)
    finally:
        L.moe_set_wait_limit_ns(2_000_000_000)
    assert code == L.MOE_ERR_TIMEOUT
    got, ref, tol = call(L, *args)
    assert status(L) == 0
    assert (got - ref).abs().max().item() <= tol
