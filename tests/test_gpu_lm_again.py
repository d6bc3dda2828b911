"""A step of TokenMoE a second time, and from a graph: from the same weights and balance biases the same bits."""
import pytest
import torch

from synth import moe_inputs as mi
from tests.gpu_util import need_gpu, status
from tests.test_gpu_lm import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    return need_gpu()


@pytest.mark.parametrize("dtype,T,d,E,F,k,n,V,tied", [("f32", 97, 96, 8, 72, 3, 2, 1000, False), ("bf16", 300, 256, 8, 256, 2, 1, 777, True)])
def test_the_same_step_again(L, dtype, T, d, E, F, k, n, V, tied):
    sh = mi.MoEShape("lm", T, d, E, F, k, dtype, normalize_topk=1)
    lm, ids, target = build(sh, V, n, L.make_gate_rule(L.MOE_SCORE_SIGMOID, 2, 2, 1, 1.5), tied, T)
    ids[-T // 8:], target[-T // 8:] = -1, -1
    bias = [b.balance_bias.clone() for b in lm.net.blocks]

    def start():
        for b, v in zip(lm.net.blocks, bias):
            b.balance_bias.copy_(v)

    def results():
        grads = dict(lm.grads())
        grads.update({(i, m): g for i, b in enumerate(lm.net.blocks) for m, g in b.grads().items()})
        return {m: g.clone() for m, g in grads.items()}, lm.loss.clone(), lm.token_loss.clone()

    def same(a, b):
        return a[0].keys() == b[0].keys() and all(torch.equal(a[0][m], b[0][m]) for m in a[0]) and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])

    lm.step(ids, target)
    first = results()
    assert all(torch.isfinite(g).all() for g in first[0].values())
    start()
    lm.evaluate(ids, target)
    assert torch.equal(lm.loss, first[1]) and torch.equal(lm.token_loss, first[2])
    start()
    lm.step(ids, target)
    assert same(results(), first)
    start()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lm.step(ids, target)
    start()
    for g in lm.grads().values():
        g.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert same(results(), first) and status(L) == 0
