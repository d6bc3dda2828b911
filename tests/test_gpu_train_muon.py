"""RoundRobinTrainer(update="muon"): a run from a loaded initialization is the same run, whatever the trainer did before."""
import pytest
import torch

from synth import moe_inputs as mi
from tests.gpu_util import need_gpu, status

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    return need_gpu()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("update", ["sgd", "muon"])
def test_a_loaded_trainer_starts_anew(L, dtype, update):
    from paper_2506_02965_gb300.train import RoundRobinTrainer
    sh = mi.MoEShape("t", 40, 128, 8, 128, 2, dtype)
    tr = RoundRobinTrainer(sh, 2, lr=0.05, update=update)
    init = mi.train_init(sh, 2, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    batches = [[tuple(torch.randn(40, 128, generator=g, device="cuda").to(dt) for _ in range(2))] for _ in range(2)]

    def run():
        tr.load(init)
        _, log = tr.run(batches, [[0, 1], [1, 0]], 1)
        state = [tr.w_router, tr.w1, tr.w2] + ([tr.m_router, tr.m1, tr.m2] if tr.master else [])
        state += [m.momentum for m in tr.muon] if tr.muon else []
        return [t.clone() for t in state + [log]]

    first, second = run(), run()
    assert all(torch.equal(a, b) for a, b in zip(first, second)) and status(L) == 0
    if tr.muon:
        assert all(m.momentum.any() for m in tr.muon)
        tr.load(init)
        assert not any(m.momentum.any() for m in tr.muon)


def test_kernels_are_counted_for_sgd_only(L):
    from paper_2506_02965_gb300.train import RoundRobinTrainer
    sh = mi.MoEShape("t", 8, 128, 4, 128, 2, "bf16")
    tr = RoundRobinTrainer(sh, 1, lr=0.1)
    assert tr.kernels_per_step() == tr.layer.kernels_per_step() + 5
    with pytest.raises(ValueError, match="sgd"):
        RoundRobinTrainer(sh, 1, lr=0.1, update="muon").kernels_per_step()
