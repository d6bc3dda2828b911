"""The embedding's gradient of large batches: what its sort does where a warp has more keys than it keeps.

A warp of the sort owns ceil(T / warps) tokens, of up to 16 CTAs of 32 warps, or 4 CTAs where dW has more than 256 MB, and reads its
keys again for the second walk above 256 of them. Tolerances as in test_gpu_embed.
"""
import pytest
import torch

from paper_2506_02965_gb300 import _lib as L
from tests.test_gpu_embed import backward, check_bwd, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,T,d,V", [("bf16", 140000, 8, 3000), ("f32", 140001, 5, 262144), ("bf16", 300000, 16, 70000),
                                        ("bf16", 40000, 1024, 140000), ("f32", 33000, 512, 140001)])
@pytest.mark.parametrize("skew", [True, False])
def test_keys_read_again(kind, T, d, V, skew):
    ids, w, dout = make(T, d, V, kind, T + d, skew=skew)
    ids[::7] = -1
    ids[T // 2:T // 2 + T // 8] = V - 1  # padding by a real id: a run of thousands of tokens
    dw = backward(ids, dout, V, kind, 0.7, torch.full_like(w, float("nan")))
    check_bwd(ids, dout, V, 0.7, dw)
    assert torch.equal(dw, backward(ids, dout, V, kind, 0.7, torch.empty_like(w)))
    base = w.clone()
    check_bwd(ids, dout, V, 0.7, backward(ids, dout, V, kind, 0.7, w, accumulate=True), base)
    assert L.moe_device_status() == 0
