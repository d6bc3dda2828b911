"""How far orthogonalised updates may be off 64 bits, as figures of their own.

The bounds are of the norm, for gradients of eight directions `strong` times their noise. They come from the roundings alone, not from
a kernel: the steps in fp32 with X to 14 bits, A and b A + c A A (+ t I) to fp16's 11, over matrices of 64 x 96 to 2048 x 2048, are
off by up to 1.3e-3 (5 steps) and 2.0e-3 (8) where the directions do not outweigh the noise 30 times, 1.9e-3 and 3.4e-3 at 100 times,
3.3e-3 and 1.5e-2 at 1000 times; the result's own rounding to bf16 is 2^-9 and a little less, 1.7e-3, independent of those. The bounds
are the roots of the squares' sums, 2.1e-3, 2.7e-3, 2.6e-3, 3.8e-3, 3.8e-3 and 1.5e-2, and 1.3 times that. With X in fp16's 11 bits alone the
roundings make 8e-3 at 30 times, 2.2e-2 at 100 and 4e-2 at 1000: what holds these bounds is better than that. fp32: the steps with plain
fp32 products are off by 2.2e-6 (5 steps) and 4.2e-6 (8), 5.7e-6 and 7.4e-6 at 30 times, 1.6e-5 and 2.1e-5, 3.0e-5 and 1.9e-4; twice that.
"""
import pytest
import torch

from tests.test_gpu_orth import make, run, steps64

pytestmark = pytest.mark.gpu
MOST = {"bf16": {(0.0, 5): 2.8e-3, (0.0, 8): 3.5e-3, (3.0, 5): 2.8e-3, (3.0, 8): 3.5e-3, (30.0, 5): 2.8e-3, (30.0, 8): 3.5e-3,
                 (100.0, 5): 3.4e-3, (100.0, 8): 5.0e-3, (1000.0, 5): 5.0e-3, (1000.0, 8): 2.0e-2},
        "f32": {(0.0, 5): 4.4e-6, (0.0, 8): 8.4e-6, (3.0, 5): 4.4e-6, (3.0, 8): 8.4e-6, (30.0, 5): 1.2e-5, (30.0, 8): 1.5e-5,
                (100.0, 5): 3.2e-5, (100.0, 8): 4.2e-5, (1000.0, 5): 6e-5, (1000.0, 8): 3.8e-4}}


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [5, 8])
@pytest.mark.parametrize("strong", [0.0, 3.0, 30.0, 100.0, 1000.0])
@pytest.mark.parametrize("G,R,C", [(3, 64, 96), (2, 333, 1000), (1, 1000, 333), (1, 512, 768)])
def test_distance_from_64_bits(kind, steps, strong, G, R, C):
    dw, _ = make(G, R, C, kind, R + int(strong), strong=strong)
    out, _ = run(dw, None, steps=steps)
    ref = steps64(dw.double(), steps)
    off = (out.double() - ref).flatten(1).norm(dim=1) / ref.flatten(1).norm(dim=1)
    assert (off <= MOST[kind][strong, steps]).all(), off


@pytest.mark.parametrize("R,C", [(1024, 2816), (2048, 2048)])
def test_distance_of_large_matrices(R, C):
    dw, mom = make(2, R, C, "bf16", 31)
    out, mo = run(dw, mom)
    u = dw.double() + 0.95 * (0.95 * mom.double() + dw.double())
    ref = steps64(u, 5)
    off = (out.double() - ref).flatten(1).norm(dim=1) / ref.flatten(1).norm(dim=1)
    assert (off <= MOST["bf16"][3.0, 5]).all(), off
