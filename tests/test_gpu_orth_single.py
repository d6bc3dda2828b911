"""Orthogonalised updates of one or two large matrices, whose norm is added up from a thousand parts and more.

The steps' tolerances are those of test_gpu_orth. The norm itself: a diagonal matrix of n equal values is X = n^-1/2 I, and one
step makes p(n^-1/2) of it, p the step's polynomial, whose largest part is a X. In it bf16 matrices have X to 2^-14, and b A + c A A,
below 2^-6 of a for n > 400, from an fp16 A and rounded to fp16 (2^-10 of that in all); so with the norm's fp32 sums p is off by
less than 2^-10 of itself, and the result by half a bf16 step, 2^-8, more. fp32: some twenty roundings of 2^-24 and the sums', below 2^-18.
A part of u that counted twice, or not at all, of a thousand would change the norm by 2^-11 of itself: the fp32 forms see it.
"""
import pytest
import torch

from paper_2506_02965_gb300 import _lib as L
from tests.test_gpu_orth import COEF, check, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G,R,C", [(1, 4096, 4096), (2, 3000, 4001), (1, 2500, 2500)])
def test_large_with_momentum(G, R, C):
    dw, mom = make(G, R, C, "bf16", 21)
    out, mo = run(dw, mom)
    check(out, mo, dw, mom, "bf16")
    again, _ = run(dw, mom)
    assert torch.equal(out, again) and L.moe_device_status() == 0


@pytest.mark.parametrize("dt,tol", [(torch.bfloat16, 2.0 ** -8 + 2.0 ** -10), (torch.float32, 2.0 ** -18)])
@pytest.mark.parametrize("n", [700, 2048, 4096])
def test_norm_of_many_parts(dt, tol, n):
    """Every part counts once: equal values on the diagonal, and the same with a part of the rows without one."""
    for gone in (0, n // 3):
        dw = torch.zeros(1, n, n, dtype=dt, device="cuda")
        i = torch.arange(gone, n, device="cuda")
        dw[0, i, i] = 3.0
        out, _ = run(dw, None, steps=1)
        s = (n - gone) ** -0.5
        want = COEF[0] * s + COEF[1] * s ** 3 + COEF[2] * s ** 5
        got = out[0].diagonal().double()
        assert not got[:gone].any() and ((got[gone:] - want).abs() <= tol * want).all(), (got[gone:] / want - 1).abs().max()
        assert (out[0] - torch.diag(out[0].diagonal())).abs().max() == 0
