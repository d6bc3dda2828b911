"""Refusals of the operators around a stack of blocks: on the host, before any device work, with a reason."""
import os

import pytest

from paper_2506_02965_gb300 import build as _build

if not os.path.exists(_build.LIB) or _build._stale(_build.LIB, os.path.join(_build.CSRC, "moe_abi.cu")):
    _build.build()
from paper_2506_02965_gb300 import _lib as L  # noqa: E402

BAD = L.MOE_ERR_INVALID_ARG


def refused(frag, fn, *args, status=BAD):
    with pytest.raises(L.MoEError) as e:
        fn(*args, stream=0)
    assert e.value.status == status and frag in str(e.value), str(e.value)


@pytest.mark.parametrize("change,frag", [
    (dict(T=-1), "rows=-1"), (dict(T=1 << 31), "rows="), (dict(d=0), "width 0"), (dict(V=0), "V=0"), (dict(V=2 ** 31 - 1), "V="),
    (dict(dtype=7), "dtype"), (dict(ids=None), "ids is NULL"), (dict(ids=18), "ids is not aligned"), (dict(w=None), "w is NULL"),
    (dict(w=17), "w is not aligned"), (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"),
    (dict(out=None), "out is NULL"), (dict(out=17), "out is not aligned")])
def test_embed_forward(change, frag):
    a = dict(T=4, d=64, V=100, dtype=L.MOE_BF16, ids=16, w=16, scale=1.0, out=16)
    a.update(change)
    refused(frag, L.moe_embed_fwd, *a.values())


@pytest.mark.parametrize("change,frag", [
    (dict(T=-1), "rows=-1"), (dict(d=-3), "width -3"), (dict(V=-1), "V=-1"), (dict(ids=None), "ids is NULL"),
    (dict(dout=None), "dout is NULL"), (dict(dout=18), "dout is not aligned"), (dict(scale=float("nan")), "scale"),
    (dict(accumulate=2), "accumulate"), (dict(dw=None), "dw is NULL"), (dict(dw=18), "dw is not aligned"),
    (dict(ws=None), "workspace is NULL"), (dict(ws=24), "workspace is not 16-byte"), (dict(wsb=64), "workspace of 64 bytes")])
def test_embed_backward(change, frag):
    a = dict(T=4, d=64, V=100, dtype=L.MOE_F32, ids=16, dout=16, scale=1.0, accumulate=0, dw=16, ws=16, wsb=1 << 20)
    a.update(change)
    refused(frag, L.moe_embed_bwd, *a.values())


def test_embed_workspace():
    assert L.moe_embed_workspace_size(0, 8, 8) >= 0
    small, large = L.moe_embed_workspace_size(4096, 64, 1000), L.moe_embed_workspace_size(65536, 4096, 131072)
    assert 4 * 4 * 4096 <= small < large
    with pytest.raises(L.MoEError):
        L.moe_embed_workspace_size(4, 0, 8)


@pytest.mark.parametrize("change,frag", [
    (dict(T=-1), "rows=-1"), (dict(d=64), "multiple of 128"), (dict(d=0), "width 0"), (dict(V=0), "V=0"), (dict(dtype=3), "dtype"),
    (dict(dtype=L.MOE_F32, d=126), "d % 4"), (dict(h=None), "h is NULL"), (dict(h=24), "h is not 16-byte"), (dict(w=None), "w is NULL"),
    (dict(w=20), "w is not 16-byte"), (dict(target=None), "target is NULL"), (dict(target=18), "target is not aligned"),
    (dict(weight=18), "weight is not aligned"), (dict(loss=None), "loss is NULL"), (dict(token=18), "token_loss is not aligned"),
    (dict(dh=None), "dh and dw"), (dict(dw=None), "dh and dw"), (dict(dh=24), "dh is not 16-byte"), (dict(dw=24), "dw is not 16-byte"),
    (dict(ws=None), "workspace is NULL"), (dict(ws=8), "workspace is not 16-byte"), (dict(wsb=1024), "workspace of 1024 bytes")])
def test_vocab_loss(change, frag):
    a = dict(T=4, d=128, V=1000, dtype=L.MOE_BF16, h=16, w=16, target=16, weight=None, loss=16, token=16, dh=16, dw=16, ws=16, wsb=1 << 30)
    a.update(change)
    refused(frag, L.moe_vocab_loss, *a.values())


def test_vocab_loss_workspace():
    """The loss alone keeps statistics; with gradients a piece of the probabilities, whatever the batch."""
    size = L.moe_vocab_loss_workspace_size
    T, d, V = 8192, 1024, 131072
    logits = T * V * 2
    assert size(T, d, V, L.MOE_BF16, False) < logits / 50
    assert size(100 * T, d, V, L.MOE_BF16, False) < logits / 4
    assert 4096 * V * 2 <= size(T, d, V, L.MOE_BF16, True) < logits + 4 * V * d
    assert size(16 * T, d, V, L.MOE_BF16, True) < size(T, d, V, L.MOE_BF16, True) * 1.05
    assert size(T, d, V, L.MOE_F32, True) < 3 * 2 ** 30
    with pytest.raises(L.MoEError):
        size(4, 100, 10, L.MOE_BF16, True)


@pytest.mark.parametrize("change,frag", [
    (dict(groups=-1), "groups=-1"), (dict(rows=0), "rows=0"), (dict(cols=-4), "cols=-4"), (dict(rows=1 << 25), "sides"), (dict(dtype=9), "dtype"),
    (dict(dw=None), "dw is NULL"), (dict(dw=24), "dw is not 16-byte"), (dict(momentum=None), "come together"),
    (dict(momentum_out=None), "come together"), (dict(momentum=20), "momentum is not 16-byte"), (dict(beta=float("nan")), "beta"),
    (dict(nesterov=2), "nesterov"), (dict(counts=18), "group_counts is not aligned"), (dict(steps=0), "steps=0"), (dict(steps=17), "steps=17"),
    (dict(scale=float("inf")), "scale"), (dict(out=None), "out is NULL"), (dict(out=8), "out is not 16-byte"),
    (dict(ws=None), "workspace is NULL"), (dict(ws=8), "workspace is not 16-byte"), (dict(wsb=100), "workspace of 100 bytes")])
def test_orthogonalise(change, frag):
    a = dict(groups=2, rows=64, cols=32, dtype=L.MOE_BF16, dw=16, momentum=16, beta=0.9, nesterov=1, counts=None, steps=5, scale=1.0,
             momentum_out=16, out=16, ws=16, wsb=1 << 30)
    a.update(change)
    refused(frag, L.moe_orthogonalise, *a.values())


def test_orthogonalise_limits():
    refused("groups=257", L.moe_orthogonalise, 257, 8, 8, L.MOE_BF16, 16, None, 0.9, 1, None, 5, 1.0, None, 16, 16, 1 << 30,
            status=L.MOE_ERR_UNSUPPORTED)
    with pytest.raises(L.MoEError):
        L.moe_orthogonalise_workspace_size(2, 0, 8, L.MOE_F32)
    for rows, cols in ((1 << 24, 1), (1, 1 << 24)):  # either side's total is an int32 offset
        assert L.moe_orthogonalise_workspace_size(127, rows, cols, L.MOE_F32) > 0
        with pytest.raises(L.MoEError, match="2\\^31"):
            L.moe_orthogonalise_workspace_size(128, rows, cols, L.MOE_F32)
    n = L.moe_orthogonalise_workspace_size(4, 5632, 1024, L.MOE_BF16)
    assert 6 * 4 * 5632 * 1024 <= n <= 7 * 4 * 5632 * 1024
    L.moe_orthogonalise(0, 8, 8, L.MOE_BF16, None, None, 0.9, 1, None, 5, 1.0, None, None, None, 0, stream=0)
