"""Limits of the operators around a stack of blocks: refused on the host, before any device work, where 32-bit counters end."""
import os

import pytest

from paper_2506_02965_gb300 import build as _build

if not os.path.exists(_build.LIB) or _build._stale(_build.LIB, os.path.join(_build.CSRC, "moe_abi.cu")):
    _build.build()
from paper_2506_02965_gb300 import _lib as L  # noqa: E402

LOSS_MAX = 2 ** 31 - 1 - 2 ** 18


@pytest.mark.parametrize("V", [LOSS_MAX + 1, 2 ** 31 - 155648, 2 ** 31 - 512, 2 ** 31 - 128, 2 ** 31 - 2])
@pytest.mark.parametrize("dtype,d", [(L.MOE_F32, 4), (L.MOE_BF16, 128)])
def test_vocab_loss_rows_near_32_bits(dtype, d, V):
    """The passes over the vocabulary step past its last row by a grid's rows, in 32 bits."""
    for grads in (16, None):
        with pytest.raises(L.MoEError) as e:
            L.moe_vocab_loss(1, d, V, dtype, 16, 16, 16, None, 16, None, grads, grads, 16, 1 << 60, stream=0)
        assert e.value.status == L.MOE_ERR_UNSUPPORTED and f"V={V}" in str(e.value)
        with pytest.raises(L.MoEError, match=f"V={V}"):
            L.moe_vocab_loss_workspace_size(1, d, V, dtype, grads is not None)


@pytest.mark.parametrize("dtype,d", [(L.MOE_F32, 4), (L.MOE_BF16, 128)])
def test_vocab_loss_largest(dtype, d):
    """The largest vocabulary is taken: what its statistics (and the fp32 logits, 4 bytes a word) come to."""
    n = L.moe_vocab_loss_workspace_size(1, d, LOSS_MAX, dtype, False)
    assert n >= LOSS_MAX * (4 if dtype == L.MOE_F32 else 0) + LOSS_MAX // 512 * 8
    # what the counters may reach: a grid's step of dz, a share of the column statistics, a tile
    for step in (16 * 152 * 64, 512, 256):
        assert LOSS_MAX + step + 63 < 2 ** 31


def test_orthogonalise_elements():
    """A matrix has fewer than 2^40 elements, and the refusal says so."""
    for rows, cols in ((1 << 24, 1 << 16), (1 << 16, 1 << 24), (1 << 20, 1 << 20)):
        with pytest.raises(L.MoEError, match="rows \\* cols < 2\\^40"):
            L.moe_orthogonalise_workspace_size(1, rows, cols, L.MOE_F32)
    assert L.moe_orthogonalise_workspace_size(1, 1 << 20, (1 << 20) - 1, L.MOE_F32) > 1 << 42
