"""CPU: what the weight-by-weight check of the 4-bit products notices, with the mistakes planted in the oracle."""
import pytest
import torch

from int4_single_util import check, places, products, rows_of
from int4_util import random_weights, unpacked
from operator_util import DTYPES, offsets_of

MISTAKES = ["none", "weights rounded", "the last values lost", "the last block lost", "a stage lost", "a scale of the next block", "a zero point of the next block", "halves of bytes swapped"]


@pytest.mark.parametrize("mistake", MISTAKES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("k", [1003, 14336])
def test_planted_mistakes(k, dtype, mistake):
    dt, n, block = DTYPES[dtype], 24, 64
    w, scale, zero = random_weights(1, n, k, block, dt, True, 1)
    at = places(k)
    off = offsets_of([len(at)])
    x, v = rows_of(at, k, dt, 2)
    q, z, s = unpacked(w, scale, zero, k, block)
    weights = (q - z) * s
    if mistake == "weights rounded":
        weights = weights.to(dt).double()
    elif mistake == "the last values lost":
        weights[:, :, -8:] = 0
    elif mistake == "the last block lost":
        weights[:, :, (k - 1) // block * block:] = 0
    elif mistake == "a stage lost":
        weights[:, :, 512:640] = 0
    elif mistake == "a scale of the next block":
        weights = (q - z) * torch.roll(s, -block, 2)
    elif mistake == "a zero point of the next block":
        weights = (q - torch.roll(z, -block, 2)) * s
    elif mistake == "halves of bytes swapped":
        weights = weights[:, :, torch.arange(k) ^ 1 if k % 2 == 0 else (torch.arange(k) ^ 1).clamp_max(k - 1)]
    y = (x.double() @ weights[0].t()).to(dt)
    if mistake == "none":
        check(y, at, v, w, scale, zero, off, k, block)
        ref, _ = products(at, v, w, scale, zero, off, k, block)
        assert torch.allclose(ref, x.double() @ weights[0].t(), rtol=1e-12, atol=0)
    else:
        with pytest.raises(AssertionError):
            check(y, at, v, w, scale, zero, off, k, block)
