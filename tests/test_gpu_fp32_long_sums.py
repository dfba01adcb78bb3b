"""Sums of very many fp32 products: no less exact than sums in parts are.

A sum's partial sums grow like a random walk, so that a chain of S steps has a relative error of sqrt(S / 2) roundings.  The matrix instructions add two products
a step: a chain of N products has N / 2 steps; in parts of 512, each has 256, and the sum over the parts N / 512.  A rounding is half a step, 2^-24, at most;
the matrix instructions may cut off instead, which counts twice."""
import math

import pytest
import torch

from int4_util import random_weights, unpacked
from operator_util import U32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def most(n):
    return 2 * U32 * (math.sqrt(256 / 2) + math.sqrt(n / 512 / 2))


def rel(got, want):
    return float((got.cpu().double() - want).norm() / want.norm())


@pytest.mark.parametrize("rows,k,n", [(3, 57344, 136), (300, 57344, 136), (40, 57343, 77)])
def test_products_with_weights_in_4_bits(rows, k, n):
    """The weights are (q - z) s, of two more roundings each, which do not add up: 2 half steps."""
    from paper_2508_18376_amd import moe_int4_matmul
    x = torch.randn(rows, k, generator=torch.Generator().manual_seed(1))
    w, scale, zero = random_weights(1, n, k, 128, torch.float32, True, 2)
    y = moe_int4_matmul(*(t.to(DEV) for t in (x, w, scale, zero)), block=128)
    q, z, s = unpacked(w, scale, zero, k, 128)
    assert rel(y, x.double() @ ((q - z) * s)[0].t()) <= most(k) + 2 * U32
