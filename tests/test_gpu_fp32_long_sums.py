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


def normal(seed, *shape, std=1.0):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV) * std


def gated_tensors(rows, k, n):
    """x, w1, w3, dh: weights so that the products are of order one."""
    return normal(3, rows, k), normal(4, 1, k, n, std=k ** -0.5), normal(5, 1, k, n, std=k ** -0.5), normal(6, rows, n)


def slopes(dh, saved):
    """da and db in 64 bits, of Swish."""
    a, b = saved.double()
    s = torch.sigmoid(a)
    return dh.double() * b * (s + a * s * (1 - s)), dh.double() * a * s


# The kernels' da and db have errors of their own, which do not add up: a few roundings, and exp's argument |z| of order one: 16 half steps
SLOPES = 16 * U32


def test_gated_products():
    from paper_2508_18376_amd import moe_gated_matmul
    x, w1, w3, _ = gated_tensors(4096, 30000, 1280)
    _, saved = moe_gated_matmul(x, w1, w3, want_saved=True)
    for got, w in zip(saved, (w1, w3)):
        assert rel(got, (x.double() @ w[0].double()).cpu()) <= most(30000)


@pytest.mark.parametrize("rows,k,n", [(4096, 1280, 30000), (60000, 64, 72), (60001, 61, 77)])
def test_gated_gradients(rows, k, n):
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    x, w1, w3, dh = gated_tensors(rows, k, n)
    _, saved = moe_gated_matmul(x, w1, w3, want_saved=True)
    got = moe_gated_matmul_backward(dh, x, w1, w3, saved)
    da, db = slopes(dh, saved)
    assert rel(got["dx"], (da @ w1[0].double().t() + db @ w3[0].double().t()).cpu()) <= most(2 * n) + SLOPES
    for name, d in (("dw1", da), ("dw3", db)):
        assert rel(got[name][0], (x.double().t() @ d).cpu()) <= most(rows) + SLOPES, name
