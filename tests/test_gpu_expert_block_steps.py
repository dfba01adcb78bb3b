"""The gated products, the clipping and the 4-bit products run together as examples/expert_block.py runs them: a training step against the same step of the plain
formulas in 64 bits, and the block in 4 bits against itself with the weights that the 4 bits stand for."""
import os
import sys

import pytest
import torch

from int4_util import unpacked
from test_gpu_expert_block import plain

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def made(dtype, T=90, D=96, F=160, E=5, K=2):
    from expert_block import ExpertBlock
    from paper_2508_18376_amd import moe_block_norm
    block = ExpertBlock(D, F, E, K, T, dtype=dtype, scale=0.5)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy, dh = (torch.randn(T, D, generator=gen, device="cuda").to(dtype) for _ in range(3))
    gate = torch.sigmoid(torch.randn(T, 1, generator=gen, device="cuda")).to(dtype)
    _, h = moe_block_norm(x, branch=torch.zeros_like(x), branch_weight=block.weights["branch_weight"], weight=block.weights["weight"])
    return block, x, h, gate, dy, dh, block.route(h)


@pytest.mark.parametrize("max_norm", [1e-3, 1e6])
def test_a_clipped_step(max_norm):
    """fp32.  The bound is that of the block's gradients in test_gpu_expert_block.py, 1e-4 of the largest value, here of the clipped gradients: their factor is off
    by the norm's error, which is below that of the gradients it is taken over."""
    from paper_2508_18376_amd import moe_clip_grads
    block, x, h, gate, dy, dh, plan = made(torch.float32)
    _, _, saved = block.forward(x, h, gate, plan)
    grads, _, _, _ = block.backward(dy, dh, x, gate, plan, saved)
    names = list(grads)
    clipped, norm = moe_clip_grads([grads[n] for n in names], max_norm, out=[grads[n] for n in names])
    torch.cuda.synchronize()

    cpu = [t.cpu() for t in plan]
    cpu[2] = cpu[2].double()
    leaves = {k: v.cpu().double().requires_grad_() for k, v in dict(block.weights, x=x, h=h).items()}
    y64, h64 = plain(leaves, gate.cpu().double(), cpu, 0.5)
    want = dict(zip(names, torch.autograd.grad((y64, h64), [leaves[n] for n in names], (dy.cpu().double(), dh.cpu().double()))))
    norm64 = torch.sqrt(sum((g ** 2).sum() for g in want.values()))
    assert abs(float(norm) - float(norm64)) <= 1e-4 * float(norm64)
    factor = min(1.0, max_norm / (float(norm64) + 1e-6))
    for name, got in zip(names, clipped):
        ref = want[name] * factor
        assert (got.cpu().double() - ref).abs().max() <= 1e-4 * ref.abs().max(), name


def test_four_bits():
    """fp32: the block with 4-bit weights against the block with the weights that they stand for, 1e-4 of the largest value as above."""
    block, x, h, gate, _, _, plan = made(torch.float32)
    block.quantize4(block=32)
    y4, h4 = block.serve(x, h, gate, plan, bits=4)
    for name, (w, scale, zero) in block.int4.items():
        q, z, s = unpacked(w.cpu(), scale.cpu(), zero.cpu(), block.weights[name].shape[1], 32)
        meant = ((q - z) * s).float().transpose(1, 2).contiguous().to("cuda")
        assert float((meant - block.weights[name]).abs().max()) <= 0.51 * float(scale.max())  # half a step, and a little of the rounded zero point
        block.weights[name] = meant
    y, h_next, _ = block.forward(x, h, gate, plan)
    for got, ref in ((y4, y), (h4, h_next)):
        assert float((got - ref).abs().max()) <= 1e-4 * float(ref.abs().max())


def test_the_step_in_a_graph():
    """Forward, backward and clipping captured once and replayed with other inputs, between eager steps of the same tensors."""
    from paper_2508_18376_amd import moe_clip_grads
    block, x, h, gate, dy, dh, plan = made(torch.bfloat16, D=128, F=256)

    def step(x, h, dy):
        _, _, saved = block.forward(x, h, gate, plan)
        grads, dx, dh_in, _ = block.backward(dy, dh, x, gate, plan, saved)
        return moe_clip_grads(list(grads.values()), 0.1)[0] + [dx, dh_in]

    sx, sh, sdy = x.clone(), h.clone(), dy.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.no_grad(), torch.cuda.graph(graph):
        got = step(sx, sh, sdy)
    for i in range(3):
        sx.copy_(x * (1 + i))
        sdy.copy_(dy if i != 1 else -dy)
        graph.replay()
        torch.cuda.synchronize()
        want = step(sx, sh, sdy)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
