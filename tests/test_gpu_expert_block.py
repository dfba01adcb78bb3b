"""The operators run together as examples/expert_block.py runs them: its gradients against automatic differentiation of the plain formulas in 64 bits,
its training step, and its 8-bit form."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def plain(leaves, gate, plan, scale):
    x, h, w1, w3, w2, wb, w = (leaves[k] for k in ("x", "h", "w1", "w3", "w2", "branch_weight", "weight"))
    token, offsets, g, place = plan
    rows, ends = h[token], offsets.tolist()
    parts = []
    for e, (lo, hi) in enumerate(zip(ends[:-1], ends[1:])):
        r = rows[lo:hi]
        parts.append((torch.nn.functional.silu(r @ w1[e]) * (r @ w3[e])) @ w2[e])
    branch = (torch.cat(parts) * g[:, None])[place].sum(1)

    def norm(v, weight):
        return v / torch.sqrt((v ** 2).mean(1, keepdim=True) + 1e-6) * weight

    y = x + scale * gate * norm(branch, wb)
    return y, norm(y, w)


def test_gradients_and_outputs():
    """fp32, so that what is off is the products' rounding.  The bound is chosen, not derived: 1e-4 of the largest value is 1700 half steps of
    fp32.  One product of 160 terms may be off by 2 * 162 half steps of its terms' magnitudes (see operator_util.product_error), which are some ten times its
    typical value and three times its largest, so the bound is near what two products can do at worst, and far from what a wrong formula does.  The
    operators by themselves are held to derived bounds in their own tests."""
    from expert_block import ExpertBlock
    from paper_2508_18376_amd import moe_block_norm
    T, D, F, E, K = 90, 96, 160, 5, 2
    block = ExpertBlock(D, F, E, K, T, dtype=torch.float32, scale=0.5)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy, dh = (torch.randn(T, D, generator=gen, device="cuda") for _ in range(3))
    gate = torch.sigmoid(torch.randn(T, 1, generator=gen, device="cuda"))
    _, h = moe_block_norm(x, branch=torch.zeros_like(x), branch_weight=block.weights["branch_weight"], weight=block.weights["weight"])
    plan = block.route(h)
    y, h_next, saved = block.forward(x, h, gate, plan)
    grads, dx, dh_in, dgate = block.backward(dy, dh, x, gate, plan, saved)
    torch.cuda.synchronize()

    cpu = [t.cpu() for t in plan]
    cpu[2] = cpu[2].double()
    leaves = {k: v.cpu().double().requires_grad_() for k, v in dict(block.weights, x=x, h=h).items()}
    gate64 = gate.cpu().double().requires_grad_()
    y64, h64 = plain(leaves, gate64, cpu, 0.5)
    want = dict(zip(list(leaves) + ["gate"], torch.autograd.grad((y64, h64), list(leaves.values()) + [gate64], (dy.cpu().double(), dh.cpu().double()))))
    got = dict(grads, x=dx, h=dh_in, gate=dgate)
    assert set(got) == set(want)
    for name, ref in list(want.items()) + [("y", y64.detach()), ("h_next", h64.detach())]:
        out = {"y": y, "h_next": h_next}.get(name, got.get(name)).cpu().double()
        assert (out - ref).abs().max() <= 1e-4 * ref.abs().max(), name


def test_training_and_eight_bits():
    import expert_block
    losses, rel = expert_block.main(steps=12)
    assert all(b < a for a, b in zip(losses, losses[1:])), losses
    # chosen, not derived: a value is rounded by up to 1 / 254 of its row's largest, so by about 0.7 % of the row's rms (3 sigma / 254 / sqrt(3)); two operands,
    # three products in all, of which two side by side: 0.7 % * sqrt(2 * 2) and the bf16 steps between
    assert rel < 0.02
