"""A block of experts fine-tuned and served with the operators beside the layer.

    h       = norm in front of the block                                     (the second output of the last block's moe_block_norm)
    rows    = every token once for each of its Top-K experts, sorted by expert (moe_route_and_mask picks them)
    branch  = sum over a token's experts of  g * (Swish(rows W1) * (rows W3)) W2            moe_grouped_matmul, three products
    y, h'   = x + scale * gate * norm(branch), norm(y)                                       moe_block_norm

and the gradients of all of it: moe_block_norm_backward, moe_grouped_matmul with the weights transposed, moe_grouped_matmul_dw.  The elementwise steps
in between are torch's.  `quantize` brings the trained weights to 8 bits, and `serve` runs the block with moe_int8_matmul.

    python examples/expert_block.py        # trains a small block for a few steps on the GPU, then compares it with its 8-bit form
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2508_18376_amd import (DualSparseLayer, moe_block_norm, moe_block_norm_backward, moe_grouped_matmul, moe_grouped_matmul_dw,  # noqa: E402
                                  moe_int8_matmul)


class ExpertBlock:
    """Weights: w1, w3 [E][D][F], w2 [E][F][D], branch_weight, weight [D]."""

    def __init__(self, D, F, E, K, max_tokens, dtype=torch.bfloat16, seed=0, scale=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)

        self.D, self.F, self.E, self.K, self.scale = D, F, E, K, scale
        self.router = torch.randn(D, E, generator=gen, device="cuda") * D ** -0.5
        self.weights = {"w1": normal(E, D, F, std=D ** -0.5), "w3": normal(E, D, F, std=D ** -0.5), "w2": normal(E, F, D, std=F ** -0.5),
                        "branch_weight": torch.ones(D, device="cuda", dtype=dtype), "weight": torch.ones(D, device="cuda", dtype=dtype)}
        # only its routing is used: which experts a token goes to, and with what weight
        self.routing = DualSparseLayer(d_model=D, d_ff=F, n_experts=E, top_k=K, n_part=1, max_tokens=max_tokens, dtype="bf16", renorm_combine=True)
        self.tau = torch.zeros(E, 1, device="cuda")

    def route(self, h):
        """(token of each row, where the experts' rows begin, each row's combine weight, where a token's rows are)."""
        idx, w, _, _ = self.routing.route_and_mask((h.float() @ self.router).contiguous(), self.tau)
        order = torch.argsort(idx.flatten(), stable=True)
        counts = torch.zeros(self.E, dtype=torch.int64, device="cuda").scatter_add_(0, idx.flatten().long(), torch.ones_like(idx.flatten(), dtype=torch.int64))
        offsets = torch.zeros(self.E + 1, dtype=torch.int32, device="cuda")
        offsets[1:] = torch.cumsum(counts, 0)
        place = torch.empty_like(order)
        place[order] = torch.arange(order.shape[0], device="cuda")
        return order // self.K, offsets, w.flatten()[order], place.view(-1, self.K)

    def experts(self, h, plan, products):
        """branch [tokens][D] and what the backward pass takes; products: the three products, on grouped rows."""
        token, offsets, w, place = plan
        rows = h[token]
        a, b = products("w1", rows, offsets), products("w3", rows, offsets)
        act = (torch.nn.functional.silu(a.float()) * b.float()).to(h.dtype)
        out = products("w2", act, offsets)
        branch = (out.float() * w[:, None])[place].sum(1).to(h.dtype)
        return branch, (rows, a, b, act)

    def norms(self, branch, gate):
        return dict(branch=branch, branch_weight=self.weights["branch_weight"], weight=self.weights["weight"], gate=gate, scale=self.scale)

    def forward(self, x, h, gate, plan):
        branch, kept = self.experts(h, plan, lambda name, rows, offsets: moe_grouped_matmul(rows, self.weights[name], offsets))
        y, h_next, stats = moe_block_norm(x, want_stats=True, **self.norms(branch, gate))
        return y, h_next, (branch, stats) + kept

    def backward(self, dy, dh_next, x, gate, plan, saved):
        """Gradients of the weights, of x (through the residual connection), of h and of the gate.  Routing is taken as given."""
        token, offsets, w, place = plan
        branch, stats, rows, a, b, act = saved
        g = moe_block_norm_backward(dy, dh_next, x, stats, **self.norms(branch, gate))
        dout = (g["dbranch"][token].float() * w[:, None]).to(x.dtype)
        grads = {"branch_weight": g["dbranch_weight"], "weight": g["dweight"], "w2": moe_grouped_matmul_dw(act, dout, offsets)}
        dact = moe_grouped_matmul(dout, self.weights["w2"], offsets, w_transposed=True).float()
        s = torch.sigmoid(a.float())
        da = (dact * b.float() * s * (1 + a.float() * (1 - s))).to(x.dtype)
        db = (dact * a.float() * s).to(x.dtype)
        grads["w1"], grads["w3"] = moe_grouped_matmul_dw(rows, da, offsets), moe_grouped_matmul_dw(rows, db, offsets)
        drows = (moe_grouped_matmul(da, self.weights["w1"], offsets, w_transposed=True).float()
                 + moe_grouped_matmul(db, self.weights["w3"], offsets, w_transposed=True).float())
        return grads, g["dx"], drows[place].sum(1).to(x.dtype), g.get("dgate")

    def quantize(self):
        """8-bit weights [E][out][in] with a scale for each output channel, rows padded to 16 bytes."""
        self.int8 = {}
        for name in ("w1", "w3", "w2"):
            w = self.weights[name].float().transpose(1, 2)
            scale = (w.abs().amax(2) / 127).clamp_min(1e-30)
            padded = torch.zeros(w.shape[0], w.shape[1], -(-w.shape[2] // 16) * 16, dtype=torch.int8, device="cuda")
            padded[:, :, :w.shape[2]] = torch.round(w / scale[:, :, None]).to(torch.int8)
            self.int8[name] = padded[:, :, :w.shape[2]], scale

    def serve(self, x, h, gate, plan):
        branch, _ = self.experts(h, plan, lambda name, rows, offsets: moe_int8_matmul(rows, *self.int8[name], offsets))
        return moe_block_norm(x, **self.norms(branch, gate))


def main(steps=20, tokens=512, D=256, F=512, E=8, K=2):
    gen = torch.Generator(device="cuda").manual_seed(1)
    block = ExpertBlock(D, F, E, K, tokens)
    x = torch.randn(tokens, D, generator=gen, device="cuda").bfloat16()
    target = torch.randn(tokens, D, generator=gen, device="cuda")
    gate = torch.sigmoid(torch.randn(tokens, 1, generator=gen, device="cuda")).bfloat16()
    _, h = moe_block_norm(x, branch=torch.zeros_like(x), branch_weight=block.weights["branch_weight"], weight=block.weights["weight"])
    plan = block.route(h)
    losses = []
    for _ in range(steps):
        y, h_next, saved = block.forward(x, h, gate, plan)
        err = h_next.float() - target
        losses.append(float((err ** 2).mean()))
        dh = (2 * err / err.numel()).to(x.dtype)
        grads, _, _, _ = block.backward(torch.zeros_like(x), dh, x, gate, plan, saved)
        for name, g in grads.items():
            block.weights[name] -= (40.0 * g.float()).to(x.dtype)
    block.quantize()
    y8, h8 = block.serve(x, h, gate, plan)
    y, h_next, _ = block.forward(x, h, gate, plan)
    rel = float((h8.float() - h_next.float()).norm() / h_next.float().norm())
    print("loss %.4f -> %.4f over %d steps; 8-bit block differs by %.4f of the output" % (losses[0], losses[-1], steps, rel))
    return losses, rel


if __name__ == "__main__":
    main()
