"""A block of experts fine-tuned and served with the operators beside the layer.

    h       = norm in front of the block                                     (the second output of the last block's moe_block_norm)
    rows    = every token once for each of its Top-K experts, sorted by expert (moe_route_and_mask picks them)
    branch  = sum over a token's experts of  g * (Swish(rows W1) * (rows W3)) W2            moe_gated_matmul, moe_grouped_matmul
    y, h'   = x + scale * gate * norm(branch), norm(y)                                       moe_block_norm

and the gradients of all of it: moe_block_norm_backward, moe_grouped_matmul with the weights transposed, moe_grouped_matmul_dw, moe_gated_matmul_backward,
clipped by their norm (moe_clip_grads).  The elementwise steps in between are torch's.  `quantize` brings the trained weights to 8 bits or 4, and
`serve` runs the block with moe_int8_matmul or moe_int4_matmul.

    python examples/expert_block.py        # trains a small block for a few steps on the GPU, then compares it with its 8-bit and 4-bit forms
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2508_18376_amd import (DualSparseLayer, moe_block_norm, moe_block_norm_backward, moe_clip_grads, moe_gated_matmul,  # noqa: E402
                                  moe_gated_matmul_backward, moe_grouped_matmul, moe_grouped_matmul_dw, moe_int4_matmul, moe_int8_matmul)


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

    def combine(self, out, plan, dtype):
        """branch [tokens][D]: each token's rows of the experts' outputs, weighted."""
        _, _, w, place = plan
        return (out.float() * w[:, None])[place].sum(1).to(dtype)

    def norms(self, branch, gate):
        return dict(branch=branch, branch_weight=self.weights["branch_weight"], weight=self.weights["weight"], gate=gate, scale=self.scale)

    def forward(self, x, h, gate, plan):
        token, offsets, _, _ = plan
        rows = h[token]
        act, both = moe_gated_matmul(rows, self.weights["w1"], self.weights["w3"], offsets, want_saved=True)
        branch = self.combine(moe_grouped_matmul(act, self.weights["w2"], offsets), plan, h.dtype)
        y, h_next, stats = moe_block_norm(x, want_stats=True, **self.norms(branch, gate))
        return y, h_next, (branch, stats, rows, act, both)

    def backward(self, dy, dh_next, x, gate, plan, saved):
        """Gradients of the weights, of x (through the residual connection), of h and of the gate.  Routing is taken as given."""
        token, offsets, w, place = plan
        branch, stats, rows, act, both = saved
        g = moe_block_norm_backward(dy, dh_next, x, stats, **self.norms(branch, gate))
        dout = (g["dbranch"][token].float() * w[:, None]).to(x.dtype)
        dact = moe_grouped_matmul(dout, self.weights["w2"], offsets, w_transposed=True)
        half = moe_gated_matmul_backward(dact, rows, self.weights["w1"], self.weights["w3"], both, offsets)
        grads = {"branch_weight": g["dbranch_weight"], "weight": g["dweight"], "w2": moe_grouped_matmul_dw(act, dout, offsets), "w1": half["dw1"], "w3": half["dw3"]}
        return grads, g["dx"], half["dx"].float()[place].sum(1).to(x.dtype), g.get("dgate")

    def quantize(self):
        """8-bit weights [E][out][in] with a scale for each output channel, rows padded to 16 bytes."""
        self.int8 = {}
        for name in ("w1", "w3", "w2"):
            w = self.weights[name].float().transpose(1, 2)
            scale = (w.abs().amax(2) / 127).clamp_min(1e-30)
            padded = torch.zeros(w.shape[0], w.shape[1], -(-w.shape[2] // 16) * 16, dtype=torch.int8, device="cuda")
            padded[:, :, :w.shape[2]] = torch.round(w / scale[:, :, None]).to(torch.int8)
            self.int8[name] = padded[:, :, :w.shape[2]], scale

    def quantize4(self, block=64):
        """4-bit weights [E][out][in / 2] with a scale and a zero point for each block of an output channel's weights."""
        self.int4, self.block = {}, block
        for name in ("w1", "w3", "w2"):
            w = self.weights[name].float().transpose(1, 2)
            parts = torch.nn.functional.pad(w, (0, -w.shape[2] % block)).unflatten(2, (-1, block))
            low, high = parts.amin(3).clamp_max(0), parts.amax(3).clamp_min(0)
            scale = ((high - low) / 15).clamp_min(1e-30)
            zero = torch.round(-low / scale)
            q = (torch.round(parts / scale[..., None]) + zero[..., None]).clamp(0, 15).flatten(2).to(torch.uint8)
            self.int4[name] = (q[:, :, 0::2] | q[:, :, 1::2] << 4)[:, :, :(w.shape[2] + 1) // 2].contiguous(), scale.contiguous(), zero.to(torch.uint8).contiguous()

    def serve(self, x, h, gate, plan, bits=8):
        token, offsets, _, _ = plan

        def product(name, rows):
            if bits == 4:
                return moe_int4_matmul(rows, *self.int4[name], offsets, block=self.block)
            return moe_int8_matmul(rows, *self.int8[name], offsets)

        rows = h[token]
        act = (torch.nn.functional.silu(product("w1", rows).float()) * product("w3", rows).float()).to(h.dtype)
        return moe_block_norm(x, **self.norms(self.combine(product("w2", act), plan, h.dtype), gate))


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
        grads = dict(zip(grads, moe_clip_grads(list(grads.values()), max_norm=1.0)[0]))
        for name, g in grads.items():
            block.weights[name] -= (40.0 * g.float()).to(x.dtype)
    block.quantize()
    block.quantize4()
    y, h_next, _ = block.forward(x, h, gate, plan)
    rel, rel4 = (float((block.serve(x, h, gate, plan, bits)[1].float() - h_next.float()).norm() / h_next.float().norm()) for bits in (8, 4))
    print("loss %.4f -> %.4f over %d steps; the 8-bit block differs by %.4f of the output, the 4-bit one by %.4f" % (losses[0], losses[-1], steps, rel, rel4))
    return losses, rel


if __name__ == "__main__":
    main()
