"""Further operators beside the layer, as cases to time: the gated half of a block of experts (both projections, the activation and the product)
with its gradients, products with weights in 4 bits and a scale for each block of them, and the norm over all gradients with clipping.

The plain forms are elementary torch operations in 32 bits.  Layer shapes are the benchmark layers of perf/cases.py (a wide layer of 8 large
experts, a fine-grained one of 64, one with shared experts, a unit-test-sized one) and odd ones.  Activations and output gradients are N(0, 1),
weights N(0, 0.02^2), the gradients that are clipped N(0, 0.001^2); the rows of the experts come from routing random tokens to their Top-K
experts, some of which are more popular than others.
"""
import math

import torch

own = False

TINY = dict(k=128, n=256, groups=8, top_k=2)
WIDE = dict(k=4096, n=14336, groups=8, top_k=2)
FINE = dict(k=2048, n=1024, groups=64, top_k=8)
SHARED = dict(k=2048, n=1408, groups=64, top_k=6)
ODD = dict(k=1001, n=1409, groups=33, top_k=3)

W_STD = 0.02
GRAD_STD = 0.001
EPS = 1e-6
MOST_GATED = 4096 * 2 * 4096 * 14336  # rows * k * n of the largest listed case
MOST_INT4 = 4096 * 4096 * 14336
MOST_CLIPPED = 3 * 8 * 4096 * 14336  # values
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _gated(shape, tokens, train, dtype="bf16", activation="silu", skew=0.5, spare=0, **more):
    return dict(shape, op="gated", tokens=tokens, train=train, dtype=dtype, activation=activation, skew=skew, spare=spare, **more)


def _int4(shape, tokens, block, zeros, dtype="bf16", scale="same", skew=0.5, **more):
    return dict(shape, op="int4", tokens=tokens, block=block, zeros=zeros, dtype=dtype, scale=scale, skew=skew, **more)


def _clip(shape, layers, dtype="bf16", max_norm=1.0, **more):
    return dict(shape, op="clip", layers=layers, dtype=dtype, max_norm=max_norm, **more)


def _dense(k, n):
    return dict(k=k, n=n, groups=0, top_k=1)


def listed():
    return [
        # the smallest training step: the unit-test-sized layer in fp32, where launches are everything
        _gated(TINY, 64, True, "f32", name="gated_tiny_train_f32"),
        # one user's decode step on the fine-grained layer: 8 experts of one row each
        _gated(FINE, 1, False, name="gated_fine_decode_1"),
        # a decode step of 64 users on the wide layer: all weights are read once
        _gated(WIDE, 64, False, name="gated_wide_decode_64"),
        # a training step (forward and all gradients) on the fine-grained layer
        _gated(FINE, 8192, True, name="gated_fine_train_8192"),
        # the same on the wide layer: long contractions, few experts
        _gated(WIDE, 4096, True, name="gated_wide_train_4096"),
        # odd widths in half precision with the other activation, and rows at the end of the buffer that belong to no expert
        _gated(ODD, 1555, True, "f16", "gelu_tanh", spare=37, name="gated_odd_train_f16"),
        # one user's decode step through a dense projection in 4 bits
        _int4(_dense(4096, 14336), 1, 128, False, name="int4_dense_decode_1"),
        # a decode step of 64 users on the wide layer's experts in 4 bits, with zero points and scales in 32 bits
        _int4(WIDE, 64, 128, True, scale="f32", name="int4_wide_decode_64"),
        # a prompt through experts in 4 bits, half precision, small blocks: ragged row lists
        _int4(SHARED, 333, 64, True, "f16", name="int4_grouped_prompt_333"),
        # prefill through the dense projection
        _int4(_dense(4096, 14336), 4096, 128, False, name="int4_dense_prefill_4096"),
        # the gradients of the unit-test-sized layer: launches again
        _clip(TINY, 1, "f32", name="clip_tiny_f32"),
        # the gradients of the wide layer: 1.4 G values, clipped
        _clip(WIDE, 1, name="clip_wide"),
    ]


def draw(rng):
    def spread(lo, hi):  # over the logarithm; odd sizes among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["gated", "gated", "int4", "int4", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "clip":
        k, n = rng.choice([(128, 256), (4096, 14336), (2048, 1024), (2048, 1408), (spread(64, 4096), spread(64, 4096))])
        groups = min(spread(1, 64), 8 if k * n > 1 << 25 else 64)
        layers = spread(1, max(1, min(10, MOST_CLIPPED // (2 if dtype == "f32" else 1) // (3 * groups * k * n + 2 * k + k * groups))))
        return _clip(dict(k=k, n=n, groups=groups, top_k=1), layers, dtype, rng.choice([0.1, 1.0, 10.0]))
    k, n = rng.choice([(128, 256), (4096, 14336), (14336, 4096), (2048, 1024), (1024, 2048), (2048, 1408), (1408, 2048), (spread(64, 4096), spread(64, 4096))])
    groups = min(spread(1, 64), 8 if k * n > 1 << 25 else 64)
    top_k = rng.randint(1, min(8, groups))
    most = (MOST_INT4 if op == "int4" else MOST_GATED) // (8 if dtype == "f32" else 1) // (k * n) // top_k
    shape = dict(k=k, n=n, groups=groups, top_k=top_k)
    tokens = spread(1, max(1, min(8192, most)))
    if op == "int4":
        if rng.random() < 0.5:
            shape = _dense(k, n)
        return _int4(shape, tokens, rng.choice([32, 64, 128, 128, 256]), rng.random() < 0.5, dtype, rng.choice(["same", "f32"]), rng.choice([0.0, 0.5, 1.0]))
    return _gated(shape, tokens, rng.random() < 0.6, dtype, rng.choice(["silu", "silu", "gelu_tanh"]), rng.choice([0.0, 0.5, 1.0]),
                  rng.choice([0, 0, rng.randint(1, 64)]))


def _offsets(case, seed):
    """Where each expert's rows begin: random tokens routed to their Top-K experts."""
    gen = torch.Generator().manual_seed(seed)
    G = case["groups"]
    logits = torch.randn(case["tokens"], G, generator=gen) + case["skew"] * torch.randn(G, generator=gen)
    count = torch.bincount(torch.topk(logits, case["top_k"], dim=1).indices.flatten(), minlength=G)
    return torch.cat([torch.zeros(1, dtype=torch.int64), torch.cumsum(count, 0)])


def _gradients_of(case):
    """(shape, type) of each gradient of a layer: the three weights of its experts, the router's, and the norms' around the block."""
    k, n, G, dt = case["k"], case["n"], case["groups"], DTYPES[case["dtype"]]
    return [((G, k, n), dt), ((G, k, n), dt), ((G, n, k), dt), ((k, G), torch.float32), ((k,), dt), ((k,), dt)]


def _packed(w, block, zeros, scale_type):
    """(two weights a byte, scales, zero points) of w [n][k]: 4 bits a weight, a scale for each block of a row."""
    n, k = w.shape
    B = -(-k // block)
    parts = torch.nn.functional.pad(w, (0, B * block - k)).view(n, B, block)
    if zeros:
        low, high = parts.amin(2).clamp_max(0), parts.amax(2).clamp_min(0)
        scale = ((high - low) / 15).to(scale_type)
        zero = torch.round(-low / scale.float()).clamp(0, 15)
    else:
        scale = (parts.abs().amax(2) / 7).to(scale_type)
        zero = torch.full_like(scale, 8, dtype=torch.float32)
    q = (torch.round(parts / scale.float()[:, :, None]) + zero[:, :, None]).clamp(0, 15).view(n, B * block)[:, :k]
    q = torch.nn.functional.pad(q, (0, k % 2)).to(torch.uint8)
    return q[:, 0::2] | q[:, 1::2] << 4, scale, zero.to(torch.uint8)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32).mul_(std).to(dtype)

    s = {"op": case["op"], "train": case.get("train", False), "dtype": dt}
    if case["op"] == "clip":
        s["grads"] = [normal(*shape, std=GRAD_STD, dtype=dtype) for _ in range(case["layers"]) for shape, dtype in _gradients_of(case)]
        s["clipped"] = [torch.empty_like(g) for g in s["grads"]]
        s["max_norm"] = case["max_norm"]
        return s
    k, n, G = case["k"], case["n"], case["groups"]
    R = case["tokens"] * case["top_k"] + case.get("spare", 0)
    if G:
        off = _offsets(case, seed)
        s["offsets"], s["longest"] = off.to(torch.int32).to(dev), int((off[1:] - off[:-1]).max())
    s["x"] = normal(R, k)
    if case["op"] == "gated":
        s["activation"] = case["activation"]
        s["w1"], s["w3"] = (torch.stack([normal(k, n, std=W_STD) for _ in range(G)]) for _ in range(2))
        if case["train"]:
            s["dh"] = normal(R, n)
        return s
    # 4-bit weights as a program loads them once: a row for each output channel, two weights a byte, rows padded to 16 bytes
    bytes_of, B, scale_type = (k + 1) // 2, -(-k // case["block"]), torch.float32 if case["scale"] == "f32" else dt
    padded = torch.zeros(max(G, 1), n, -(-bytes_of // 16) * 16, dtype=torch.uint8, device=dev)
    s["w_scale"] = torch.empty(max(G, 1), n, B, dtype=scale_type, device=dev)
    s["w_zero"] = torch.empty(max(G, 1), n, B, dtype=torch.uint8, device=dev)
    for g in range(max(G, 1)):
        packed, s["w_scale"][g], s["w_zero"][g] = _packed(normal(n, k, std=W_STD, dtype=torch.float32), case["block"], case["zeros"], scale_type)
        padded[g, :, :bytes_of] = packed
    s["w"], s["block"] = padded[:, :, :bytes_of], case["block"]
    if not case["zeros"]:
        s["w_zero"] = None
    return s


def _rows_of_groups(s):
    """(row of each place [G][longest], whether the place holds one, group of each row, its place there, whether it has one)."""
    off = s["offsets"].long()
    rows = torch.arange(s["x"].shape[0], device=off.device)
    place = torch.arange(max(s["longest"], 1), device=off.device)
    held = place[None, :] < (off[1:] - off[:-1])[:, None]
    row = torch.where(held, off[:-1, None] + place[None, :], torch.zeros_like(held, dtype=torch.long))
    group = (rows[:, None] >= off[None, 1:]).sum(1)
    has = group < off.shape[0] - 1
    group = torch.where(has, group, torch.zeros_like(group))
    at = torch.where(has, rows - off[group], torch.zeros_like(rows))
    return row, held, group, at, has


GELU_C, GELU_A = math.sqrt(2 / math.pi), 0.044715


def _activation(a, kind):
    """(f(a), f'(a))"""
    if kind == "silu":
        sig = torch.sigmoid(a)
        return a * sig, sig * (1 + a * (1 - sig))
    t = torch.tanh(GELU_C * (a + GELU_A * a * a * a))
    return 0.5 * a * (1 + t), 0.5 * (1 + t) + 0.5 * a * (1 - t * t) * GELU_C * (1 + 3 * GELU_A * a * a)


def _plain_gated(s):
    row, held, group, at, has = _rows_of_groups(s)

    def places(t):
        return t[row] * held[:, :, None]

    def back(p):
        return (p[group, at] * has[:, None]).to(s["dtype"])

    x, w1, w3 = places(s["x"].float()), s["w1"].float(), s["w3"].float()
    a, b = torch.bmm(x, w1), torch.bmm(x, w3)
    f, slope = _activation(a, s["activation"])
    out = {"h": back(f * b)}
    if s["train"]:
        dh = places(s["dh"].float())
        da, db = dh * b * slope, dh * f
        xt = x.transpose(1, 2).contiguous()
        out["dx"] = back(torch.bmm(da, w1.transpose(1, 2).contiguous()) + torch.bmm(db, w3.transpose(1, 2).contiguous()))
        out["dw1"], out["dw3"] = torch.bmm(xt, da).to(s["dtype"]), torch.bmm(xt, db).to(s["dtype"])
    return out


def _weights_of(s, like):
    """The weights that the 4-bit ones stand for, [groups][n][k], in the type `like`."""
    k = s["x"].shape[1]
    q = torch.stack([s["w"] & 15, s["w"] >> 4], 3).flatten(2)[:, :, :k]
    block = torch.arange(k, device=q.device) // s["block"]
    zero = 8 if s["w_zero"] is None else s["w_zero"].to(like)[:, :, block]
    return (q.to(like) - zero) * s["w_scale"].to(like)[:, :, block]


def _plain_int4(s):
    x, w = s["x"].float(), _weights_of(s, torch.float32)
    if "offsets" not in s:
        return {"y": torch.matmul(x, w[0].t().contiguous()).to(s["dtype"])}
    row, held, group, at, has = _rows_of_groups(s)
    y = torch.bmm(x[row] * held[:, :, None], w.transpose(1, 2).contiguous())
    return {"y": (y[group, at] * has[:, None]).to(s["dtype"])}


def _plain_clip(s):
    total = torch.zeros((), dtype=torch.float64, device=s["grads"][0].device)
    for g in s["grads"]:
        g = g.float()
        total = total + (g * g).sum(dtype=torch.float64)
    norm = torch.sqrt(total).float()
    factor = torch.clamp(s["max_norm"] / (norm + EPS), max=1.0)
    return {"norm": norm, "grads": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


def _own_gated(s):
    from paper_2508_18376_amd import moe_gated_matmul, moe_gated_matmul_backward
    how = (s["x"], s["w1"], s["w3"])
    if not s["train"]:
        return {"h": moe_gated_matmul(*how, s["offsets"], activation=s["activation"])}
    h, saved = moe_gated_matmul(*how, s["offsets"], activation=s["activation"], want_saved=True)
    return {"h": h, **moe_gated_matmul_backward(s["dh"], *how, saved, s["offsets"], activation=s["activation"])}


def _own_int4(s):
    from paper_2508_18376_amd import moe_int4_matmul
    return {"y": moe_int4_matmul(s["x"], s["w"], s["w_scale"], s["w_zero"], s.get("offsets"), block=s["block"])}


def _own_clip(s):
    from paper_2508_18376_amd import moe_clip_grads
    clipped, norm = moe_clip_grads(s["grads"], s["max_norm"], eps=EPS, out=s["clipped"])
    return {"norm": norm, "grads": clipped}


def run(state):
    if own:
        return {"gated": _own_gated, "int4": _own_int4, "clip": _own_clip}[state["op"]](state)
    return {"gated": _plain_gated, "int4": _plain_int4, "clip": _plain_clip}[state["op"]](state)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "clip":
        sizes = [(math.prod(shape), 4 if dtype == torch.float32 else 2) for shape, dtype in _gradients_of(case)]
        return {"bytes": 2 * case["layers"] * sum(n * b for n, b in sizes) + 4, "flops": 3 * case["layers"] * sum(n for n, _ in sizes)}
    k, n, G = case["k"], case["n"], case["groups"]
    R = case["tokens"] * case["top_k"]
    used = min(max(G, 1), R)  # experts that can have a row
    if case["op"] == "int4":
        B = -(-k // case["block"])
        row = (k + 1) // 2 + B * ((4 if case["scale"] == "f32" else e) + (1 if case["zeros"] else 0))
        return {"bytes": R * (k + n) * e + used * n * row, "flops": 2 * R * k * n}
    out = R + case["spare"]
    if not case["train"]:
        return {"bytes": (R * k + out * n + 2 * used * k * n) * e, "flops": 4 * R * k * n}
    # x, dh and both weights in; h, dx and both weights' gradients out
    return {"bytes": (R * (k + n) + out * (k + n) + 2 * (used + G) * k * n) * e, "flops": 12 * R * k * n}


def _exact_gated(s):
    ends = s["offsets"].tolist()
    x = s["x"].double()
    h = torch.zeros(x.shape[0], s["w1"].shape[2], dtype=torch.float64, device=x.device)
    out = {"h": h}
    if s["train"]:
        out["dx"] = torch.zeros_like(x)
        out["dw1"], out["dw3"] = (torch.zeros(s["w1"].shape, dtype=torch.float64, device=x.device) for _ in range(2))
    for g, (lo, hi) in enumerate(zip(ends[:-1], ends[1:])):
        if hi == lo:
            continue
        leaves = [t.double().requires_grad_() for t in (x[lo:hi], s["w1"][g], s["w3"][g])]
        a = leaves[0] @ leaves[1]
        f = a / (1 + torch.exp(-a)) if s["activation"] == "silu" else a * (1 + torch.tanh(math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3))) / 2
        y = f * (leaves[0] @ leaves[2])
        h[lo:hi] = y.detach()
        if s["train"]:
            out["dx"][lo:hi], out["dw1"][g], out["dw3"][g] = torch.autograd.grad(y, leaves, s["dh"][lo:hi].double())
    return out


def _exact_int4(s):
    x, k = s["x"].double(), s["x"].shape[1]
    ends = s["offsets"].tolist() if "offsets" in s else [0, x.shape[0]]
    y = torch.zeros(x.shape[0], s["w"].shape[1], dtype=torch.float64, device=x.device)
    for g, (lo, hi) in enumerate(zip(ends[:-1], ends[1:])):
        if hi == lo:
            continue
        w = torch.empty(s["w"].shape[1], 2 * s["w"].shape[2], dtype=torch.float64, device=x.device)
        w[:, 0::2], w[:, 1::2] = (s["w"][g] % 16).double(), torch.div(s["w"][g], 16, rounding_mode="floor").double()
        for j in range(s["w_scale"].shape[2]):
            part = w[:, j * s["block"]:min((j + 1) * s["block"], k)]
            part -= 8 if s["w_zero"] is None else s["w_zero"][g, :, j, None].double()
            part *= s["w_scale"][g, :, j, None].double()
        y[lo:hi] = x[lo:hi] @ w[:, :k].t().contiguous()
    return {"y": y}


def _exact_clip(s):
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.flatten(), dtype=torch.float64)) ** 2 for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / (norm + EPS))
    return {"norm": torch.tensor(norm, dtype=torch.float64, device=s["grads"][0].device), "grads": [g.double() * factor for g in s["grads"]]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"gated": _exact_gated, "int4": _exact_int4, "clip": _exact_clip}[s["op"]](s)
