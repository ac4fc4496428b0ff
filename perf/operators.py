"""Performance cases of the training operators, with their plain forms and their definitions in 64 bits.

Three operators make one training step of a pre-norm MLP block:

* ``mlp``: the two-layer MLP ``Y = act(X @ W1) @ W2`` (SwiGLU with ``W1`` =
  ``[2, H, F]``, or GELU / identity with ``[H, F]``).  ``fwd`` also returns the
  pre-activations ``P = X @ W1`` that training keeps; ``bwd`` returns ``dX``,
  ``dW1`` and ``dW2`` from ``dY`` and that ``P``.
* ``norm``: layer norm in front of it.  ``fwd`` returns ``Y`` and the rows' mean
  and 1 / standard deviation; ``bwd`` returns ``dX`` and the gradients of weight
  and bias.
* ``ortho``: the weights' update, a stack of matrices orthogonalised by
  Newton-Schulz products: ``X <- a X + (b A + c A A) X`` with ``A = X X^T``,
  five times, from ``X = G / |G|``.

Every case is a dict of plain values: ``op`` and ``dir``, the sizes, and the
types.  ``own`` (set by whoever runs the file) chooses between the plain forms,
elementary torch operations in 32 bits rounded once at the end, and the
library's kernels through ``binding``.
"""
import math

import torch

own = False

EPS = 1e-5  # layer norm
ORTHO_EPS = 1e-7
ORTHO_STEPS = 5
ORTHO_COEFFS = (3.4445, -4.7750, 2.0315)

# The most that a drawn case may cost: the backward pass of 4096 rows through an
# 8B model's gated MLP (bytes: a layer norm over 32768 rows of 8192).
MOST_FLOPS = 12 * 4096.0 * 4096 * 14336
MOST_BYTES = 1.7e9

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _mlp(name, direction, M, H, F, act="swiglu"):
    return {"name": name, "op": "mlp", "dir": direction, "M": M, "H": H, "F": F, "act": act}


def _norm(name, direction, M, H, x="bf16", y="bf16", pad=0):
    return {"name": name, "op": "norm", "dir": direction, "M": M, "H": H, "x": x, "y": y, "pad": pad}


def _ortho(name, count, rows, cols, x="f32"):
    return {"name": name, "op": "ortho", "count": count, "rows": rows, "cols": cols, "x": x}


def listed():
    return [
        # the smallest layer of the benchmark: launches and latencies
        _mlp("mlp_bwd_64x512x2048", "bwd", 64, 512, 2048),
        # few tokens (an expert's share, a short fine-tuning batch) through an 8B layer: the weights' traffic
        _mlp("mlp_fwd_24x4096x14336", "fwd", 24, 4096, 14336),
        # a ragged batch through widths that are multiples of 64 only, without gate
        _mlp("mlp_bwd_777x2112x5440_gelu", "bwd", 777, 2112, 5440, "gelu_tanh"),
        # a micro-batch of 2048 tokens through an 8B model's gated MLP, both directions
        _mlp("mlp_fwd_2048x4096x14336", "fwd", 2048, 4096, 14336),
        _mlp("mlp_bwd_2048x4096x14336", "bwd", 2048, 4096, 14336),
        # the largest: 4096 tokens through the same layer
        _mlp("mlp_bwd_4096x4096x14336", "bwd", 4096, 4096, 14336),
        # one token of one sequence in front of an 8B layer
        _norm("norm_fwd_1x4096", "fwd", 1, 4096),
        # 16384 tokens of a 32-bit residual stream of a 70B layer, normalised to bf16
        _norm("norm_fwd_16384x8192_f32", "fwd", 16384, 8192, "f32", "bf16"),
        # a ragged batch of rows out of a wider buffer, odd width
        _norm("norm_bwd_777x2111_pad", "bwd", 777, 2111, pad=65),
        # a micro-batch of 8192 tokens, backward, with the reduction of the weight's gradient
        _norm("norm_bwd_8192x4096", "bwd", 8192, 4096),
        # both halves of a small gated layer's first weight
        _ortho("ortho_2x512x2048", 2, 512, 2048),
        # the second weight of an 8B layer
        _ortho("ortho_14336x4096", 1, 14336, 4096, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["mlp", "mlp", "norm", "ortho"])
        if op == "mlp":
            H, F = 64 * _log_int(rng, 4, 128), 64 * _log_int(rng, 8, 448)
            if rng.random() < 0.5:  # most models' widths are multiples of 256
                H, F = -(-H // 256) * 256, -(-F // 256) * 256
            c = _mlp("", rng.choice(["fwd", "bwd", "bwd"]), _log_int(rng, 1, 8192), H, F,
                     rng.choice(["swiglu", "swiglu", "gelu_tanh", "identity"]))
        elif op == "norm":
            x, y = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
            H = _log_int(rng, 16, 16384)
            if rng.random() < 0.6:
                H = -(-H // 64) * 64
            c = _norm("", rng.choice(["fwd", "bwd"]), _log_int(rng, 1, 32768), H, x, y,
                      rng.choice([0, 0, 64, rng.randint(1, 200)]))
        else:
            rows, cols = _log_int(rng, 16, 8192), _log_int(rng, 16, 16384)
            if rng.random() < 0.5:
                rows, cols = -(-rows // 64) * 64, -(-cols // 64) * 64
            if rng.random() < 0.3:
                rows, cols = cols, rows
            c = _ortho("", rng.randint(1, 4), rows, cols, rng.choice(["f32", "bf16"]))
        del c["name"]
        w = work(c)
        if 3072 not in c.values() and w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c  # (no workload of this library is 3072 wide)


# ------------------------------------------------------------------ inputs


def _gates(case):
    return 2 if case["act"] == "swiglu" else 1


def _inputs(case, seed):
    """The tensors a user's program holds before the call, made on the GPU from the seed."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(shape, std=1.0, dtype=torch.bfloat16):
        return torch.randn(shape, generator=gen, dtype=torch.float32, device="cuda").mul_(std).to(dtype)

    if case["op"] == "mlp":
        M, H, F, nb = case["M"], case["H"], case["F"], _gates(case)
        t = {"X": normal((M, H)), "W1": normal((nb, H, F), H**-0.5), "W2": normal((F, H), F**-0.5)}
        if case["dir"] == "bwd":
            # what the forward pass kept: the pre-activations, rounded to bf16
            t["P"] = torch.matmul(t["X"].float(), t["W1"].float()).to(torch.bfloat16)
            t["dY"] = normal((M, H), 1e-2)
        return t
    if case["op"] == "norm":
        # activations with an offset for each row and channels of their own size, a few of them large
        M, H, wide = case["M"], case["H"], case["H"] + case["pad"]
        size = torch.exp(0.5 * torch.randn(wide, generator=gen, device="cuda"))
        size[:: 97] *= 20.0
        X = torch.randn((M, wide), generator=gen, device="cuda").mul_(size)
        X += 0.5 * torch.randn((M, 1), generator=gen, device="cuda")
        t = {"X": X.to(TYPES[case["x"]])[:, :H], "w": 1.0 + normal((H,), 0.1, torch.float32), "b": normal((H,), 0.1, torch.float32)}
        if case["dir"] == "bwd":
            x = t["X"].float()
            var, mean = torch.var_mean(x, dim=1, correction=0)
            t["mean"], t["rstd"] = mean, torch.rsqrt(var + EPS)
            t["dY"] = normal((M, wide), 1e-2, TYPES[case["y"]])[:, :H]
        return t
    # a gradient's spectrum: a few strong directions over a floor of noise
    n, r, c = case["count"], case["rows"], case["cols"]
    k = min(32, r, c)
    left, right = normal((n, r, k), 1.0, torch.float32), normal((n, k, c), 1.0, torch.float32)
    G = torch.matmul(left * torch.logspace(0, -2, k, device="cuda"), right)
    G += normal((n, r, c), 0.1, torch.float32)
    return {"G": (1e-3 * G).to(TYPES[case["x"]])}


def prepare(case, seed):
    """The inputs, and with the library's kernels the plan and the output buffers of this shape."""
    t = _inputs(case, seed)
    state = {"case": case, "t": t}
    if not own:
        return state
    from paper_2607_07862_amd import binding as B

    new = torch.empty_like
    if case["op"] == "mlp":
        M, H, F = case["M"], case["H"], case["F"]
        act = {"identity": B.ACT_IDENTITY, "gelu_tanh": B.ACT_GELU_TANH, "swiglu": B.ACT_SWIGLU}[case["act"]]
        state["plan"] = B.TrainPlan(M, H, F, act)
        if case["dir"] == "fwd":
            P = torch.empty((_gates(case), M, F), dtype=torch.bfloat16, device="cuda")
            state["out"] = {"P": P, "Y": new(t["X"])}
        else:
            state["out"] = {"dX": new(t["X"]), "dW1": new(t["W1"]), "dW2": new(t["W2"])}
    elif case["op"] == "norm":
        M, H, x, y = case["M"], case["H"], TYPES[case["x"]], TYPES[case["y"]]
        state["plan"] = B.NormPlan(M, H, x, y)
        if case["dir"] == "fwd":
            state["out"] = {"Y": torch.empty((M, H), dtype=y, device="cuda"),
                            "mean": torch.empty(M, device="cuda"), "rstd": torch.empty(M, device="cuda")}
        else:
            state["out"] = {"dX": torch.empty((M, H), dtype=x, device="cuda"), "dw": new(t["w"]), "db": new(t["b"])}
    else:
        state["plan"] = B.OrthoPlan(case["count"], case["rows"], case["cols"], TYPES[case["x"]])
        state["out"] = {"O": torch.empty(t["G"].shape, dtype=torch.bfloat16, device="cuda")}
    return state


# ------------------------------------------------------------------ one pass


def run(state):
    case, t = state["case"], state["t"]
    if not own:
        return {"mlp_fwd": _plain_mlp_fwd, "mlp_bwd": _plain_mlp_bwd, "norm_fwd": _plain_norm_fwd,
                "norm_bwd": _plain_norm_bwd, "ortho": _plain_ortho}[_key(case)](case, t)
    plan, out = state["plan"], state["out"]
    key = _key(case)
    if key == "mlp_fwd":
        plan.forward(t["X"], t["W1"], t["W2"], out["P"], out["Y"])
    elif key == "mlp_bwd":
        plan.backward(t["dY"], t["X"], t["W1"], t["W2"], t["P"], out["dX"], out["dW1"], out["dW2"])
    elif key == "norm_fwd":
        plan.forward(t["X"], t["w"], t["b"], out["Y"], out["mean"], out["rstd"], eps=EPS)
    elif key == "norm_bwd":
        plan.backward(t["dY"], t["X"], t["w"], t["mean"], t["rstd"], out["dX"], out["dw"], out["db"])
    else:
        plan.run(t["G"], out["O"], steps=ORTHO_STEPS, coeffs=ORTHO_COEFFS, eps=ORTHO_EPS)
    return out


def _key(case):
    return case["op"] if case["op"] == "ortho" else case["op"] + "_" + case["dir"]


_GELU_C = math.sqrt(2.0 / math.pi)


def _plain_mlp_fwd(case, t):
    P = torch.matmul(t["X"].float(), t["W1"].float())
    if case["act"] == "swiglu":
        Z = P[0] / (1.0 + torch.exp(-P[0])) * P[1]
    elif case["act"] == "gelu_tanh":
        Z = 0.5 * P[0] * (1.0 + torch.tanh(_GELU_C * (P[0] + 0.044715 * P[0] ** 3)))
    else:
        Z = P[0]
    return {"P": P.to(torch.bfloat16), "Y": torch.matmul(Z, t["W2"].float()).to(torch.bfloat16)}


def _plain_mlp_bwd(case, t):
    X, W1, W2, P, dY = (t[k].float() for k in ("X", "W1", "W2", "P", "dY"))
    dZ = torch.matmul(dY, W2.t())
    if case["act"] == "swiglu":
        s = 1.0 / (1.0 + torch.exp(-P[0]))
        Z = P[0] * s * P[1]
        dP = torch.stack([dZ * P[1] * s * (1.0 + P[0] * (1.0 - s)), dZ * P[0] * s])
    elif case["act"] == "gelu_tanh":
        h = torch.tanh(_GELU_C * (P[0] + 0.044715 * P[0] ** 3))
        Z = 0.5 * P[0] * (1.0 + h)
        slope = _GELU_C * (1.0 + 3 * 0.044715 * P[0] ** 2)
        dP = (dZ * (0.5 * (1.0 + h) + 0.5 * P[0] * (1.0 - h * h) * slope)).unsqueeze(0)
    else:
        Z, dP = P[0], dZ.unsqueeze(0)
    dX = torch.matmul(dP[0], W1[0].t())
    if case["act"] == "swiglu":
        dX += torch.matmul(dP[1], W1[1].t())
    dW1 = torch.matmul(X.t(), dP)
    return {k: v.to(torch.bfloat16) for k, v in (("dX", dX), ("dW1", dW1), ("dW2", torch.matmul(Z.t(), dY)))}


def _plain_norm_fwd(case, t):
    x = t["X"].float()
    mean = x.mean(dim=1)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(dim=1) + EPS)
    return {"Y": (d * rstd[:, None] * t["w"] + t["b"]).to(TYPES[case["y"]]), "mean": mean, "rstd": rstd}


def _plain_norm_bwd(case, t):
    dy = t["dY"].float()
    xhat = (t["X"].float() - t["mean"][:, None]) * t["rstd"][:, None]
    g = dy * t["w"]
    dx = t["rstd"][:, None] * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    return {"dX": dx.to(TYPES[case["x"]]), "dw": (dy * xhat).sum(dim=0), "db": dy.sum(dim=0)}


def _plain_ortho_step(X):
    a, b, c = ORTHO_COEFFS
    A = torch.matmul(X, X.transpose(1, 2).contiguous())
    return a * X + torch.matmul(b * A + c * torch.matmul(A, A), X)


def _plain_ortho(case, t):
    X = t["G"].float()
    tall = case["rows"] > case["cols"]
    if tall:
        X = X.transpose(1, 2).contiguous()
    X = X / (torch.sqrt((X * X).sum(dim=(1, 2), keepdim=True)) + ORTHO_EPS)
    X = _plain_ortho_step(_plain_ortho_step(_plain_ortho_step(_plain_ortho_step(_plain_ortho_step(X)))))
    return {"O": (X.transpose(1, 2).contiguous() if tall else X).to(torch.bfloat16)}


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    """Bytes: every input read and every output written once.  Operations: two for each multiply-add; a
    symmetric product counts once for each pair."""
    if case["op"] == "mlp":
        M, H, F, nb = case["M"], case["H"], case["F"], _gates(case)
        weights = (nb + 1) * H * F
        if case["dir"] == "fwd":
            return {"bytes": 2.0 * (weights + 2 * M * H + nb * M * F), "flops": 2.0 * M * weights}
        return {"bytes": 2.0 * (2 * weights + 3 * M * H + nb * M * F), "flops": 4.0 * M * weights}
    if case["op"] == "norm":
        M, H = case["M"], case["H"]
        x, y = (4 if case[k] == "f32" else 2 for k in ("x", "y"))
        if case["dir"] == "fwd":
            return {"bytes": 1.0 * M * H * (x + y) + 8 * (H + M), "flops": 8.0 * M * H}
        return {"bytes": 1.0 * M * H * (2 * x + y) + 8 * M + 12 * H, "flops": 14.0 * M * H}
    n, m = sorted((case["rows"], case["cols"]))
    size = (4 if case["x"] == "f32" else 2) + 2
    per_step = 1.0 * n * n * m + 1.0 * n**3 + 2.0 * n * n * m
    return {"bytes": 1.0 * case["count"] * n * m * size, "flops": case["count"] * ORTHO_STEPS * per_step}


# ------------------------------------------------------------------ the definitions in 64 bits


def _exact_act(act, p):
    """act and its partial derivatives at the pre-activations p[0] (and p[1])."""
    if act == "identity":
        return p[0], [torch.ones_like(p[0])]
    if act == "swiglu":
        sig = torch.sigmoid(p[0])
        silu = p[0] * sig
        return silu * p[1], [p[1] * (sig + silu * (1 - sig)), silu]
    k = (2 / math.pi) ** 0.5
    # 0.5 (1 + tanh(u)) = sigmoid(2 u)
    u = k * (p[0] + 0.044715 * p[0].pow(3))
    s = torch.sigmoid(2 * u)
    return p[0] * s, [s + p[0] * 2 * s * (1 - s) * k * (1 + 0.134145 * p[0].pow(2))]


def exact(case, seed):
    t = {k: v.double() for k, v in _inputs(case, seed).items()}
    if case["op"] == "mlp":
        nb = _gates(case)
        if case["dir"] == "fwd":
            P = [t["X"].mm(t["W1"][i]) for i in range(nb)]
            return {"P": torch.stack(P), "Y": _exact_act(case["act"], P)[0].mm(t["W2"])}
        Z, slopes = _exact_act(case["act"], t["P"])
        dZ = (t["W2"].mm(t["dY"].t())).t()
        dP = [dZ * s for s in slopes]
        dX = sum(t["W1"][i].mm(dP[i].t()) for i in range(nb)).t().contiguous()
        dW1 = torch.stack([t["X"].t().mm(dP[i]) for i in range(nb)])
        return {"dX": dX, "dW1": dW1, "dW2": Z.t().mm(t["dY"])}
    if case["op"] == "norm":
        x, H = t["X"], case["H"]
        if case["dir"] == "fwd":
            mean = x.sum(1) / H
            var = (x - mean[:, None]).pow(2).sum(1) / H
            rstd = (var + EPS).pow(-0.5)
            return {"Y": torch.addcmul(t["b"], (x - mean[:, None]) * rstd[:, None], t["w"]), "mean": mean, "rstd": rstd}
        r = t["rstd"][:, None]
        n = (x - t["mean"][:, None]) * r
        g = t["dY"] * t["w"]
        dX = r / H * (H * g - g.sum(1, keepdim=True) - n * (g * n).sum(1, keepdim=True))
        return {"dX": dX, "dw": torch.einsum("mh,mh->h", t["dY"], n), "db": t["dY"].sum(0)}
    outs = []
    a, b, c = ORTHO_COEFFS
    for G in t["G"]:
        X = G if G.shape[0] <= G.shape[1] else G.t().contiguous()
        X = X / (torch.linalg.vector_norm(X) + ORTHO_EPS)
        for _ in range(ORTHO_STEPS):
            S = X.mm(X.t())
            SX = S.mm(X)
            X = a * X + b * SX + c * S.mm(SX)
        outs.append(X if G.shape[0] <= G.shape[1] else X.t())
    return {"O": torch.stack(outs)}
