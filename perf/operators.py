"""The dense operators around the LM-head -- layer norm, the matrix product with bias, activation and
residual, and the orthogonalised update -- as cases to be measured: each in a plain form made of
elementary torch operations in 32 bits, in the library's own calls, and in 64 bits from its definition."""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
NS = (3.4445, -4.7750, 2.0315)          # the quintic of the Newton-Schulz steps


def listed():
    return [
        # the final norm of one generated token
        {"name": "norm fwd, one token", "op": "norm_fwd", "M": 1, "N": 5120, "type": "bf16"},
        # the final norm in front of the LM-head over a whole micro-batch
        {"name": "norm fwd, micro-batch", "op": "norm_fwd", "M": 16384, "N": 5120, "type": "bf16"},
        # its backward pass, with the weight's and the bias' gradients
        {"name": "norm bwd, micro-batch", "op": "norm_bwd", "M": 16384, "N": 5120, "type": "bf16"},
        # a small fp32 model of odd width: forward and backward pass
        {"name": "norm fwd+bwd, odd fp32", "op": "norm_step", "M": 4099, "N": 1283, "type": "f32"},
        # one generated token through a projection
        {"name": "linear fwd, one token", "op": "linear_fwd", "M": 1, "K": 5120, "N": 5120, "act": "silu",
         "bias": True, "residual": True, "keep": False, "out": "bf16"},
        # the critic's value head: one column, fp32 values
        {"name": "linear fwd, value head", "op": "linear_fwd", "M": 16384, "K": 5120, "N": 1, "act": "none",
         "bias": True, "residual": False, "keep": False, "out": "f32"},
        # a projection of a micro-batch in training: the pre-activation is kept for the backward pass
        {"name": "linear fwd, micro-batch", "op": "linear_fwd", "M": 16384, "K": 5120, "N": 5120, "act": "gelu_tanh",
         "bias": True, "residual": True, "keep": True, "out": "bf16"},
        # its backward pass
        {"name": "linear bwd, micro-batch", "op": "linear_bwd", "M": 16384, "K": 5120, "N": 5120, "act": "gelu_tanh",
         "bias": True, "out": "bf16"},
        # a ragged handful of tokens, odd widths
        {"name": "linear bwd, odd", "op": "linear_bwd", "M": 1001, "K": 515, "N": 777, "act": "gelu",
         "bias": True, "out": "bf16"},
        # the update of a small matrix: launches count
        {"name": "update, small", "op": "update", "R": 256, "C": 1024, "type": "bf16", "nesterov": True},
        # a tall matrix of odd sizes, fp32 gradient
        {"name": "update, tall and odd", "op": "update", "R": 2001, "C": 515, "type": "f32", "nesterov": False},
        # a square projection
        {"name": "update, projection", "op": "update", "R": 5120, "C": 5120, "type": "bf16", "nesterov": True},
    ]


def draw(rng):
    def size(lo, hi):
        n = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return n if rng.random() < 0.5 else max(lo, n // 8 * 8)

    op = rng.choice(("norm_fwd", "norm_bwd", "norm_step", "linear_fwd", "linear_bwd", "update"))
    if op.startswith("norm"):
        N = size(16, 16384)
        return {"op": op, "M": size(1, min(16384, 16384 * 5120 // N)), "N": N, "type": rng.choice(("bf16", "f32"))}
    if op.startswith("linear"):
        K, N = size(8, 8192), size(1, 8192)
        case = {"op": op, "M": size(1, min(16384, 16384 * 5120 * 5120 // (K * N))), "K": K, "N": N,
                "act": rng.choice(ACTS), "bias": rng.random() < 0.8, "out": rng.choice(("bf16", "bf16", "f32"))}
        if op == "linear_fwd":
            case |= {"residual": rng.random() < 0.5, "keep": rng.random() < 0.5}
        return case
    R = size(8, 5120)
    return {"op": op, "R": R, "C": size(8, min(8192, 5120 * 5120 // R)), "type": rng.choice(("bf16", "f32")),
            "nesterov": rng.random() < 0.5}


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape, scale=1.0, to=torch.float32):
        return torch.randn(shape, generator=g, device=DEV).mul_(scale).to(to)

    s = dict(case, status=torch.zeros(1, dtype=torch.int32, device=DEV))
    op = case["op"]
    if op.startswith("norm"):
        M, N, t = case["M"], case["N"], TYPES[case["type"]]
        # hidden states: a few channels far larger than the rest, a non-zero mean
        channel = torch.exp(0.7 * normal(N))
        s["x"] = (normal(M, N) * channel + 0.3).to(t)
        s["gamma"], s["beta"] = (1 + normal(N, scale=0.2)).to(t), normal(N, scale=0.1, to=t)
        s["eps"] = 1e-5
        s["mean"], s["rstd"] = (torch.empty(M, device=DEV) for _ in range(2))
        if op != "norm_bwd":
            s["y"] = torch.empty_like(s["x"])
        if op != "norm_fwd":
            s["dy"] = normal(M, N, scale=1e-2, to=t)
            s["dx"] = torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
        if op == "norm_bwd":             # the forward pass left them
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = (x.var(1, unbiased=False) + s["eps"]).rsqrt()
    elif op.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        bf = torch.bfloat16
        s["x"] = normal(M, K, to=bf)
        s["w"] = normal(K, N, scale=K ** -0.5, to=bf)
        s["bias"] = normal(N, scale=0.3, to=bf) if case["bias"] else None
        if op == "linear_fwd":
            s["residual"] = normal(M, N, to=bf) if case["residual"] else None
            s["y"] = torch.empty((M, N), dtype=TYPES[case["out"]], device=DEV)
            s["pre"] = torch.empty((M, N), dtype=bf, device=DEV) if case["keep"] else None
        else:
            s["dy"] = normal(M, N, scale=1e-2, to=TYPES[case["out"]])
            s["pre"] = normal(M, N, to=bf) if case["act"] != "none" else None
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
            s["dbias"] = torch.empty(N, device=DEV) if case["bias"] else None
    else:
        R, C = case["R"], case["C"]
        # a weight gradient is a sum over tokens of outer products, with channels of unequal size
        tokens = 2 * min(R, C)
        def gradient():
            a = normal(tokens, R) * torch.exp(0.5 * normal(R))
            return a.t().bfloat16() @ normal(tokens, C, to=torch.bfloat16) * (tokens ** -0.5 * 1e-3)
        s["momentum"] = 8 * gradient().float()
        s["grad"] = gradient().to(TYPES[case["type"]])
        s["update"] = torch.empty((R, C), dtype=torch.bfloat16, device=DEV)
        s |= {"mu": 0.95, "eps": 1e-7, "steps": 5, "scale": max(1.0, R / C) ** 0.5}
    return s


def run(s):
    return {"norm_fwd": norm_fwd, "norm_bwd": norm_bwd, "norm_step": norm_step, "linear_fwd": linear_fwd,
            "linear_bwd": linear_bwd, "update": update}[s["op"]](s)


def scratch(s, op, *sizes):
    """The workspace that a program keeps beside its buffers; made in the first call."""
    from paper_2506_15050_b200 import binding as b
    if "ws" not in s:
        s["ws"] = b.workspace(getattr(b, op), *sizes, DEV)
    return s["ws"]


def norm_fwd(s):
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_layer_norm_fwd(s["x"], s["gamma"], s["beta"], s["eps"], s["y"], s["mean"], s["rstd"], s["status"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    x = s["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = (d.square().mean(1) + s["eps"]).rsqrt()
    y = d * rstd[:, None] * s["gamma"].float() + s["beta"].float()
    return {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd}


def norm_bwd(s, mean=None, rstd=None):
    mean, rstd = (s["mean"], s["rstd"]) if mean is None else (mean, rstd)
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_layer_norm_bwd(s["dy"], s["x"], s["gamma"], mean, rstd, s["dx"], s["dgamma"], s["dbeta"], s["status"],
                              scratch(s, "OP_LAYER_NORM", s["M"], 0, 0, s["N"]))
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    dy, t = s["dy"].float(), s["x"].dtype
    h = (s["x"].float() - mean[:, None]) * rstd[:, None]
    a = dy * s["gamma"].float()
    dx = (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True)) * rstd[:, None]
    return {"dx": dx.to(t), "dgamma": (dy * h).sum(0).to(t), "dbeta": dy.sum(0).to(t)}


def norm_step(s):
    out = norm_fwd(s)
    return out | norm_bwd(s, out["mean"], out["rstd"])


def act_plain(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        k = (2 / math.pi) ** 0.5
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    e = 1 / (1 + torch.exp(-z))
    return e * (1 + z * (1 - e))


def linear_fwd(s):
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_linear_fwd(s["x"], s["w"], s["bias"], ACTS.index(s["act"]), s["residual"], s["y"], s["pre"], s["status"],
                          scratch(s, "OP_LINEAR", s["M"], s["K"], 0, s["N"]))
        return {"y": s["y"]} if s["pre"] is None else {"y": s["y"], "pre": s["pre"]}
    z = s["x"].float() @ s["w"].float()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = act_plain(z, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(s["y"].dtype)}
    return out if s["pre"] is None else out | {"pre": z.to(s["pre"].dtype)}


def linear_bwd(s):
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_linear_bwd(s["dy"], s["x"], s["w"], ACTS.index(s["act"]), s["pre"], s["dx"], s["dw"], s["dbias"],
                          s["status"], scratch(s, "OP_LINEAR", s["M"], s["K"], 0, s["N"]))
        return {"dx": s["dx"], "dw": s["dw"]} if s["dbias"] is None else {"dx": s["dx"], "dw": s["dw"], "dbias": s["dbias"]}
    dz = s["dy"].float()
    if s["pre"] is not None:
        dz = dz * act_slope(s["pre"].float(), s["act"])
    out = {"dx": (dz @ s["w"].float().t()).to(s["dx"].dtype), "dw": (s["x"].float().t() @ dz).to(s["dw"].dtype)}
    return out if s["dbias"] is None else out | {"dbias": dz.sum(0)}


def update(s):
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_muon_orthogonalize(s["grad"], s["momentum"], s["mu"], s["nesterov"], s["eps"], s["steps"], s["scale"],
                                  s["update"], s["status"], scratch(s, "OP_MUON", s["R"], 0, 0, s["C"]))
        return {"update": s["update"], "momentum": s["momentum"]}
    g, m, mu = s["grad"].float(), s["momentum"], s["mu"]
    m.mul_(mu).add_(g)
    x = g + mu * m if s["nesterov"] else m
    x = x / (x.square().sum().sqrt() + s["eps"])
    flip = s["R"] > s["C"]
    x = x.t() if flip else x
    for _ in range(s["steps"]):
        a = x @ x.t()
        x = NS[0] * x + (NS[1] * a + NS[2] * (a @ a)) @ x
    x = x.t() if flip else x
    return {"update": (s["scale"] * x).to(torch.bfloat16), "momentum": m}


def work(case):
    op, size = case["op"], {"bf16": 2, "f32": 4}
    if op.startswith("norm"):
        M, N, e = case["M"], case["N"], size[case["type"]]
        passes = {"norm_fwd": 2, "norm_bwd": 3, "norm_step": 4}[op]      # x once, dy, y, dx
        small = {"norm_fwd": 2, "norm_bwd": 3, "norm_step": 4}[op] * N * e + 8 * M
        return {"bytes": passes * M * N * e + small, "flops": {"norm_fwd": 8, "norm_bwd": 14, "norm_step": 22}[op] * M * N}
    if op.startswith("linear"):
        M, K, N, out = case["M"], case["K"], case["N"], size[case["out"]]
        if op == "linear_fwd":
            many = 2 * (M * K + K * N + N * case["bias"]) + M * N * (out + 2 * case["residual"] + 2 * case["keep"])
            return {"bytes": many, "flops": 2 * M * K * N}
        many = 2 * 2 * (M * K + K * N) + M * N * (out + (2 if case["act"] != "none" else 0)) + 4 * N * case["bias"]
        return {"bytes": many, "flops": 4 * M * K * N}
    m, n = sorted((case["R"], case["C"]))
    # five steps; A and A^2 are symmetric, so half of each product suffices
    return {"bytes": m * n * (size[case["type"]] + 4 + 4 + 2), "flops": 5 * (m * m * n + m ** 3 + 2 * m * m * n)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op.startswith("norm"):
        x = wide["x"]
        if op == "norm_bwd":
            mean, rstd = wide["mean"][:, None], wide["rstd"][:, None]
        else:
            var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
            rstd = 1 / torch.sqrt(var + s["eps"])
        h = torch.addcmul(-mean * rstd, x, rstd)
        out = {}
        if op != "norm_bwd":
            out = {"y": torch.addcmul(wide["beta"], h, wide["gamma"]), "mean": mean[:, 0], "rstd": rstd[:, 0]}
        if op != "norm_fwd":
            a = wide["dy"] * wide["gamma"]
            N = case["N"]
            dx = rstd / N * (N * a - torch.einsum("mn->m", a)[:, None] - h * torch.einsum("mn,mn->m", a, h)[:, None])
            out |= {"dx": dx, "dgamma": torch.einsum("mn,mn->n", wide["dy"], h), "dbeta": torch.einsum("mn->n", wide["dy"])}
        return out
    if op.startswith("linear"):
        phi = lambda z: torch.special.ndtr(z)  # noqa: E731
        tanh_arg = lambda z: math.sqrt(2 / math.pi) * z * (1 + 0.044715 * z * z)  # noqa: E731
        value = {"none": lambda z: z, "relu": torch.relu, "gelu": lambda z: z * phi(z),
                 "gelu_tanh": lambda z: z * torch.sigmoid(2 * tanh_arg(z)), "silu": lambda z: z * torch.sigmoid(z)}[case["act"]]
        if op == "linear_fwd":
            z = torch.mm(wide["x"], wide["w"])
            z += wide["bias"] if case["bias"] else 0
            y = value(z)
            out = {"y": y + wide["residual"] if case["residual"] else y}
            return out | {"pre": z} if case["keep"] else out
        dz = wide["dy"]
        if case["act"] != "none":
            z = wide["pre"].requires_grad_(True)
            dz = torch.autograd.grad(value(z), z, dz)[0]
        out = {"dx": torch.mm(dz, wide["w"].t()), "dw": torch.mm(wide["x"].t(), dz)}
        return out | {"dbias": torch.einsum("mn->n", dz)} if case["bias"] else out
    m = wide["momentum"] * s["mu"] + wide["grad"]
    u = torch.add(wide["grad"], m, alpha=s["mu"]) if case["nesterov"] else m
    x = u / (torch.linalg.matrix_norm(u) + s["eps"])
    left = case["R"] <= case["C"]
    eye = torch.eye(min(x.shape), dtype=torch.float64, device=DEV)
    for _ in range(s["steps"]):
        a = x @ x.T if left else x.T @ x
        q = NS[0] * eye + a @ (NS[1] * eye + NS[2] * a)
        x = q @ x if left else x @ q
    return {"update": s["scale"] * x, "momentum": m}
