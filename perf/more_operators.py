"""The operators of a block's ends and of the step behind its backward pass -- the residual join with the norms
before and after it, products in 8 bits with a scale per block of 128, the global gradient norm with clipping --
as cases to be measured: each in a plain form made of elementary torch operations in 32 bits, in the library's
own calls, and in 64 bits from its definition."""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn
BLOCK = 128                             # elements that share a scale
EPS = 1e-6


def listed():
    return [
        # one generated token between two blocks
        {"name": "join fwd, one token", "op": "join_fwd", "M": 1, "N": 5120, "type": "bf16", "gate": "row", "norms": 3},
        # a micro-batch of hidden states between two blocks
        {"name": "join fwd, micro-batch", "op": "join_fwd", "M": 16384, "N": 5120, "type": "bf16", "gate": "row", "norms": 3},
        # its backward pass, with the gradients of both norms' weights and of the gate
        {"name": "join bwd, micro-batch", "op": "join_bwd", "M": 16384, "N": 5120, "type": "bf16", "gate": "row", "norms": 3},
        # a small fp32 model of odd width whose gate is computed per token: forward and backward pass
        {"name": "join fwd+bwd, odd fp32", "op": "join_step", "M": 4099, "N": 1283, "type": "f32", "gate": "full", "norms": 3},
        # one generated token through an 8-bit projection
        {"name": "fp8 fwd, one token", "op": "fp8_fwd", "M": 1, "K": 5120, "N": 5120},
        # a projection of a micro-batch: activations quantised, then the product
        {"name": "fp8 fwd, micro-batch", "op": "fp8_fwd", "M": 16384, "K": 5120, "N": 5120},
        # its backward pass: the output's gradient quantised both ways, the input's and the weight's gradient
        {"name": "fp8 bwd, micro-batch", "op": "fp8_bwd", "M": 16384, "K": 5120, "N": 5120},
        # a ragged handful of tokens, odd widths: forward and backward pass
        {"name": "fp8 fwd+bwd, odd", "op": "fp8_step", "M": 1001, "K": 515, "N": 777},
        # the adapters and norms of a small model
        {"name": "clip, small tensors", "op": "clip", "count": 40, "total": 60000, "type": "mix", "to": "same", "clips": True, "packed": True},
        # gradients accumulated in fp32 over micro-batches, handed to the update as bf16
        {"name": "clip, accumulators", "op": "clip", "count": 250, "total": 150000000, "type": "f32", "to": "bf16", "clips": True, "packed": False},
        # a step whose norm is under the limit: gradients stay where they are
        {"name": "norm under the limit", "op": "clip", "count": 600, "total": 600000000, "type": "bf16", "to": "place", "clips": False,
         "packed": False},
        # ... and one over it
        {"name": "clip, many tensors", "op": "clip", "count": 600, "total": 600000000, "type": "bf16", "to": "same", "clips": True,
         "packed": False},
    ]


def draw(rng):
    def size(lo, hi):
        n = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        return n if rng.random() < 0.5 else max(lo, n // 8 * 8)

    op = rng.choice(("join_fwd", "join_bwd", "join_step", "fp8_fwd", "fp8_bwd", "fp8_step", "clip", "clip"))
    if op.startswith("join"):
        N = size(16, 16384)
        return {"op": op, "M": size(1, min(16384, 16384 * 5120 // N)), "N": N, "type": rng.choice(("bf16", "f32")),
                "gate": rng.choice(("none", "row", "full")), "norms": rng.choice((1, 2, 3, 3))}
    if op.startswith("fp8"):
        K, N = size(8, 8192), size(8, 8192)
        return {"op": op, "M": size(1, min(16384, 16384 * 5120 * 5120 // (K * N))), "K": K, "N": N}
    total = size(1000, 600000000)
    to, kind = rng.choice(("same", "bf16", "place")), rng.choice(("bf16", "f32", "mix"))
    if kind != "bf16":
        total //= 2
    return {"op": op, "count": size(1, 800), "total": total, "type": kind, "to": to, "clips": to != "place",
            "packed": rng.random() < 0.5}


def sizes_of(case):
    """Lengths of the gradients: matrices of all sizes, and among them vectors, single numbers and an empty one."""
    rng = random.Random(f"{case['count']} {case['total']}")
    n = case["count"]
    share = [math.exp(rng.gauss(0, 1)) if rng.random() < 0.6 else 1e-5 for _ in range(n)]
    unit = case["total"] / sum(share)
    sizes = [max(1, round(s * unit)) for s in share]
    if n > 3:
        sizes[n // 2] = 0
    return sizes


def rows16(r, c, dtype):
    """A matrix whose rows start on 16-byte boundaries."""
    step = 16 // dtype.itemsize
    return torch.empty((r, -(-c // step) * step), dtype=dtype, device=DEV)[:, :c]


def pieces(sizes, types, packed):
    """([a zeroed buffer per type], [a piece of it for each size])"""
    at, where = {}, []
    for n, t in zip(sizes, types):
        a = at.get(t, 0)
        where.append(a)
        at[t] = a + (n if packed else -(-n // 8) * 8)
    flat = {t: torch.zeros(n, dtype=t, device=DEV) for t, n in at.items()}
    return list(flat.values()), [flat[t][a:a + n] for n, t, a in zip(sizes, types, where)]


def quantise_plain(x, rows, cols):
    """Blocks of rows x cols: (values, as float8; scale of each block), scale the least power of two that holds them."""
    M, K = x.shape
    mb, kb = -(-M // rows), -(-K // cols)
    amax = torch.zeros((mb * rows, kb * cols), device=DEV)
    amax[:M, :K] = x.abs()
    amax = amax.view(mb, rows, kb, cols).amax((1, 3))
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp_min(-126)
    e = torch.where(amax > 0, e, 0)
    s = torch.ldexp(torch.ones_like(amax), e)
    wide = spread(s, rows, cols, M, K)
    q = rows16(M, K, F8)
    q.copy_((x / wide).to(F8))
    return q, s


def spread(s, rows, cols, M, K):
    return s.repeat_interleave(rows, 0)[:M].repeat_interleave(cols, 1)[:, :K]


def store(s):
    t = rows16(*s.shape, torch.float32)
    return t.copy_(s)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape, scale=1.0, to=torch.float32):
        return torch.randn(shape, generator=g, device=DEV).mul_(scale).to(to)

    s = dict(case, status=torch.zeros(1, dtype=torch.int32, device=DEV))
    op = case["op"]
    if op.startswith("join"):
        M, N, t = case["M"], case["N"], TYPES[case["type"]]
        # hidden states: a few channels far larger than the rest
        channel = torch.exp(0.7 * normal(N))
        s["z"], s["residual"] = normal(M, N).mul_(2).to(t), normal(M, N).mul_(channel).to(t)
        s["gamma_post"] = (1 + normal(N, scale=0.2)).to(t) if case["norms"] & 1 else None
        s["gamma_pre"] = (1 + normal(N, scale=0.2)).to(t) if case["norms"] & 2 else None
        s["gate"] = {"none": lambda: None, "row": lambda: normal(N, scale=0.5, to=t),
                     "full": lambda: torch.sigmoid(normal(M, N)).to(t)}[case["gate"]]()
        s["alpha"] = 0.75
        s["h"] = torch.empty_like(s["z"])
        s["n"] = torch.empty_like(s["z"]) if case["norms"] & 2 else None
        s["r_post"] = torch.empty(M, device=DEV) if case["norms"] & 1 else None
        s["r_pre"] = torch.empty(M, device=DEV) if case["norms"] & 2 else None
        if op != "join_fwd":
            s["dh"] = normal(M, N, scale=1e-2, to=t)
            s["dn"] = normal(M, N, scale=1e-2, to=t) if case["norms"] & 2 else None
            for k in ("z", "residual", "gate", "gamma_post", "gamma_pre"):
                s["d" + k] = None if s[k] is None else torch.empty_like(s[k])
        if op == "join_bwd":            # the forward pass left them
            out = join_fwd_plain(s)
            s["h"] = out["h"]
            s["r_post"], s["r_pre"] = out.get("r_post"), out.get("r_pre")
    elif op.startswith("fp8"):
        M, K, N, bf = case["M"], case["K"], case["N"], torch.bfloat16
        channel = torch.exp(0.7 * normal(K))
        x = normal(M, K).mul_(channel).to(bf)
        # the weight [K, N] is kept in 8 bits, as it is and transposed
        w = normal(K, N, scale=K ** -0.5)
        q, sc = quantise_plain(w, BLOCK, BLOCK)
        s["w"], s["w_scale"] = q, sc.contiguous()
        s["wt"], s["wt_scale"] = rows16(N, K, F8).copy_(q.t()), sc.t().contiguous()
        if op != "fp8_bwd":
            s["x"] = x
            s["xq"], s["x_scale"] = rows16(M, K, F8), rows16(-(-K // BLOCK), M, torch.float32)
            s["y"] = torch.empty((M, N), dtype=bf, device=DEV)
        if op != "fp8_fwd":
            s["dy"] = normal(M, N, scale=1e-3, to=bf)
            s["dyq"], s["dy_scale"] = rows16(M, N, F8), rows16(-(-N // BLOCK), M, torch.float32)
            s["dyt"], s["dyt_scale"] = rows16(N, M, F8), rows16(-(-M // BLOCK), N, torch.float32)
            s["dx"], s["dw"] = torch.empty((M, K), dtype=bf, device=DEV), torch.empty((K, N), device=DEV)
            if op == "fp8_bwd":         # the forward pass left the activations, quantised along the tokens
                q, sc = quantise_plain(x.float().t(), 1, BLOCK)
                s["xt"], s["xt_scale"] = q, store(sc.t())
            else:
                s["xt"], s["xt_scale"] = rows16(K, M, F8), rows16(-(-M // BLOCK), K, torch.float32)
    else:
        # gradients are pieces of one buffer per type, as programs keep them; packed, or each on a 16-byte boundary
        sizes, kind = sizes_of(case), case["type"]
        types = [TYPES[kind] if kind != "mix" else (torch.bfloat16, torch.float32)[i % 2] for i in range(len(sizes))]
        s["flat"], s["grads"] = pieces(sizes, types, case["packed"])
        for i, t in enumerate(s["grads"]):
            t.copy_(normal(t.numel(), scale=1e-3 * (1 + i % 7)))
        if case["to"] == "place":
            s["out_flat"], s["out"] = s["flat"], s["grads"]
        else:
            s["out_flat"], s["out"] = pieces(sizes, types if case["to"] == "same" else [torch.bfloat16] * len(sizes), case["packed"])
        norm = 1e-3 * math.sqrt(sum(n * (1 + i % 7) ** 2 for i, n in enumerate(sizes)))
        s["max_norm"] = norm * (0.3 if case["clips"] else 3.0)
        s["sum_sq"] = torch.empty(1, dtype=torch.float64, device=DEV)
        s["norm"], s["coef"] = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    return s


def run(s):
    return {"join_fwd": join_fwd, "join_bwd": join_bwd, "join_step": join_step, "fp8_fwd": fp8_fwd, "fp8_bwd": fp8_bwd,
            "fp8_step": fp8_step, "clip": clip}[s["op"]](s)


def given(**out):
    return {k: v for k, v in out.items() if v is not None}


def join_fwd(s):
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_residual_norm_fwd(s["z"], s["residual"], s["gate"], s["gamma_post"], s["gamma_pre"], s["alpha"], EPS, s["norms"],
                                 s["h"], s["n"], s["r_post"], s["r_pre"], s["status"])
        return given(h=s["h"], n=s["n"], r_post=s["r_post"], r_pre=s["r_pre"])
    return join_fwd_plain(s)


def join_fwd_plain(s):
    t, out = s["z"].dtype, {}
    u = s["z"].float()
    if s["norms"] & 1:
        out["r_post"] = (u.square().mean(1) + EPS).rsqrt()
        u = u * out["r_post"][:, None] * s["gamma_post"].float()
    if s["gate"] is not None:
        u = u * s["gate"].float()
    h = u + s["alpha"] * s["residual"].float()
    out["h"] = h.to(t)
    if s["norms"] & 2:
        out["r_pre"] = (h.square().mean(1) + EPS).rsqrt()
        out["n"] = (h * out["r_pre"][:, None] * s["gamma_pre"].float()).to(t)
    return out


def join_bwd(s, saved=None):
    saved = saved or s
    if own:
        from paper_2506_15050_b200 import binding as b
        if "ws" not in s:               # the workspace that a program keeps beside its buffers
            s["ws"] = b.workspace(b.OP_RESIDUAL_NORM, s["M"], 0, 0, s["N"], DEV)
        b.tppo_residual_norm_bwd(s["dh"], s["dn"], s["z"], saved["h"], s["gate"], s["gamma_post"], s["gamma_pre"],
                                 saved.get("r_post"), saved.get("r_pre"), s["alpha"], s["norms"], s["dz"], s["dresidual"],
                                 s["dgate"], s["dgamma_post"], s["dgamma_pre"], s["status"], s["ws"])
        return given(dz=s["dz"], dresidual=s["dresidual"], dgate=s["dgate"], dgamma_post=s["dgamma_post"], dgamma_pre=s["dgamma_pre"])
    t, z, d, out = s["z"].dtype, s["z"].float(), s["dh"].float(), {}
    if s["norms"] & 2:
        r, dn = saved["r_pre"][:, None], s["dn"].float()
        hh = saved["h"].float() * r
        a = dn * s["gamma_pre"].float()
        d = d + r * (a - hh * (a * hh).mean(1, keepdim=True))
        out["dgamma_pre"] = (dn * hh).sum(0).to(t)
    out["dresidual"] = (s["alpha"] * d).to(t)
    zz = z * saved["r_post"][:, None] if s["norms"] & 1 else z
    gate = 1.0 if s["gate"] is None else s["gate"].float()
    gamma = s["gamma_post"].float() if s["norms"] & 1 else 1.0
    if s["gate"] is not None:
        dg = d * zz * gamma
        out["dgate"] = (dg.sum(0) if s["gate"].dim() == 1 else dg).to(t)
    a = d * gate
    if s["norms"] & 1:
        out["dgamma_post"] = (a * zz).sum(0).to(t)
        a = a * gamma
        a = saved["r_post"][:, None] * (a - zz * (a * zz).mean(1, keepdim=True))
    out["dz"] = a.to(t)
    return out


def join_step(s):
    out = join_fwd(s)
    return out | join_bwd(s, out)


def dequantised(q, scale, rows, cols):
    return q.float() * spread(scale, rows, cols, *q.shape)


def fp8_fwd(s, transposed=False):
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_fp8_quantize(s["x"], b.FP8_ROWS, s["xq"], s["x_scale"], s["xt"] if transposed else None,
                            s["xt_scale"] if transposed else None, s["status"])
        b.tppo_fp8_matmul(s["xq"], s["x_scale"], s["wt"], s["wt_scale"], b.FP8_SQUARE, s["y"], s["status"])
        return {"y": s["y"]}
    x = s["x"].float()
    q, sc = quantise_plain(x, 1, BLOCK)
    y = dequantised(q, sc, 1, BLOCK) @ dequantised(s["wt"], s["wt_scale"], BLOCK, BLOCK).t()
    if transposed:
        q, sc = quantise_plain(x.t(), 1, BLOCK)
        s["xt"], s["xt_scale"] = q, store(sc.t())
    return {"y": y.to(s["y"].dtype)}


def fp8_bwd(s):
    if own:
        from paper_2506_15050_b200 import binding as b
        b.tppo_fp8_quantize(s["dy"], b.FP8_ROWS, s["dyq"], s["dy_scale"], s["dyt"], s["dyt_scale"], s["status"])
        b.tppo_fp8_matmul(s["dyq"], s["dy_scale"], s["w"], s["w_scale"], b.FP8_SQUARE, s["dx"], s["status"])
        b.tppo_fp8_matmul(s["xt"], s["xt_scale"], s["dyt"], s["dyt_scale"], b.FP8_ROWS, s["dw"], s["status"])
        return {"dx": s["dx"], "dw": s["dw"]}
    dy = s["dy"].float()
    q, sc = quantise_plain(dy, 1, BLOCK)
    dx = dequantised(q, sc, 1, BLOCK) @ dequantised(s["w"], s["w_scale"], BLOCK, BLOCK).t()
    q, sc = quantise_plain(dy.t(), 1, BLOCK)
    dw = dequantised(s["xt"], s["xt_scale"].t(), 1, BLOCK) @ dequantised(q, sc, 1, BLOCK).t()
    return {"dx": dx.to(s["dx"].dtype), "dw": dw}


def fp8_step(s):
    return fp8_fwd(s, transposed=True) | fp8_bwd(s)


def clip(s):
    if own:
        from paper_2506_15050_b200 import binding as b
        if "list" not in s:             # what a program makes once, beside its gradients
            s["list"] = b.tensor_list(s["grads"])
            s["out_list"] = s["list"] if s["out"] is s["grads"] else b.tensor_list(s["out"])
            s["ws"] = b.workspace(b.OP_GRAD_NORM, len(s["grads"]), 0, 0, 0, DEV)
        b.tppo_grad_norm(s["list"], s["sum_sq"], s["norm"], s["status"], s["ws"])
        b.tppo_grad_clip(s["list"], s["sum_sq"], s["max_norm"], s["out_list"], s["coef"], s["status"])
        return {"norm": s["norm"], "coef": s["coef"], "out": s["out_flat"]}
    total = torch.zeros(1, dtype=torch.float64, device=DEV)
    for g in s["grads"]:                # a long sum
        total += g.double().square().sum()
    norm = total.sqrt()
    coef = (s["max_norm"] / norm).clamp_max(1).float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * coef)
    return {"norm": norm.float(), "coef": coef, "out": s["out_flat"]}


def work(case):
    op, size = case["op"], {"bf16": 2, "f32": 4}
    if op.startswith("join"):
        M, N, e = case["M"], case["N"], size[case["type"]]
        pre, post, full = case["norms"] >> 1, case["norms"] & 1, case["gate"] == "full"
        row = case["gate"] == "row"
        fwd = 3 + pre + full                              # z, residual, h; n; gate
        bwd = 5 + 2 * pre + 2 * full                      # dh, z, dz, dresidual, (with n:) dn, h; gate, dgate
        if not (pre or post or full or row):
            bwd -= 1
        step = fwd + bwd - 1 - pre - full                 # z, h and the gate are read once
        many = {"join_fwd": fwd, "join_bwd": bwd, "join_step": step}[op] * M * N * e
        vectors = (pre + post + row) * N * e * (1 if op == "join_fwd" else 2) + 4 * M * (pre + post)
        return {"bytes": many + vectors, "flops": {"join_fwd": 9, "join_bwd": 22, "join_step": 31}[op] * M * N}
    if op.startswith("fp8"):
        M, K, N = case["M"], case["K"], case["N"]
        if op == "fp8_fwd":
            return {"bytes": 2 * M * K + K * N + 2 * M * N, "flops": 2 * M * K * N}
        if op == "fp8_bwd":
            return {"bytes": 2 * M * N + K * N + M * K + 2 * M * K + 4 * K * N, "flops": 4 * M * K * N}
        return {"bytes": 2 * M * K + K * N + 2 * M * N + 2 * M * N + 2 * M * K + 4 * K * N, "flops": 6 * M * K * N}
    sizes, kind = sizes_of(case), case["type"]
    e = [size[kind] if kind != "mix" else (2, 4)[i % 2] for i in range(len(sizes))]
    many = sum(n * k for n, k in zip(sizes, e))
    if case["to"] != "place":
        many += sum(n * (2 if case["to"] == "bf16" else k) for n, k in zip(sizes, e))
    return {"bytes": many, "flops": 3 * sum(sizes)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("join"):
        wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
        z, N, out = wide["z"], case["N"], {}
        one = torch.ones(N, dtype=torch.float64, device=DEV)
        c = wide.get("gate", one) * wide.get("gamma_post", one)         # what multiplies the normed z
        length = lambda v: torch.linalg.vector_norm(v, dim=1) / math.sqrt(N)  # noqa: E731
        if op == "join_bwd":
            h, rp, rn = wide["h"], wide.get("r_post"), wide.get("r_pre")
        else:
            rp = 1 / torch.sqrt(length(z) ** 2 + EPS) if case["norms"] & 1 else None
            h = torch.addcmul(wide["residual"] * s["alpha"], c, z if rp is None else z * rp[:, None])
            rn = 1 / torch.sqrt(length(h) ** 2 + EPS) if case["norms"] & 2 else None
            out = given(h=h, r_post=rp, r_pre=rn, n=None if rn is None else torch.einsum("mn,m,n->mn", h, rn, wide["gamma_pre"]))
        if op == "join_fwd":
            return out
        d = wide["dh"]
        if rn is not None:
            a = torch.einsum("mn,n,m->mn", wide["dn"], wide["gamma_pre"], rn)
            d = d + a - h * (torch.einsum("mn,mn,m->m", a, h, rn * rn) / N)[:, None]
            out["dgamma_pre"] = torch.einsum("mn,mn,m->n", wide["dn"], h, rn)
        out["dresidual"] = d * s["alpha"]
        zz = z if rp is None else torch.einsum("mn,m->mn", z, rp)
        if case["gate"] == "row":
            out["dgate"] = torch.einsum("mn,mn,n->n", d, zz, wide.get("gamma_post", one))
        elif case["gate"] == "full":
            out["dgate"] = torch.einsum("mn,mn,n->mn", d, zz, wide.get("gamma_post", one))
        dz = d * c
        if rp is not None:
            out["dgamma_post"] = (d * wide.get("gate", one) * zz).sum(0)
            dz = rp[:, None] * (dz - zz * torch.einsum("mn,mn->m", dz, zz)[:, None] / N)
        out["dz"] = dz
        return out
    if op.startswith("fp8"):
        def held(x, dim):
            """The values that x stands for once blocks of 128 along `dim` share a power of two and keep four bits each."""
            x = x.double().movedim(dim, -1)
            shape = x.shape
            x = torch.nn.functional.pad(x, (0, -shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK))
            top = x.abs().amax(-1, keepdim=True)
            unit = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp_min(-126))
            unit = torch.where(unit / 2 * 448 >= top, unit / 2, unit)   # log2 rounds
            unit = torch.where(unit * 448 < top, unit * 2, unit)
            unit = torch.where(top > 0, unit, 1.0)
            v = x / unit
            step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
            return (torch.round(v / step) * step * unit).flatten(-2)[..., :shape[-1]].movedim(-1, dim)

        def kept(q, scale, rows, cols):
            r, c = (torch.arange(n, device=DEV) // k for n, k in zip(q.shape, (rows, cols)))
            return q.double() * scale.double()[r][:, c]

        out, w = {}, kept(s["w"], s["w_scale"], BLOCK, BLOCK)
        if op != "fp8_bwd":
            out["y"] = torch.einsum("mk,kn->mn", held(s["x"], 1), w)
        if op != "fp8_fwd":
            xt = held(s["x"], 0).t() if op == "fp8_step" else kept(s["xt"], s["xt_scale"].t(), 1, BLOCK)
            out["dx"] = torch.einsum("mn,kn->mk", held(s["dy"], 1), w)
            out["dw"] = torch.einsum("km,mn->kn", xt, held(s["dy"], 0))
        return out
    norm = math.sqrt(math.fsum(float(torch.dot(g.double(), g.double())) for g in s["grads"]))
    coef = min(1.0, s["max_norm"] / norm)
    one = lambda v: torch.tensor([v], dtype=torch.float64, device=DEV)  # noqa: E731
    return {"norm": one(norm), "coef": one(coef), "out": scaled(s, coef)}


def scaled(s, coef):
    out = [torch.zeros(f.shape, dtype=torch.float64, device=DEV) for f in s["out_flat"]]
    first = {f.untyped_storage().data_ptr(): o for f, o in zip(s["out_flat"], out)}
    for g, o in zip(s["grads"], s["out"]):
        at = o.storage_offset()
        torch.mul(g.double(), coef, out=first[o.untyped_storage().data_ptr()][at:at + o.numel()])
    return out
