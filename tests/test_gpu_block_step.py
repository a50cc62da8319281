"""The residual join, the 8-bit products, the gradient norm and clipping as a training step uses them together with the update:
join -> 8-bit projection -> join, backward through all three, the norm of all gradients, clipping into bf16, orthogonalised
update.  Every stage is compared with its float64 formulas on the inputs it got; the whole run is captured, replayed, and run
beside itself on a second stream; and one token goes through the forward part."""
import math

import pytest
import torch

from dense_util import BF, DEV, F32, F64, U32, gen, half_step
from test_gpu_fp8 import expected, spread
from test_gpu_muon import reference
from test_gpu_residual_norm import backward64, forward64, within

pytestmark = pytest.mark.gpu
EPS, ALPHA, LIMIT = 1e-6, 0.75, 0.5


class Step:
    """Two blocks' ends around a square projection held in 8 bits."""

    def __init__(self, M=520, K=256, seed=1):
        from paper_2506_15050_b200 import binding as b
        g = gen(seed)
        r = lambda *s, scale=1.0, to=BF: (scale * torch.randn(s, generator=g, device=DEV)).to(to)
        self.M, self.K = M, K
        self.z, self.stream = r(M, K), r(M, K)
        self.p = [dict(post=1 + r(K, scale=0.2, to=F32), pre=1 + r(K, scale=0.2, to=F32), gate=r(K, scale=0.5, to=F32)) for _ in range(2)]
        w = r(K, K, scale=K ** -0.5, to=F32)
        f8 = lambda rows, cols, block: (b.fp8_empty(rows, cols, DEV), b.fp8_scales(rows, cols, block, DEV))
        self.wq, self.ws = f8(K, K, b.FP8_SQUARE)
        self.wt, self.wts = f8(K, K, b.FP8_SQUARE)
        b.tppo_fp8_quantize(w, b.FP8_SQUARE, self.wq, self.ws, self.wt, self.wts, None)
        self.dn2, self.dh2, self.momentum0 = r(M, K, scale=1e-2), r(M, K, scale=1e-2), r(K, K, scale=1e-4, to=F32)
        n = lambda *s, to=F32: torch.full(s, 7, dtype=to, device=DEV)
        m = lambda: n(M, K, to=BF)
        self.out = dict(h1=m(), n1=m(), y=m(), h2=m(), n2=m(), dy=m(), ds1=m(), dn1=m(), dz=m(), ds0=m(), rp1=n(M), rn1=n(M), rp2=n(M), rn2=n(M),
                        dw=n(K, K), sq=n(1, to=F64), norm=n(1), coef=n(1), cw=n(K, K, to=BF), momentum=n(K, K), update=n(K, K, to=BF),
                        status=n(1, to=torch.int32), **{f"d{k}{i}": n(K) for i in (1, 2) for k in ("post", "pre", "gate")},
                        **{f"c{k}{i}": n(K) for i in (1, 2) for k in ("post", "pre", "gate")})
        (self.nq, self.ns), (self.nt, self.nts) = f8(M, K, b.FP8_ROWS), f8(K, M, b.FP8_ROWS)
        (self.dq, self.ds), (self.dt, self.dts) = f8(M, K, b.FP8_ROWS), f8(K, M, b.FP8_ROWS)
        o = self.out
        names = ["post1", "pre1", "gate1", "post2", "pre2", "gate2"]
        self.grads, self.clipped = [o["dw"].view(-1)] + [o["d" + k] for k in names], [o["cw"].view(-1)] + [o["c" + k] for k in names]
        self.grad_list, self.clip_list = b.tensor_list(self.grads), b.tensor_list(self.clipped)
        self.ws_join, self.ws_norm = b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, K, DEV), b.workspace(b.OP_GRAD_NORM, 7, 0, 0, 0, DEV)
        self.ws_muon = b.workspace(b.OP_MUON, K, 0, 0, K, DEV)

    def forward(self):
        from paper_2506_15050_b200 import binding as b
        o, (p, q), st = self.out, self.p, self.out["status"]
        b.tppo_residual_norm_fwd(self.z, self.stream, p["gate"], p["post"], p["pre"], ALPHA, EPS, 3, o["h1"], o["n1"], o["rp1"], o["rn1"], st)
        b.tppo_fp8_quantize(o["n1"], b.FP8_ROWS, self.nq, self.ns, self.nt, self.nts, st)
        b.tppo_fp8_matmul(self.nq, self.ns, self.wt, self.wts, b.FP8_SQUARE, o["y"], st)
        b.tppo_residual_norm_fwd(o["y"], o["h1"], q["gate"], q["post"], q["pre"], ALPHA, EPS, 3, o["h2"], o["n2"], o["rp2"], o["rn2"], st)

    def step(self):
        from paper_2506_15050_b200 import binding as b
        o, (p, q), st = self.out, self.p, self.out["status"]
        st.zero_()
        o["momentum"].copy_(self.momentum0)
        self.forward()
        b.tppo_residual_norm_bwd(self.dh2, self.dn2, o["y"], o["h2"], q["gate"], q["post"], q["pre"], o["rp2"], o["rn2"], ALPHA, 3, o["dy"], o["ds1"],
                                 o["dgate2"], o["dpost2"], o["dpre2"], st, self.ws_join)
        b.tppo_fp8_quantize(o["dy"], b.FP8_ROWS, self.dq, self.ds, self.dt, self.dts, st)
        b.tppo_fp8_matmul(self.dq, self.ds, self.wq, self.ws, b.FP8_SQUARE, o["dn1"], st)
        b.tppo_fp8_matmul(self.nt, self.nts, self.dt, self.dts, b.FP8_ROWS, o["dw"], st)
        b.tppo_residual_norm_bwd(o["ds1"], o["dn1"], self.z, o["h1"], p["gate"], p["post"], p["pre"], o["rp1"], o["rn1"], ALPHA, 3, o["dz"], o["ds0"],
                                 o["dgate1"], o["dpost1"], o["dpre1"], st, self.ws_join)
        b.tppo_grad_norm(self.grad_list, o["sq"], o["norm"], st, self.ws_norm)
        b.tppo_grad_clip(self.grad_list, o["sq"], LIMIT, self.clip_list, o["coef"], st)
        b.tppo_muon_orthogonalize(o["cw"], o["momentum"], 0.95, True, 1e-12, 5, 1.0, o["update"], st, self.ws_muon)


def check_forward(c):
    o, M, K = c.out, c.M, c.K
    for z, s, p, h, n, r1, r2 in ((c.z, c.stream, c.p[0], "h1", "n1", "rp1", "rn1"), (o["y"], o["h1"], c.p[1], "h2", "n2", "rp2", "rn2")):
        rh, rn, q1, q2, eh, en, e1, e2 = forward64(z, s, p["gate"], p["post"], p["pre"], ALPHA, EPS, 3)
        within(o[h], rh, eh + half_step(BF) * rh.abs(), h)
        within(o[n], rn, en + (half_step(BF) + U32) * rn.abs(), n)
        within(o[r1], q1, (e1 + U32) * q1, r1)
        within(o[r2], q2, (e2 + U32) * q2, r2)
    x, xs, _, _ = expected(o["n1"], 1)
    assert torch.equal(c.nq.to(F64), x) and torch.equal(c.ns.double(), xs)
    X, W = x * spread(xs.t(), 1, 128, M, K), c.wt.to(F64) * spread(c.wts, 128, 128, K, K)
    ref = X @ W.t()
    within(o["y"], ref, 2 * (K + 2) * U32 * (X.abs() @ W.abs().t()) + half_step(BF) * ref.abs(), "y")
    return W


@pytest.mark.parametrize("M,K", [(520, 256), (1, 392), (1300, 1031)])
def test_every_stage(M, K):
    c = Step(M, K, seed=M)
    c.step()
    o = c.out
    assert int(o["status"]) == 0
    W = check_forward(c)
    # backward
    d, ds, dt, dts = expected(o["dy"], 1)
    D, Dt = d * spread(ds.t(), 1, 128, M, K), dt * spread(dts.t(), 1, 128, K, M)
    X = c.nt.to(F64) * spread(c.nts.t(), 1, 128, K, M)
    for got, a, w, k in ((o["dn1"], D, W, K), (o["dw"], X, Dt.t(), M)):
        ref = a @ w
        within(got, ref, 2 * (k + 2) * U32 * (a.abs() @ w.abs()) + half_step(got.dtype) * ref.abs() + 1e-37)
    for i, dh, dn, z, h, p, dz, ds in ((2, c.dh2, c.dn2, o["y"], o["h2"], c.p[1], "dy", "ds1"), (1, o["ds1"], o["dn1"], c.z, o["h1"], c.p[0], "dz", "ds0")):
        ref = backward64(dh, dn, z, h, p["gate"], p["post"], p["pre"], o[f"rp{i}"], o[f"rn{i}"], ALPHA, 3)
        for name, key in ((dz, "dz"), (ds, "dresidual"), (f"dgate{i}", "dgate"), (f"dpost{i}", "dgamma_post"), (f"dpre{i}", "dgamma_pre")):
            v, tol = ref[key]
            within(o[name], v, tol + (half_step(o[name].dtype) + U32) * v.abs() + 1e-37, name)
    # norm, clipping, update
    norm = math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in c.grads))
    assert abs(float(o["norm"]) - norm) <= 7 * U32 * norm
    coef = min(1.0, LIMIT / norm)
    assert abs(float(o["coef"]) - coef) <= 8 * U32 * coef
    for got, t in zip(c.clipped, c.grads):
        r = t.double() * coef
        within(got, r, (10 * U32 + half_step(got.dtype)) * r.abs() + 1e-37)
    mu = float(torch.tensor(0.95, dtype=F32))
    u = o["cw"].double() + mu * o["momentum"].double()
    ref = reference(u, 5, 1e-12)
    assert (o["update"].double() - ref).norm() <= (1.16e-2 + half_step(BF)) * ref.norm()


def outputs(c):
    return {k: v.clone() for k, v in c.out.items()}


@pytest.mark.parametrize("M,K", [(520, 256), (1, 72), (2600, 1030)])
def test_captured_step_replays_bit_for_bit(M, K):
    c = Step(M, K, seed=M + 1)
    c.step()
    torch.cuda.synchronize()
    eager = outputs(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for v in c.out.values():
            v.fill_(3)
        for w in (c.ws_join, c.ws_norm, c.ws_muon):
            w.fill_(0xff)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.step()
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for k, v in eager.items():
            assert torch.equal(c.out[k], v), k
    c.z.copy_((c.z.float() * 0.5 + 1).to(BF))              # new inputs in the same buffers
    graph.replay()
    torch.cuda.synchronize()
    got = outputs(c)
    c.step()
    for k, v in got.items():
        assert torch.equal(c.out[k], v), k


def test_two_steps_beside_each_other():
    """Own buffers and workspaces on two streams: nothing is shared."""
    a, b = Step(900, 320, seed=3), Step(2100, 1928, seed=4)
    a.step()
    b.step()
    torch.cuda.synchronize()
    want = outputs(a), outputs(b)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        for c, st in ((a, s), (b, t)):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                c.step()
    torch.cuda.synchronize()
    for c, w in ((a, want[0]), (b, want[1])):
        for k, v in w.items():
            assert torch.equal(c.out[k], v), k


def test_a_token_of_a_batch_comes_out_as_by_itself():
    """What a row gets does not depend on the rows beside it, beyond the order of its sums."""
    a, one = Step(70, 640, seed=8), Step(1, 640, seed=8)
    a.step()
    one.p, one.wt, one.wts = a.p, a.wt, a.wts
    one.z.copy_(a.z[33:34])
    one.stream.copy_(a.stream[33:34])
    one.out["status"].zero_()
    one.forward()
    assert int(one.out["status"]) == 0
    check_forward(one)
