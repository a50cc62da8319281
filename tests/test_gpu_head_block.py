"""The dense operators as a training step uses them together: layer norm -> projection with residual ->
LM-head loss and its gradients -> backward pass -> orthogonalised updates; value head -> advantages ->
value loss -> its gradient.  Every stage is compared with its float64 formulas on the inputs it got;
the whole run is captured, replayed, and run beside itself on a second stream."""
import pytest
import torch

from dense_util import BF, DEV, F32, F64, U32, act64, gen, half_step, norm64, norm64_bwd, slope64
from test_gpu_muon import reference

pytestmark = pytest.mark.gpu


class Block:
    """One head block: parameters, buffers and workspaces, and the calls of a step."""

    def __init__(self, M=520, K=256, V=1024, seed=1):
        from paper_2506_15050_b200 import binding as b
        g = gen(seed)
        r = lambda *s, scale=1.0, to=F32: (scale * torch.randn(s, generator=g, device=DEV)).to(to)
        self.M, self.K, self.V = M, K, V
        self.h, self.w, self.bias = r(M, K, to=BF), r(K, K, scale=K ** -0.5, to=BF), r(K, scale=0.1)
        self.gamma, self.beta = 1 + r(K, scale=0.2), r(K, scale=0.1)
        self.head = r(K, V, scale=K ** -0.5, to=BF)
        self.vw, self.vb = r(K, 1, scale=K ** -0.5, to=BF), r(1)
        self.targets = torch.randint(0, V, (M,), generator=g, device=DEV, dtype=torch.int32)
        self.old_logp, self.adv_in = torch.full((M,), -7.0, device=DEV), r(M)
        self.rewards, self.old_values = r(M), r(M, scale=0.3)
        self.seg_b = torch.tensor([0, M // 3], dtype=torch.int32, device=DEV)
        self.seg_e = torch.tensor([M // 3, M], dtype=torch.int32, device=DEV)
        self.cut = torch.tensor([0, 1], dtype=torch.uint8, device=DEV)
        self.momentum0 = r(K, K, scale=1e-4)
        n = lambda *s, to=F32: torch.full(s, 7, dtype=to, device=DEV)
        self.out = dict(n=n(M, K, to=BF), mean=n(M), rstd=n(M), y=n(M, K, to=BF), pre=n(M, K, to=BF), logp=n(M), loss=n(1),
                        stats=n(4, to=torch.int32), dy=n(M, K, to=BF), dhead=n(K, V, to=BF), dn=n(M, K, to=BF), dw=n(K, K, to=BF), db=n(K),
                        dx=n(M, K, to=BF), dgamma=n(K), dbeta=n(K), update=n(K, K, to=BF), head_update=n(K, V, to=BF), momentum=n(K, K),
                        values=n(M, 1), adv=n(M), ret=n(M), est=n(1, to=torch.int32), vloss=n(1), dvalues=n(M), vst=n(2, to=torch.int32),
                        dvx=n(M, K, to=BF), dvw=n(K, 1, to=BF), dvb=n(1), status=n(1, to=torch.int32))
        ws = lambda op, *s: b.workspace(op, *s, DEV)
        self.ws = dict(ln=ws(b.OP_LAYER_NORM, M, 0, 0, K), lin=ws(b.OP_LINEAR, M, K, 0, K), head=ws(b.OP_LMHEAD, M, K, 0, V),
                       mu=ws(b.OP_MUON, K, 0, 0, K), mh=ws(b.OP_MUON, K, 0, 0, V), vl=ws(b.OP_LINEAR, M, K, 0, 1),
                       egae=ws(b.OP_EGAE, M, 2, 0, 0), val=ws(b.OP_VALUE_LOSS, M, 0, M, 0))

    def step(self):
        from paper_2506_15050_b200 import binding as b
        o, w, st = self.out, self.ws, self.out["status"]
        st.zero_()
        o["momentum"].copy_(self.momentum0)
        b.tppo_layer_norm_fwd(self.h, self.gamma, self.beta, 1e-5, o["n"], o["mean"], o["rstd"], st)
        b.tppo_linear_fwd(o["n"], self.w, self.bias, b.ACT_GELU, self.h, o["y"], o["pre"], st, w["lin"])
        b.tppo_lmhead_logprob_fwd_bwd(o["y"], self.head, self.targets, None, self.old_logp, self.adv_in, 0.2, 0.28, 0.0, o["logp"], None,
                                      o["loss"], o["stats"], o["dy"], o["dhead"], w["head"])
        b.tppo_linear_bwd(o["dy"], o["n"], self.w, b.ACT_GELU, o["pre"], o["dn"], o["dw"], o["db"], st, w["lin"])
        b.tppo_layer_norm_bwd(o["dn"], self.h, self.gamma, o["mean"], o["rstd"], o["dx"], o["dgamma"], o["dbeta"], st, w["ln"])
        b.tppo_muon_orthogonalize(o["dw"], o["momentum"], 0.95, True, 1e-12, 5, 1.0, o["update"], st, w["mu"])
        b.tppo_muon_orthogonalize(o["dhead"], None, 0.0, False, 1e-12, 5, 1.0, o["head_update"], st, w["mh"])
        b.tppo_linear_fwd(o["n"], self.vw, self.vb, b.ACT_NONE, None, o["values"], None, st, w["vl"])
        v = o["values"].view(-1)
        b.tppo_egae(self.rewards, v, self.seg_b, self.seg_e, self.cut, None, 1.0, 0.95, o["adv"], o["ret"], o["est"], w["egae"])
        b.tppo_value_loss(v, self.old_values, o["ret"], None, None, self.M, 0.5, 0.6, 0.0, o["vloss"], o["dvalues"], o["vst"], w["val"])
        b.tppo_linear_bwd(o["dvalues"].view(-1, 1), o["n"], self.vw, b.ACT_NONE, None, o["dvx"], o["dvw"], o["dvb"], st, w["vl"])


def within(got, ref, tol):
    assert bool(((got.double() - ref).abs() <= tol).all()), ((got.double() - ref).abs() / tol).max().item()


def test_every_stage_of_a_step():
    c = Block()
    c.step()
    o, M, K = c.out, c.M, c.K
    assert int(o["status"]) == 0 and int(o["stats"][3]) == 0 and int(o["est"]) == 0 and int(o["vst"][1]) == 0
    # layer norm (tolerances: test_gpu_layer_norm; here 64 roundings cover a row of 256)
    y, mean, rstd, h = norm64(c.h, c.gamma, c.beta, 1e-5)
    within(o["n"], y, 64 * U32 * (c.gamma.double().abs() * (h.abs() + rstd[:, None] * c.h.double().abs().mean(1, keepdim=True)) + y.abs())
           + half_step(BF) * y.abs())
    # projection: sums of K products at 2^-23 each, act' <= 1.13, then one bf16 rounding
    n, w = o["n"].double(), c.w.double()
    z = n @ w + c.bias.double()
    e = 2 * (K + 2) * U32 * (n.abs() @ w.abs() + c.bias.double().abs())
    ref = act64(z, 2) + c.h.double()
    within(o["pre"], z, e + half_step(BF) * z.abs())
    within(o["y"], ref, 1.13 * e + 16 * U32 * (z.abs() + 1e-6) + (half_step(BF) + U32) * ref.abs())
    # its backward pass: dz rounded to bf16 once, one more rounding of the outputs
    dz = o["dy"].double() * slope64(o["pre"].double(), 2)
    e_dz = half_step(BF) * dz.abs() + 24 * U32 * o["dy"].double().abs() * (1 + o["pre"].double().abs())
    for got, ref, err, mag, k in ((o["dn"], dz @ w.t(), e_dz @ w.abs().t(), dz.abs() @ w.abs().t(), K),
                                  (o["dw"], n.t() @ dz, n.abs().t() @ e_dz, n.abs().t() @ dz.abs(), M)):
        within(got, ref, 1.01 * err + 2 * k * U32 * mag * 1.01 + half_step(BF) * ref.abs())
    within(o["db"], dz.sum(0), (24 * U32 * o["dy"].double().abs() * (1 + o["pre"].double().abs())).sum(0) + M * U32 * dz.abs().sum(0))
    # layer norm's backward pass from the mean and rstd of the forward call
    hh = (c.h.double() - o["mean"].double()[:, None]) * o["rstd"].double()[:, None]
    dx, dg, db = norm64_bwd(o["dn"], hh, o["rstd"].double(), c.gamma)
    a = o["dn"].double() * c.gamma.double()
    terms = a.abs() + 64 * a.abs().mean(1, keepdim=True) + 64 * hh.abs() * (a * hh).abs().mean(1, keepdim=True)
    within(o["dx"], dx, 5 * U32 * o["rstd"].double()[:, None] * terms + half_step(BF) * dx.abs() + 1e-30)
    within(o["dgamma"], dg, 300 * U32 * (o["dn"].double() * hh).abs().sum(0) + 1e-30)
    within(o["dbeta"], db, 300 * U32 * o["dn"].double().abs().sum(0) + 1e-30)
    # updates (1.16e-2 of the norm: test_gpu_muon)
    mu = float(torch.tensor(0.95, dtype=F32))
    mom = mu * c.momentum0.double() + o["dw"].double()
    within(o["momentum"], mom, 2 * U32 * (mom.abs() + o["dw"].double().abs()))
    for up, u in ((o["update"], o["dw"].double() + mu * o["momentum"].double()), (o["head_update"], o["dhead"].double())):
        ref = reference(u, 5, 1e-12)
        assert (up.double() - ref).norm() <= (1.16e-2 + half_step(BF)) * ref.norm()
    # value head and the gradient of its loss
    vw = c.vw.double()
    within(o["values"], n @ vw + c.vb.double(), (K + 2) * U32 * (n.abs() @ vw.abs() + c.vb.double().abs()))
    d = o["dvalues"].double().view(-1, 1)
    e_d = half_step(BF) * d.abs()
    within(o["dvx"], d @ vw.t(), 1.01 * e_d @ vw.abs().t() + (half_step(BF) + U32) * (d @ vw.t()).abs() + 1e-30)
    within(o["dvw"], n.t() @ d, n.abs().t() @ e_d * 1.01 + 2 * M * U32 * (n.abs().t() @ d.abs()) * 1.01 + half_step(BF) * (n.t() @ d).abs())
    within(o["dvb"], d.sum(0), M * U32 * d.abs().sum(0))
    assert bool(torch.isfinite(o["vloss"]).all()) and bool(torch.isfinite(o["loss"]).all())


def outputs(c):
    return {k: v.clone() for k, v in c.out.items()}


@pytest.mark.parametrize("M,K,V", [(520, 256, 1024), (1, 72, 88), (2600, 1030 // 8 * 8, 2048)])
def test_captured_step_replays_bit_for_bit(M, K, V):
    c = Block(M, K, V, seed=M)
    c.step()
    torch.cuda.synchronize()
    eager = outputs(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for v in c.out.values():
            v.fill_(3)
        for w in c.ws.values():
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
    # new inputs in the same buffers
    c.h.copy_((c.h.float() * 0.5 + 1).to(BF))
    graph.replay()
    torch.cuda.synchronize()
    got = outputs(c)
    c.step()
    for k, v in got.items():
        assert torch.equal(c.out[k], v), k


def test_two_steps_beside_each_other():
    """Own buffers and workspaces on two streams: nothing is shared."""
    a, b = Block(900, 320, 1024, seed=3), Block(700, 456, 1288, seed=4)
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
