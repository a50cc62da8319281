"""tppo_residual_norm_fwd / _bwd against float64 forms, element by element.

Tolerances, with U = 2^-24 and k = 64 + N / 512 roundings in a sum over a row (a thread adds at most 48 elements, or every
512th, then at most 32 partial sums are added): every rounding of an intermediate is counted at its own magnitude and carried
through the formulas, and the result's own rounding is half a step of its type."""
import pytest
import torch

from dense_util import BF, DEV, F32, F64, U32, Guarded, gen, half_step, strided

pytestmark = pytest.mark.gpu
POST, PRE = 1, 2
U = U32


def within(got, ref, tol, what=""):
    d = (got.double() - ref).abs()
    assert bool((d <= tol).all()), (what, (d / tol).max().item())


def wide(t):
    return None if t is None else t.double()


def one(t):
    return torch.ones((), dtype=F64, device=DEV) if t is None else t.double()


def forward64(z, res, gate, gp, gn, alpha, eps, norms):
    """(h, n, r1, r2) and their tolerances before the rounding to the output type."""
    z, res = z.double(), res.double()
    N, k = z.shape[1], 64 + z.shape[1] / 512
    r1, e1 = torch.ones(len(z), dtype=F64, device=DEV), 0.0
    if norms & POST:
        r1, e1 = 1 / torch.sqrt((z * z).mean(1) + eps), (k / 2 + 6) * U      # half of the sum's error, rsqrt 2 ulp
    c = one(gate) * one(gp)
    u = z * r1[:, None] * c
    h = alpha * res + u
    eh = u.abs() * (e1 + 4 * U) + 2 * U * (alpha * res).abs() + U * h.abs()
    n = r2 = en = e2 = None
    if norms & PRE:
        s = (h * h).sum(1)
        r2 = 1 / torch.sqrt(s / N + eps)
        e2 = (k / 2 + 6) * U + (h.abs() * eh).sum(1) / s.clamp_min(1e-300)
        n = h * r2[:, None] * one(gn)
        en = (r2[:, None] * one(gn)).abs() * (eh + h.abs() * (e2[:, None] + 3 * U))
    return h, n, r1, r2, eh, en, e1, e2


def backward64(dh, dn, z, h, gate, gp, gn, r1, r2, alpha, norms):
    """The gradients and their tolerances before the rounding to the output type (column sums: tolerances of sums over
    all rows, M + 8 roundings)."""
    z = z.double()
    M, N = z.shape
    k = (64 + N / 512) * U
    zero = torch.zeros_like(z)
    d0 = zero if dh is None else dh.double()
    r1 = torch.ones(M, 1, dtype=F64, device=DEV) if r1 is None else r1.double()[:, None]
    c = one(gate) * one(gp)
    w = z * c
    if norms & PRE:
        h, dn, r2 = h.double(), dn.double(), r2.double()[:, None]
        a2 = dn * one(gn)
        k2 = r2 ** 3 * (a2 * h).sum(1, keepdim=True) / N
        ek2 = r2 ** 3 / N * k * (a2 * h).abs().sum(1, keepdim=True) + 6 * U * k2.abs()
        d = d0 + r2 * a2 - k2 * h
        ed = 4 * U * (d0.abs() + r2 * a2.abs() + (k2 * h).abs()) + ek2 * h.abs()
        plus = d0.abs() + r2 * a2.abs()
    else:
        h, k2, ek2, d, ed, plus = zero, 0.0, 0.0, d0, zero, d0.abs()
    a = d * c
    if norms & POST:
        k1 = r1 ** 3 * (a * z).sum(1, keepdim=True) / N
        hw = (h * w).abs().sum(1, keepdim=True)
        ek1 = r1 ** 3 / N * (k * (plus * w.abs()).sum(1, keepdim=True) + (abs(k2) * (k + 6 * U) + ek2) * hw) + 8 * U * k1.abs()
        dz = r1 * a - k1 * z
        edz = r1 * c.abs() * (ed + 5 * U * d.abs()) + ek1 * z.abs() + 3 * U * (k1 * z).abs()
    else:
        dz, edz = a, c.abs() * (ed + 4 * U * d.abs())
    zz = z * r1
    dres, edres = alpha * d, abs(alpha) * (ed + 2 * U * d.abs())
    dg = d * zz * one(gp)
    edg = (zz * one(gp)).abs() * (ed + 5 * U * d.abs())
    m = (M + 8) * U
    out = dict(dz=(dz, edz), dresidual=(dres, edres))
    row = gate is not None and gate.dim() == 1
    if row:
        out["dgate"] = (dg.sum(0), edg.sum(0) + m * dg.abs().sum(0))
    elif gate is not None:
        out["dgate"] = (dg, edg)
    if norms & POST:
        g = d * one(gate) * zz
        out["dgamma_post"] = (g.sum(0), ((one(gate) * zz).abs() * (ed + 5 * U * d.abs())).sum(0) + m * g.abs().sum(0))
    if norms & PRE:
        g = dn * h * r2
        out["dgamma_pre"] = (g.sum(0), (m + 4 * U) * g.abs().sum(0))
    return out


def inputs(M, N, dtype, gate, norms, pdtype=None, seed=0):
    g = gen(seed + 7 * M + N)
    r = lambda *s, scale=1.0, to=dtype: (scale * torch.randn(s, generator=g, device=DEV)).to(to)
    p = pdtype or dtype
    c = dict(z=r(M, N, scale=2.0), res=r(M, N), gate={"none": None, "row": r(N, scale=0.5, to=p), "full": torch.rand((M, N), generator=g, device=DEV).to(dtype)}[gate],
             gp=(1 + 0.2 * r(N, to=F32)).to(p) if norms & POST else None, gn=(1 + 0.2 * r(N, to=F32)).to(p) if norms & PRE else None,
             dh=r(M, N, scale=1e-2), dn=r(M, N, scale=1e-2) if norms & PRE else None, alpha=0.75, eps=1e-6, norms=norms)
    return c


def run(c, left=0, right=0, in_place=False, dh=True):
    """Forward and backward; every output checked element by element and for writes outside it."""
    from paper_2506_15050_b200 import binding as b
    M, N = c["z"].shape
    dt, norms = c["z"].dtype, c["norms"]
    view = (lambda t: None if t is None else t if t.dim() == 1 else strided(t, left, right)) if left or right else (lambda t: t)
    z, res, gate, dn = (view(c[k]) for k in ("z", "res", "gate", "dn"))
    d0 = view(c["dh"]) if dh else None
    new = lambda: Guarded(M, N, dt, left, right)
    h, n, dz, dres, dg = (new() for _ in range(5))
    vec = lambda t: None if t is None else torch.full_like(t, float("nan"))
    r1 = torch.full((M,), float("nan"), device=DEV) if norms & POST else None
    r2 = torch.full((M,), float("nan"), device=DEV) if norms & PRE else None
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV)
    ws.fill_(0xff)
    if in_place:
        h.t.copy_(res)
        n.t.copy_(z)
        b.tppo_residual_norm_fwd(n.t, h.t, gate, c["gp"], c["gn"], c["alpha"], c["eps"], norms, h.t, n.t, r1, r2, st)
    else:
        b.tppo_residual_norm_fwd(z, res, gate, c["gp"], c["gn"], c["alpha"], c["eps"], norms, h.t, n.t if norms & PRE else None, r1, r2, st)
    assert int(st) == 0
    rh, rn, q1, q2, eh, en, e1, e2 = forward64(z, res, gate, c["gp"], c["gn"], c["alpha"], c["eps"], norms)
    hs = half_step(dt)
    within(h.t, rh, eh + hs * rh.abs() + 1e-37, "h")
    if norms & POST:
        within(r1, q1, (e1 + U) * q1, "r1")
    if norms & PRE:
        within(r2, q2, (e2 + U) * q2, "r2")
        within(n.t, rn, en + (hs + U) * rn.abs() + 1e-37, "n")
    h.check(), n.check()
    full = gate is not None and gate.dim() == 2
    dgate = dg.t if full else vec(gate)
    dgp, dgn = vec(c["gp"]), vec(c["gn"])
    hh = h.t
    if in_place:
        if d0 is not None:
            dres.t.copy_(d0)
            d0 = dres.t
        if norms & PRE:
            dz.t.copy_(dn)
            dn = dz.t
    given = dict(d0=None if d0 is None else d0.clone(), dn=None if dn is None else dn.clone())
    b.tppo_residual_norm_bwd(d0, dn, z, hh, gate, c["gp"], c["gn"], r1, r2, c["alpha"], norms, dz.t, dres.t, dgate, dgp, dgn, st, ws)
    assert int(st) == 0
    ref = backward64(given["d0"], given["dn"], z, hh, gate, c["gp"], c["gn"], r1, r2, c["alpha"], norms)
    got = dict(dz=dz.t, dresidual=dres.t, dgate=dgate, dgamma_post=dgp, dgamma_pre=dgn)
    for k, (v, tol) in ref.items():
        within(got[k], v, tol + (half_step(got[k].dtype) + U) * v.abs() + 1e-37, k)
    dz.check(), dres.check()
    if full:
        dg.check()
    return h.t, got


SIZES = [(1, 1), (1, 8), (3, 7), (1, 5120), (2, 257), (150, 8), (700, 64), (33, 515), (300, 1024), (611, 1283), (200, 2048), (149, 5121), (5, 8191),
         (40, 10240), (17, 16384), (3, 20000), (2, 40001)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N", SIZES)
def test_sizes(M, N, dtype):
    run(inputs(M, N, dtype, "row", 3))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("norms", [0, POST, PRE, 3])
@pytest.mark.parametrize("gate", ["none", "row", "full"])
@pytest.mark.parametrize("M,N", [(160, 520), (65, 1031), (9, 12296)])
def test_forms(M, N, gate, norms, dtype):
    run(inputs(M, N, dtype, gate, norms))


@pytest.mark.parametrize("dtype,left,right", [(BF, 1, 0), (BF, 3, 2), (BF, 8, 8), (F32, 1, 2), (F32, 4, 4), (BF, 0, 5)])
@pytest.mark.parametrize("M,N", [(37, 640), (210, 1285), (6, 9000)])
def test_strides_and_alignment(M, N, dtype, left, right):
    run(inputs(M, N, dtype, "full", 3), left, right)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_matrices_that_start_at_different_places(dtype):
    """Each matrix at an offset and stride of its own."""
    from paper_2506_15050_b200 import binding as b
    M, N = 70, 700
    c = inputs(M, N, dtype, "full", 3)
    z, res, gate = strided(c["z"], 1, 2), strided(c["res"], 0, 3), strided(c["gate"], 2, 0)
    h, n = Guarded(M, N, dtype, 3, 1), Guarded(M, N, dtype, 0, 0)
    r1, r2, st = torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_residual_norm_fwd(z, res, gate, c["gp"], c["gn"], 0.75, 1e-6, 3, h.t, n.t, r1, r2, st)
    rh, rn, _, _, eh, en, _, _ = forward64(z, res, gate, c["gp"], c["gn"], 0.75, 1e-6, 3)
    within(h.t, rh, eh + half_step(dtype) * rh.abs())
    within(n.t, rn, en + (half_step(dtype) + U) * rn.abs())
    dz, dres, dg = Guarded(M, N, dtype, 1, 0), Guarded(M, N, dtype, 0, 1), Guarded(M, N, dtype, 5, 5)
    dgp, dgn = torch.empty_like(c["gp"]), torch.empty_like(c["gn"])
    b.tppo_residual_norm_bwd(strided(c["dh"], 4, 1), c["dn"], z, h.t, gate, c["gp"], c["gn"], r1, r2, 0.75, 3, dz.t, dres.t, dg.t, dgp, dgn, st,
                             b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV))
    ref = backward64(c["dh"], c["dn"], z, h.t, gate, c["gp"], c["gn"], r1, r2, 0.75, 3)
    for got, k in ((dz.t, "dz"), (dres.t, "dresidual"), (dg.t, "dgate"), (dgp, "dgamma_post"), (dgn, "dgamma_pre")):
        within(got, ref[k][0], ref[k][1] + (half_step(dtype) + U) * ref[k][0].abs() + 1e-37, k)
    for g in (h, n, dz, dres, dg):
        g.check()
    assert int(st) == 0


@pytest.mark.parametrize("M,N", [(50, 1024), (31, 333), (4, 20000)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_place_gives_the_same(M, N, dtype):
    c = inputs(M, N, dtype, "row", 3)
    h, a = run(c)
    h2, b = run(c, in_place=True)        # against float64
    if N % 8:                            # the guarded outputs start elsewhere in a 16-byte piece than the inputs, so that the
        return                           # first run sums its rows in another order
    assert torch.equal(h, h2)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_parameters_of_the_other_type_and_no_dh():
    run(inputs(90, 700, BF, "row", 3, pdtype=F32))
    run(inputs(90, 700, F32, "row", 3, pdtype=BF))
    run(inputs(90, 704, BF, "full", 3, pdtype=F32), dh=False)
    run(inputs(3, 20000, BF, "none", 3), dh=False)


@pytest.mark.parametrize("M,N", [(20, 256), (300, 1285), (6, 20000)])
def test_outputs_left_out(M, N):
    from paper_2506_15050_b200 import binding as b
    c = inputs(M, N, F32, "row", 3)
    h, n, r1, r2 = torch.empty_like(c["z"]), torch.empty_like(c["z"]), torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    ws = b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV)
    b.tppo_residual_norm_fwd(c["z"], c["res"], c["gate"], c["gp"], c["gn"], 0.75, 1e-6, 3, h, n, r1, r2, None)
    shapes = dict(dz=c["z"], dresidual=c["z"], dgate=c["gate"], dgamma_post=c["gp"], dgamma_pre=c["gn"])
    def call(names):
        o = {k: torch.empty_like(v) if k in names else None for k, v in shapes.items()}
        b.tppo_residual_norm_bwd(c["dh"], c["dn"], c["z"], h, c["gate"], c["gp"], c["gn"], r1, r2, 0.75, 3, o["dz"], o["dresidual"], o["dgate"],
                                 o["dgamma_post"], o["dgamma_pre"], None, ws)
        return o
    all_of = call(shapes)
    for name in all_of:
        assert torch.equal(call([name])[name], all_of[name]), name


@pytest.mark.parametrize("dtype,M,N", [(BF, 40, 520), (F32, 40, 519), (BF, 9, 20000), (BF, 40, 521)])
def test_rows_without_statistics(dtype, M, N):
    """NaN, infinities, sums beyond fp32, and a row of zeros without eps: such rows are 0, the others as they were."""
    from paper_2506_15050_b200 import binding as b
    c = inputs(M, N, dtype, "full", 3)
    clean, x = torch.empty_like(c["z"]), torch.empty_like(c["z"])
    b.tppo_residual_norm_fwd(c["z"], c["res"], c["gate"], c["gp"], c["gn"], 0.75, 1e-6, 3, clean, x, None, None, None)
    bad = {0: ("z", float("nan")), 1: ("res", float("inf")), 2: ("gate", float("-inf")), 3: ("z", 3e38), 4: ("res", 3e38)}
    for r, (k, v) in bad.items():
        c[k][r, N // 2] = v
    h, n, r1, r2 = torch.empty_like(c["z"]), torch.empty_like(c["z"]), torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_residual_norm_fwd(c["z"], c["res"], c["gate"], c["gp"], c["gn"], 0.75, 1e-6, 3, h, n, r1, r2, st)
    assert int(st) == b.DEV_NONFINITE
    for t in (h, n, r1, r2):
        assert not bool(t[:5].any())
    assert torch.equal(h[5:], clean[5:])
    # backward: rows with an rstd of 0 are silent, a NaN in a gradient is not
    st.zero_()
    o = dict(dz=torch.empty_like(h), dresidual=torch.empty_like(h), dgate=torch.empty_like(h), dgamma_post=torch.empty_like(c["gp"]),
             dgamma_pre=torch.empty_like(c["gn"]))
    ws = b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV)
    call = lambda: b.tppo_residual_norm_bwd(c["dh"], c["dn"], c["z"], h, c["gate"], c["gp"], c["gn"], r1, r2, 0.75, 3, o["dz"], o["dresidual"], o["dgate"],
                                            o["dgamma_post"], o["dgamma_pre"], st, ws)
    call()
    assert int(st) == 0
    c["dh"][6, 3], c["dn"][7, 4] = float("nan"), float("inf")
    call()
    assert int(st) == b.DEV_NONFINITE
    silent = [0, 1, 2, 3, 4, 6, 7]
    for k in ("dz", "dresidual", "dgate"):
        assert not bool(o[k][silent].any()), k
    keep = [r for r in range(M) if r not in silent]
    ref = backward64(c["dh"][keep], c["dn"][keep], c["z"][keep], h[keep], c["gate"][keep], c["gp"], c["gn"], r1[keep], r2[keep], 0.75, 3)
    for k, v in o.items():
        got = v if k.startswith("dgamma") else v[keep]
        within(got, ref[k][0], ref[k][1] + (half_step(dtype) + U) * ref[k][0].abs() + 1e-37, k)


def test_zero_rows_and_eps():
    from paper_2506_15050_b200 import binding as b
    z, res = torch.zeros((3, 64), device=DEV), torch.ones((3, 64), device=DEV)
    h, n, r1, r2 = torch.empty_like(z), torch.empty_like(z), torch.empty(3, device=DEV), torch.empty(3, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_residual_norm_fwd(z, res, None, None, None, 1.0, 1e-6, 3, h, n, r1, r2, st)
    assert int(st) == 0 and torch.equal(h, res)
    b.tppo_residual_norm_fwd(z, res, None, None, None, 1.0, 0.0, 3, h, n, r1, r2, st)
    assert int(st) == b.DEV_NONFINITE and not bool(h.any()) and not bool(r1.any())
    # a block whose output cancels the stream: the norm of what is left is right
    g = gen(5)
    res = torch.randn((64, 5120), generator=g, device=DEV)
    left = 1e-3 * torch.randn((64, 5120), generator=g, device=DEV)
    z = left - res
    h, n, r1, r2 = torch.empty_like(z), torch.empty_like(z), None, torch.empty(64, device=DEV)
    b.tppo_residual_norm_fwd(z, res, None, None, None, 1.0, 0.0, PRE, h, n, r1, r2, st)
    ref = forward64(z, res, None, None, None, 1.0, 0.0, PRE)
    within(r2, ref[3], (ref[7] + U) * ref[3])


def test_empty_and_repeatable():
    from paper_2506_15050_b200 import binding as b
    e = torch.empty((0, 24), dtype=BF, device=DEV)
    v = torch.empty(0, device=DEV)
    g = torch.full((24,), 7.0, dtype=BF, device=DEV)
    b.tppo_residual_norm_fwd(e, e, g, g, g, 1.0, 1e-6, 3, e, e, v, v, None)
    dg, dp, dn = (torch.full_like(g, 5) for _ in range(3))
    b.tppo_residual_norm_bwd(e, e, e, e, g, g, g, v, v, 1.0, 3, e, e, dg, dp, dn, None, b.workspace(b.OP_RESIDUAL_NORM, 0, 0, 0, 24, DEV))
    assert not bool(dg.any()) and not bool(dp.any()) and not bool(dn.any())
    c = inputs(3000, 1000, BF, "row", 3)
    a, b2 = run(c)[1], run(c)[1]
    for k in a:
        if a[k] is not None:
            assert torch.equal(a[k], b2[k]), k


def test_gradients_against_differences():
    """Central differences of the forward call itself, fp32, along random directions of each input."""
    from paper_2506_15050_b200 import binding as b
    M, N = 6, 96
    c = inputs(M, N, F32, "full", 3, seed=3)
    wh, wn = c["dh"] * 100, c["dn"] * 100
    def value(d):
        h, n = torch.empty_like(d["z"]), torch.empty_like(d["z"])
        b.tppo_residual_norm_fwd(d["z"], d["res"], d["gate"], d["gp"], d["gn"], 0.75, 1e-6, 3, h, n, None, None, None)
        return (h.double() * wh.double() + n.double() * wn.double()).sum()
    h, n, r1, r2 = torch.empty_like(c["z"]), torch.empty_like(c["z"]), torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    b.tppo_residual_norm_fwd(c["z"], c["res"], c["gate"], c["gp"], c["gn"], 0.75, 1e-6, 3, h, n, r1, r2, None)
    o = [torch.empty_like(c[k]) for k in ("z", "res", "gate", "gp", "gn")]
    b.tppo_residual_norm_bwd(wh, wn, c["z"], h, c["gate"], c["gp"], c["gn"], r1, r2, 0.75, 3, *o, None, b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV))
    for k, grad in zip(("z", "res", "gate", "gp", "gn"), o):
        v = torch.randn(grad.shape, generator=gen(9), device=DEV)
        step = 2.0 ** -7
        up, down = dict(c), dict(c)
        up[k], down[k] = c[k] + step * v, c[k] - step * v
        v = (up[k].double() - down[k].double()) / (2 * step)          # the step that was taken
        diff = (value(up) - value(down)) / (2 * step)
        want = (grad.double() * v).sum()
        # third derivatives of an rms norm of unit scale are O(1): step^2 of the terms' size, and the values' roundings
        size = (grad.double() * v).abs().sum()
        noise = 16 * U * ((h.double() * wh.double()).abs().sum() + (n.double() * wn.double()).abs().sum()) / step
        assert abs(diff - want) <= 4 * step ** 2 * size + noise, k


def test_more_than_two_to_the_31_elements():
    from paper_2506_15050_b200 import binding as b
    M, N = (1 << 20) + 3, 2056
    z, res = (torch.empty((M, N), dtype=BF, device=DEV) for _ in range(2))
    z.fill_(0.5), res.fill_(-0.25)
    last = inputs(5, N, BF, "row", 3)
    z[-5:], res[-5:] = last["z"], last["res"]
    h, n = torch.empty_like(z), torch.empty_like(z)
    r1, r2, st = torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_residual_norm_fwd(z, res, last["gate"], last["gp"], last["gn"], 0.75, 1e-6, 3, h, n, r1, r2, st)
    rh, rn, q1, q2, eh, en, e1, e2 = forward64(last["z"], last["res"], last["gate"], last["gp"], last["gn"], 0.75, 1e-6, 3)
    within(h[-5:], rh, eh + half_step(BF) * rh.abs())
    within(n[-5:], rn, en + (half_step(BF) + U) * rn.abs())
    assert torch.equal(h[0], h[M - 6]) and torch.equal(n[0], n[M // 2])
    dh, dn = torch.zeros_like(z), torch.zeros_like(z)
    dh[-5:], dn[-5:] = last["dh"], last["dn"]
    dz, dres = res, torch.empty_like(z)
    dg, dgp, dgn = (torch.empty_like(last["gp"]) for _ in range(3))
    b.tppo_residual_norm_bwd(dh, dn, z, h, last["gate"], last["gp"], last["gn"], r1, r2, 0.75, 3, dz, dres, dg, dgp, dgn, st,
                             b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV))
    ref = backward64(last["dh"], last["dn"], last["z"], h[-5:], last["gate"], last["gp"], last["gn"], r1[-5:], r2[-5:], 0.75, 3)
    for got, k in ((dz[-5:], "dz"), (dres[-5:], "dresidual"), (dg, "dgate"), (dgp, "dgamma_post"), (dgn, "dgamma_pre")):
        within(got, ref[k][0], ref[k][1] + 1e-6 * ref[k][0].abs() + (half_step(BF) + U) * ref[k][0].abs() + 1e-37, k)
    assert not bool(dz[:-5].any()) and not bool(dres[:-5].any()) and int(st) == 0


@pytest.mark.parametrize("dtype,M,N", [(BF, 40, 520), (F32, 40, 519), (BF, 9, 20000)])
@pytest.mark.parametrize("norms", [0, POST, 3])
@pytest.mark.parametrize("which,value", [("gate", float("inf")), ("gate", float("nan")), ("gp", float("-inf")), ("gp", float("nan"))])
def test_a_row_parameter_that_is_not_finite_gives_zeros(dtype, M, N, norms, which, value):
    """It enters every row, so no row contributes: all gradients are 0, the parameter's own among them."""
    from paper_2506_15050_b200 import binding as b
    if which == "gp" and not norms & POST:
        return
    c = inputs(M, N, dtype, "row", norms)
    c[which][N // 3] = value
    h, n = torch.empty_like(c["z"]), torch.empty_like(c["z"]) if norms & PRE else None
    r1, r2 = torch.empty(M, device=DEV) if norms & POST else None, torch.empty(M, device=DEV) if norms & PRE else None
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_residual_norm_fwd(c["z"], c["res"], c["gate"], c["gp"], c["gn"], 0.75, 1e-6, norms, h, n, r1, r2, st)
    assert int(st) == b.DEV_NONFINITE and not bool(h.any())
    o = [None if c[k] is None else torch.full_like(c[k], 7) for k in ("z", "res", "gate", "gp", "gn")]
    b.tppo_residual_norm_bwd(c["dh"], c["dn"], c["z"], h, c["gate"], c["gp"], c["gn"], r1, r2, 0.75, norms, *o, st,
                             b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV))
    assert not any(bool(t.ne(0).any()) for t in o if t is not None)
    # nor does it without a single row
    e, v = c["z"][:0], torch.empty(0, device=DEV)
    o = [None if c[k] is None else torch.full_like(c[k], 7) for k in ("gate", "gp", "gn")]
    b.tppo_residual_norm_bwd(e, e if norms & PRE else None, e, e, c["gate"], c["gp"], c["gn"], v if norms & POST else None, v if norms & PRE else None,
                             0.75, norms, e, e, *o, None, b.workspace(b.OP_RESIDUAL_NORM, 0, 0, 0, N, DEV))
    assert not any(bool(t.ne(0).any()) for t in o if t is not None)


@pytest.mark.parametrize("dtype,N", [(F32, 64), (BF, 519), (F32, 5120), (BF, 20000)])
@pytest.mark.parametrize("norms", [POST, PRE])
def test_small_rows_are_right_or_refused(dtype, N, norms):
    """Without eps, a mean square below fp32's normal range has lost bits: such a row is 0 and raises a bit.  From 2^-126 on its
    error of up to 2^-150 is within half a rounding of the mean, U / 4 of the rstd."""
    from paper_2506_15050_b200 import binding as b
    e = torch.arange(-76, -50, device=DEV)
    z = (torch.randn((len(e), N), generator=gen(N), device=DEV) * torch.exp2(e.float())[:, None]).to(dtype)
    res = torch.zeros_like(z)
    mean = (z.double() ** 2).mean(1)
    tiny, clear = mean < 2.0 ** -126 * (1 - 2.0 ** -20), mean > 2.0 ** -126 * (1 + 2.0 ** -20)
    assert bool(tiny.any()) and bool(clear.any()) and bool((tiny | clear).all())
    for eps in (0.0, 2.0 ** -100):
        h, n, r, st = torch.empty_like(z), torch.empty_like(z), torch.empty(len(e), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        post = norms & POST
        b.tppo_residual_norm_fwd(z, res, None, None, None, 1.0, eps, norms, h, None if post else n, r if post else None, None if post else r, st)
        rh, rn, q1, q2, eh, en, e1, e2 = forward64(z, res, None, None, None, 1.0, eps, norms)
        bad = tiny if eps == 0 else torch.zeros_like(tiny)
        assert int(st) == (b.DEV_NONFINITE if eps == 0 else 0)
        out, want, tol, q, eq = (h, rh, eh, q1, e1) if post else (n, rn, en, q2, e2)
        assert not bool(out[bad].any()) and not bool(h[bad].any()) and not bool(r[bad].any())
        eq = torch.as_tensor(eq, device=DEV).expand(len(e))
        within(r[~bad], q[~bad], ((eq + 1.25 * U) * q)[~bad], "rstd")
        within(out[~bad], want[~bad], (tol + (half_step(dtype) + 1.25 * U) * want.abs() + 1e-37)[~bad], "out")


@pytest.mark.parametrize("dtype,N", [(F32, 64), (F32, 519), (F32, 5120), (F32, 20000), (BF, 520), (BF, 5120), (BF, 5121), (BF, 12001)])
@pytest.mark.parametrize("norms", [POST, PRE, 3])
@pytest.mark.parametrize("ez,er,eg", [(0, 0, -20), (20, -20, -80), (-20, 20, -80), (50, 0, -20), (55, 3, -60), (-50, 0, -20), (-50, -45, 10), (0, 50, -40), (50, 50, -30), (40, -40, -60),
                                      (-60, 30, -60)])
def test_gradients_of_large_and_small_rows(dtype, N, norms, ez, er, eg):
    """Rows of scale 2^ez and 2^er, gradients of scale 2^eg: the result is in fp32's range, and so is every step towards it."""
    from paper_2506_15050_b200 import binding as b
    M = 700 if (dtype, N) == (BF, 5120) else 40            # several rows for each group of a block
    r = lambda e, seed: (torch.randn((M, N), generator=gen(seed + N), device=DEV) * 2.0 ** e).to(dtype)
    z, res = r(ez, 1), r(er, 2)
    z[::3] *= 0.5                                          # rows on both sides of a power of two
    h, n = torch.empty_like(z), torch.empty_like(z) if norms & PRE else None
    r1, r2 = torch.empty(M, device=DEV) if norms & POST else None, torch.empty(M, device=DEV) if norms & PRE else None
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_residual_norm_fwd(z, res, None, None, None, 1.0, 0.0, norms, h, n, r1, r2, st)
    assert int(st) == 0
    dh = (r(eg, 3) * (float(r2.median()) if norms & PRE else 1.0)).to(dtype)
    dn = r(eg, 4) if norms & PRE else None
    dz, dres = torch.empty_like(z), torch.empty_like(z)
    dgp, dgn = torch.empty(N, device=DEV) if norms & POST else None, torch.empty(N, device=DEV) if norms & PRE else None
    b.tppo_residual_norm_bwd(dh, dn, z, h, None, None, None, r1, r2, 1.0, norms, dz, dres, None, dgp, dgn, st,
                             b.workspace(b.OP_RESIDUAL_NORM, M, 0, 0, N, DEV))
    assert int(st) == 0
    ref = backward64(dh, dn, z, h, None, None, None, r1, r2, 1.0, norms)
    got = dict(dz=dz, dresidual=dres, dgamma_post=dgp, dgamma_pre=dgn)
    for k, (v, tol) in ref.items():
        within(got[k], v, tol + (half_step(got[k].dtype) + U) * v.abs() + (2.0 ** -148 if got[k].dtype == F32 else 2.0 ** -133), k)


@pytest.mark.parametrize("dtype,M,N", [(BF, 70, 520), (F32, 70, 519), (BF, 9, 20000), (F32, 5, 30001)])
def test_joined_stream_in_the_place_of_the_block_output(dtype, M, N):
    from paper_2506_15050_b200 import binding as b
    c = inputs(M, N, dtype, "full", 3)
    out = []
    for place in (False, True):
        z = c["z"].clone()
        h, n, r1, r2 = z if place else torch.empty_like(z), torch.empty_like(z), torch.empty(M, device=DEV), torch.empty(M, device=DEV)
        b.tppo_residual_norm_fwd(z, c["res"], c["gate"], c["gp"], c["gn"], 0.75, 1e-6, 3, h, n, r1, r2, None)
        out.append((h, n, r1, r2))
    rh, rn, _, _, eh, en, _, _ = forward64(c["z"], c["res"], c["gate"], c["gp"], c["gn"], 0.75, 1e-6, 3)
    within(out[1][0], rh, eh + half_step(dtype) * rh.abs(), "h")
    within(out[1][1], rn, en + (half_step(dtype) + U) * rn.abs(), "n")
    assert all(torch.equal(a, o) for a, o in zip(*out))
