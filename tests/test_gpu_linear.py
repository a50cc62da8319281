"""tppo_linear_fwd / _bwd.

Whole numbers: with small integers as operands every product and sum is exact in fp32, so an fp32
output has to be equal to the float64 product and a bf16 output to its one rounding -- any index or
tail error shows.  Real numbers: a sum of K products in fp32 is off by at most K 2^-23 times the sum
of magnitudes (2^-23: a tensor core may cut instead of round); what the epilogue adds is written at
each check."""
import math

import pytest
import torch

from dense_util import BF, DEV, F32, F64, Guarded, U32, act64, gen, half_step, slope64, strided

pytestmark = pytest.mark.gpu


def whole(g, *shape, top=4):
    return torch.randint(-top, top + 1, shape, generator=g, device=DEV).to(BF)


def workspace(M, K, N, copies=0):
    from paper_2506_15050_b200 import binding as b
    ws = b.workspace(b.OP_LINEAR, M, K, copies, N, DEV)
    ws.fill_(0xff)
    return ws


SIZES = [(1, 1, 1), (200, 1, 100), (5000, 1, 2000), (1, 8, 8), (1, 64, 256), (1, 5120, 640), (2, 5, 3), (5, 63, 7), (16, 64, 128), (17, 65, 129), (31, 200, 33),
         (33, 515, 130), (64, 128, 64), (65, 72, 1000), (100, 1000, 40), (128, 64, 264), (129, 8, 257), (250, 77, 510),
         (1000, 136, 1), (777, 300, 2), (1001, 515, 777), (300, 1024, 1024),
         (2500, 72, 2000), (2561, 130, 2049), (19000, 24, 130),
         (5000, 1000, 1000), (4100, 1004, 1501)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_whole_numbers(M, K, N):
    from paper_2506_15050_b200 import binding as b
    g = gen(M + 7 * K + 31 * N)
    x, w = whole(g, M, K), whole(g, K, N)
    bias, residual = whole(g, N, top=9), whole(g, M, N, top=9)
    ws, status = workspace(M, K, N), torch.zeros(1, dtype=torch.int32, device=DEV)
    z = x.double() @ w.double()
    y = Guarded(M, N, F32)
    b.tppo_linear_fwd(x, w, None, b.ACT_NONE, None, y.t, None, status, ws)
    assert torch.equal(y.t.double(), z)
    y.check()
    zb = z + bias.double()
    yb, pre = Guarded(M, N, BF), Guarded(M, N, BF)
    b.tppo_linear_fwd(x, w, bias, b.ACT_RELU, residual, yb.t, pre.t, status, ws)
    assert torch.equal(yb.t, (torch.relu(zb) + residual.double()).to(BF)) and torch.equal(pre.t, zb.to(BF))
    yb.check()
    pre.check()
    assert int(status) == 0

    # backward: slopes 0 and 1, whole dy
    dy = whole(g, M, N)
    dz = dy.double() * (pre.t.double() > 0)
    dx, dw = Guarded(M, K, BF), Guarded(K, N, BF)
    db = torch.full((N,), float("nan"), device=DEV)
    b.tppo_linear_bwd(dy, x, w, b.ACT_RELU, pre.t, dx.t, dw.t, db, status, ws)
    assert torch.equal(dx.t, (dz @ w.double().t()).to(BF)) and torch.equal(dw.t, (x.double().t() @ dz).to(BF))
    assert torch.equal(db.double(), dz.sum(0))
    dx.check()
    dw.check()
    # without an activation, fp32 dy, bf16 dbias; any subset of the outputs
    dx2, dw2, db2 = torch.empty_like(x), torch.empty_like(w), torch.empty(N, dtype=BF, device=DEV)
    b.tppo_linear_bwd(dy.float(), x, w, b.ACT_NONE, None, dx2, None, None, status, ws)
    b.tppo_linear_bwd(dy, x, w, b.ACT_NONE, None, None, dw2, None, status, ws)
    b.tppo_linear_bwd(dy, x, w, b.ACT_NONE, None, None, None, db2, status, ws)
    assert torch.equal(dx2, (dy.double() @ w.double().t()).to(BF)) and torch.equal(dw2, (x.double().t() @ dy.double()).to(BF))
    assert torch.equal(db2, dy.double().sum(0).to(BF))
    assert int(status) == 0


@pytest.mark.parametrize("left,right", [(0, 8), (8, 16), (1, 0), (0, 3), (5, 3)])
@pytest.mark.parametrize("M,K,N", [(3, 64, 40), (70, 72, 136), (130, 61, 75), (2500, 64, 2000)])
def test_strided_rows_of_any_alignment(M, K, N, left, right):
    from paper_2506_15050_b200 import binding as b
    g = gen(left + 10 * right + M)
    x, w, r, dy = whole(g, M, K), whole(g, K, N), whole(g, M, N), whole(g, M, N)
    ws, status = workspace(M, K, N, 1), torch.zeros(1, dtype=torch.int32, device=DEV)
    xs, wsd, rs, ds = (strided(t, left, right) for t in (x, w, r, dy))
    y, pre = Guarded(M, N, BF, left, right), Guarded(M, N, BF, right, left)
    b.tppo_linear_fwd(xs, wsd, None, b.ACT_RELU, rs, y.t, pre.t, status, ws)
    z = x.double() @ w.double()
    assert torch.equal(y.t, (torch.relu(z) + r.double()).to(BF)) and torch.equal(pre.t, z.to(BF))
    dz = dy.double() * (pre.t.double() > 0)
    dx, dw, db = Guarded(M, K, BF, left, right), Guarded(K, N, BF, right, left), torch.empty(N, device=DEV)
    b.tppo_linear_bwd(ds, xs, wsd, b.ACT_RELU, pre.t, dx.t, dw.t, db, status, ws)
    assert torch.equal(dx.t, (dz @ w.double().t()).to(BF)) and torch.equal(dw.t, (x.double().t() @ dz).to(BF))
    b.tppo_linear_bwd(ds, xs, wsd, b.ACT_NONE, None, dx.t, dw.t, db, status, ws)
    assert torch.equal(dx.t, (dy.double() @ w.double().t()).to(BF)) and torch.equal(db.double(), dy.double().sum(0))
    for o in (y, pre, dx, dw):
        o.check()
    # the residual may be the output
    acc = Guarded(M, N, BF, left, right)
    acc.t.copy_(r)
    b.tppo_linear_fwd(xs, wsd, None, b.ACT_NONE, acc.t, acc.t, None, status, ws)
    assert torch.equal(acc.t, (z + r.double()).to(BF))
    assert int(status) == 0


def act_tol(z, act, e_z):
    """The activations' slopes lie within 1.13 in magnitude; evaluated in fp32 from expf / erff (2 ulp
    each) and fewer than ten further roundings of values of at most |z|: 16 u (|z| + 1e-6)."""
    return 1.13 * e_z + 16 * U32 * (z.abs() + 1e-6)


@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("M,K,N", [(1, 300, 200), (40, 129, 77), (200, 512, 264), (2500, 96, 2000)])
def test_real_numbers(M, K, N, act):
    from paper_2506_15050_b200 import binding as b
    g = gen(act + K)
    x = torch.randn((M, K), generator=g, device=DEV).to(BF)
    w = (torch.randn((K, N), generator=g, device=DEV) * 2 * K ** -0.5).to(BF)
    bias = torch.randn(N, generator=g, device=DEV)
    r = torch.randn((M, N), generator=g, device=DEV).to(BF)
    ws, status = workspace(M, K, N), torch.zeros(1, dtype=torch.int32, device=DEV)
    z = x.double() @ w.double() + bias.double()
    e_z = (K + 2) * 2 * U32 * (x.double().abs() @ w.double().abs() + bias.double().abs())
    for dt in (F32, BF):
        y, pre = torch.empty((M, N), dtype=dt, device=DEV), torch.empty((M, N), dtype=BF, device=DEV)
        b.tppo_linear_fwd(x, w, bias, act, r, y, pre, status, ws)
        ref = act64(z, act) + r.double()
        tol = act_tol(z, act, e_z) + ref.abs() * (half_step(dt) + U32)
        assert bool(((y.double() - ref).abs() <= tol).all()), ((y.double() - ref).abs() / tol).max().item()
        assert bool(((pre.double() - z).abs() <= e_z + z.abs() * half_step(BF)).all())
    # backward from that preact: dz = dy act'(z), its bf16 rounding half a step; the slope 24 u
    dy = torch.randn((M, N), generator=g, device=DEV)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV)
    b.tppo_linear_bwd(dy, x, w, act, pre if act else None, dx, dw, db, status, ws)
    dz = dy.double() * (slope64(pre.double(), act) if act else 1.0)
    e_dz = dz.abs() * half_step(BF) + 24 * U32 * dy.double().abs() * (1 + pre.double().abs())
    for got, ref, mag, err, n in ((dx, dz @ w.double().t(), dz.abs() @ w.double().abs().t(), e_dz @ w.double().abs().t(), N),
                                  (dw, x.double().t() @ dz, x.double().abs().t() @ dz.abs(), x.double().abs().t() @ e_dz, M)):
        tol = err * (1 + half_step(BF)) + n * 2 * U32 * mag * 1.01 + ref.abs() * half_step(BF)
        assert bool(((got.double() - ref).abs() <= tol).all()), ((got.double() - ref).abs() / tol).max().item()
    tol = (24 * U32 * dy.double().abs() * (1 + pre.double().abs())).sum(0) + (M / 8 + 300) * U32 * dz.abs().sum(0)
    assert bool(((db.double() - dz.sum(0)).abs() <= tol).all())
    assert int(status) == 0


def test_gradient_against_differences():
    """Central differences of <dy, y> in float64.  The gradients hold bf16 roundings (2^-8 of a value each
    for dz and the output), so the directional derivative is off by 2^-7 of the sum of magnitudes at most."""
    from paper_2506_15050_b200 import binding as b
    M, K, N = 24, 40, 56
    g = gen(3)
    x, w = torch.randn((M, K), generator=g, device=DEV).to(BF), (torch.randn((K, N), generator=g, device=DEV) / 4).to(BF)
    bias, dy = torch.randn(N, generator=g, device=DEV), torch.randn((M, N), generator=g, device=DEV)
    for act in (2, 3, 4):
        pre, y = torch.empty((M, N), dtype=BF, device=DEV), torch.empty((M, N), device=DEV)
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV)
        ws = workspace(M, K, N)
        b.tppo_linear_fwd(x, w, bias, act, None, y, pre, None, ws)
        b.tppo_linear_bwd(dy, x, w, act, pre, dx, dw, db, None, ws)
        f = lambda x, w, c: (dy.double() * act64(x @ w + c, act)).sum()
        args = [x.double(), w.double(), bias.double()]
        for k, grad in enumerate((dx, dw, db)):
            v = torch.randn(args[k].shape, generator=g, device=DEV, dtype=F64)
            lo, hi = list(args), list(args)
            lo[k], hi[k] = args[k] - 1e-4 * v, args[k] + 1e-4 * v
            want, got = (f(*hi) - f(*lo)) / 2e-4, (grad.double() * v).sum()
            # preact's own rounding moves act' by at most 1.2 |z| 2^-8: |z| < 8 here
            assert abs(want - got) <= 2.0 ** -5 * (grad.double() * v).abs().sum()


def test_far_activations_and_slopes():
    """Large |z|: no overflow in between, tails exactly 0 or z."""
    from paper_2506_15050_b200 import binding as b
    z = torch.tensor([-3e38, -1e20, -300.0, -90.0, -20.0, -5.0, 0.0, 5.0, 20.0, 90.0, 300.0, 1e20, 3e38], device=DEV).to(BF)
    x, w = torch.ones((1, 1), dtype=BF, device=DEV), z[None, :].contiguous()
    N = z.numel()
    ws = workspace(1, 1, N)
    for act in range(5):
        y, status = torch.empty((1, N), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        b.tppo_linear_fwd(x, w, None, act, None, y, None, status, ws)
        ref = act64(z.double(), act)
        if act == 3:
            ref = torch.where(z.double().abs() > 1e3, torch.relu(z.double()), ref)
        assert bool(((y[0].double() - ref).abs() <= act_tol(z.double(), act, 0.0) + 1e-38).all())
        assert bool((y[0][z < -100] == 0).all()) or act == 0
        db, dy = torch.empty(N, device=DEV), torch.ones((1, N), device=DEV)
        b.tppo_linear_bwd(dy, x, w, act, z[None, :].contiguous(), None, None, db, status, ws)
        far = z.double().clamp(-200, 200)                  # the slopes are 0 and 1 there already
        ref = slope64(far, act) if act else torch.ones(N, dtype=F64, device=DEV)
        assert bool(((db.double() - ref).abs() <= 24 * U32 * (1 + far.abs()) * 1.2).all())
        assert int(status) == 0


def test_elements_that_are_not_finite():
    from paper_2506_15050_b200 import binding as b
    for M, N in ((20, 48), (2500, 2000)):
        K, g = 64, gen(1)
        x, w, dy = whole(g, M, K), whole(g, K, N), whole(g, M, N)
        x[3, 5], w[7, 11] = float("nan"), float("inf")
        ws, status = workspace(M, K, N), torch.zeros(1, dtype=torch.int32, device=DEV)
        y, pre = torch.empty((M, N), dtype=BF, device=DEV), torch.empty((M, N), dtype=BF, device=DEV)
        b.tppo_linear_fwd(x, w, None, b.ACT_NONE, None, y, pre, status, ws)
        ref = x.double() @ w.double()
        ref = torch.where(torch.isfinite(ref), ref, 0.0)
        assert torch.equal(y, ref.to(BF)) and torch.equal(pre, y) and int(status) == b.DEV_NONFINITE
        status.zero_()
        x[3, 5], w[7, 11] = 1.0, 2.0
        dy[2, 9] = float("nan")
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV)
        b.tppo_linear_bwd(dy.float(), x, w, b.ACT_NONE, None, dx, dw, db, status, ws)
        d = torch.nan_to_num(dy.double(), nan=0.0)
        assert torch.equal(dx, (d @ w.double().t()).to(BF)) and torch.equal(dw, (x.double().t() @ d).to(BF))
        assert torch.equal(db.double(), d.sum(0)) and int(status) == b.DEV_NONFINITE


def test_bias_gradient_beyond_its_type():
    """Sums of finite dy that leave the range of dbias are written 0; the other columns keep theirs."""
    from paper_2506_15050_b200 import binding as b
    M, K, N = 70, 16, 24
    x, w = torch.ones((M, K), dtype=BF, device=DEV), torch.ones((K, N), dtype=BF, device=DEV)
    dy = torch.ones((M, N), dtype=BF, device=DEV)
    dy[:, 5] = 1e37                                         # 70 of them pass both types' largest value
    for dt in (BF, F32):
        db, status = torch.empty(N, dtype=dt, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        b.tppo_linear_bwd(dy, x, w, b.ACT_NONE, None, None, None, db, status, workspace(M, K, N))
        assert db.tolist() == [0.0 if n == 5 else 70.0 for n in range(N)] and int(status) == b.DEV_NONFINITE


def test_gradient_operand_that_is_not_finite():
    """A NaN of a bf16 dy that the products take as it is: what it enters is 0, the rest stays exact."""
    from paper_2506_15050_b200 import binding as b
    M, K, N, g = 40, 64, 64, gen(5)
    x, w, dy = whole(g, M, K), whole(g, K, N), whole(g, M, N)
    dy[3, 9] = float("nan")
    dx, dw, status = torch.empty_like(x), torch.empty_like(w), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_linear_bwd(dy, x, w, b.ACT_NONE, None, dx, dw, None, status, workspace(M, K, N))
    d = torch.nan_to_num(dy.double(), nan=0.0)
    rx, rw = d @ w.double().t(), x.double().t() @ d
    rx[3], rw[:, 9] = 0.0, 0.0
    assert torch.equal(dx.double(), rx.to(BF).double()) and torch.equal(dw.double(), rw.to(BF).double())
    assert int(status) == b.DEV_NONFINITE


@pytest.mark.parametrize("M,K,N,act", [(1001, 515, 777, 2), (300, 264, 520, 1), (2500, 1000, 2000, 0), (40, 24, 16, 4)])
def test_calls_one_behind_the_other(M, K, N, act):
    """Backward calls that share a workspace, each taking the dx of the one before as its dy: launches of a
    call that run side by side must neither overtake what they need nor leave anything behind them open."""
    from paper_2506_15050_b200 import binding as b
    g = gen(M + act)
    ws, wt = workspace(M, K, N), workspace(M, N, K)
    x, z = torch.randn((M, K), generator=g, device=DEV).to(BF), torch.randn((M, N), generator=g, device=DEV).to(BF)
    w = (torch.randn((K, N), generator=g, device=DEV) / math.sqrt(N)).to(BF)
    back = (torch.randn((N, K), generator=g, device=DEV) / math.sqrt(K)).to(BF)
    dy0 = torch.randn((M, N), generator=g, device=DEV).to(BF)

    def chain(wait):
        dy, out = dy0, []
        for k in range(6):
            dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV)
            b.tppo_linear_bwd(dy, x, w, act, z, dx, dw, db, None, ws)
            wait()
            dn, dv = torch.empty_like(dy), torch.empty_like(back)
            b.tppo_linear_bwd(dx, z, back, act, x, dn, dv, None, None, wt)
            wait()
            out += [dx, dw, db, dn, dv]
            dy = dn
        torch.cuda.synchronize()
        return out

    apart = chain(torch.cuda.synchronize)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(chain(lambda: None), apart))


@pytest.mark.parametrize("M,K,N", [(1001, 515, 777), (300, 264, 520), (2500, 1000, 2)])
def test_captured_calls_one_behind_the_other(M, K, N):
    from paper_2506_15050_b200 import binding as b
    g = gen(M)
    ws = workspace(M, K, N)
    x, z, dy = (torch.randn((M, c), generator=g, device=DEV).to(BF) for c in (K, N, N))
    w = (torch.randn((K, N), generator=g, device=DEV) / math.sqrt(N)).to(BF)
    outs = [[torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV), torch.empty((M, N), dtype=BF, device=DEV)] for _ in range(4)]

    def chain():
        for dx, dw, db, y in outs:                           # each forward call reads the gradients just written
            b.tppo_linear_bwd(dy, x, w, b.ACT_GELU, z, dx, dw, db, None, ws)
            b.tppo_linear_fwd(dx, dw, db, b.ACT_NONE, None, y, None, None, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        chain()
        side.synchronize()
        want = [t.clone() for t in outs[0]]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            chain()
        for o in outs:
            for t in o:
                t.fill_(7.0)
        for _ in range(3):
            graph.replay()
        side.synchronize()
    assert all(torch.equal(t, v) for o in outs for t, v in zip(o, want))
    del graph


@pytest.mark.parametrize("left,right", [(0, 0), (8, 8), (3, 2)])
@pytest.mark.parametrize("M,K,N", [(9000, 5120, 1), (3001, 2056, 2), (2500, 4100, 3), (70, 2050, 5), (1300, 520, 8), (1, 7000, 4),
                                   (5000, 3, 6), (200_000, 40, 1)])
def test_gradients_of_few_columns(M, K, N, left, right):
    from paper_2506_15050_b200 import binding as b
    g = gen(M + K + N)
    x, w, dy, z = whole(g, M, K, top=2), whole(g, K, N), whole(g, M, N, top=2), whole(g, M, N)
    dz = dy.double() * (z.double() > 0)
    rx, rw, rb = (dz @ w.double().t()).to(BF), (x.double().t() @ dz).to(BF), dz.sum(0)
    x, w, dy, z = (strided(t, left, right) for t in (x, w, dy, z))
    ws, status = workspace(M, K, N, 1), torch.zeros(1, dtype=torch.int32, device=DEV)
    for f in (lambda t: t, lambda t: t.float()):                 # dy in either type
        dx, dw, db = Guarded(M, K, BF, left, right), Guarded(K, N, BF, right, left), torch.full((N,), float("nan"), device=DEV)
        b.tppo_linear_bwd(f(dy), x, w, b.ACT_RELU, z, dx.t, dw.t, db, status, ws)
        assert torch.equal(dx.t, rx) and torch.equal(dw.t, rw) and torch.equal(db.double(), rb)
        dx.check()
        dw.check()
    # any subset of the outputs
    dx, dw, db = (torch.empty(n, dtype=BF, device=DEV) for n in ((M, K), (K, N), N))
    b.tppo_linear_bwd(dy, x, w, b.ACT_RELU, z, dx, None, None, status, ws)
    b.tppo_linear_bwd(dy, x, w, b.ACT_RELU, z, None, dw, None, status, ws)
    b.tppo_linear_bwd(dy, x, w, b.ACT_RELU, z, None, None, db, status, ws)
    assert torch.equal(dx, rx) and torch.equal(dw, rw) and torch.equal(db, rb.to(BF))
    assert int(status) == 0


def test_no_rows():
    from paper_2506_15050_b200 import binding as b
    K, N = 24, 16
    w = torch.ones((K, N), dtype=BF, device=DEV)
    x, dy = torch.empty((0, K), dtype=BF, device=DEV), torch.empty((0, N), dtype=BF, device=DEV)
    dw, db = Guarded(K, N, BF, 3, 2, fill=7.0), torch.ones(N, device=DEV)
    b.tppo_linear_fwd(x, w, None, 0, None, torch.empty((0, N), dtype=BF, device=DEV), None, None, None)
    b.tppo_linear_bwd(dy, x, w, 0, None, None, dw.t, db, None, None)
    assert not dw.t.any() and not db.any()
    dw.check()


def test_outputs_beyond_32_bits():
    """More than 2^31 elements of y, dx and dz; whole numbers, the last rows compared."""
    from paper_2506_15050_b200 import binding as b
    M, K, N, g = 530_001, 64, 4096, gen(2)
    x, w = whole(g, M, K), whole(g, K, N)
    y, ws = torch.empty((M, N), dtype=BF, device=DEV), workspace(M, K, N)
    b.tppo_linear_fwd(x, w, None, b.ACT_RELU, None, y, None, None, ws)
    for s in (slice(0, 300), slice(524_200, 524_400), slice(M - 300, M)):
        assert torch.equal(y[s], torch.relu(x[s].double() @ w.double()).to(BF))
    # backward: the kept pre-activation may be any bf16 matrix with the same signs
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV)
    dy = torch.ones((1, N), dtype=BF, device=DEV).expand(M, N).contiguous()
    b.tppo_linear_bwd(dy, x, w, b.ACT_RELU, y, dx, dw, db, None, ws)
    for s in (slice(0, 300), slice(524_200, 524_400), slice(M - 300, M)):
        assert torch.equal(dx[s], ((y[s] > 0).double() @ w.double().t()).to(BF))
    assert torch.equal(db.double(), (y > 0).sum(0).double())


def test_refusals_on_the_device():
    from paper_2506_15050_b200 import binding as b
    x, w = torch.ones((4, 24), dtype=BF, device=DEV), torch.ones((24, 40), dtype=BF, device=DEV)
    y = torch.full((4, 40), 7.0, dtype=BF, device=DEV)
    with pytest.raises(b.TppoError) as e:                  # misaligned rows need the copies' workspace
        b.tppo_linear_fwd(strided(x, 1, 0), w, None, 0, None, y, None, None, None)
    assert e.value.status == 2
    with pytest.raises(b.TppoError) as e:                  # and so does dz
        b.tppo_linear_bwd(y, x, w, b.ACT_RELU, y, x.clone(), None, None, None, None)
    assert e.value.status == 2
    for bad in (lambda: b.tppo_linear_fwd(x, w, None, 9, None, y, None, None, None),):
        with pytest.raises(b.TppoError) as e:
            bad()
        assert e.value.status == 1
    for bad in (lambda: b.tppo_linear_fwd(x.float(), w, None, 0, None, y, None, None, None),
                lambda: b.tppo_linear_fwd(x, w.t(), None, 0, None, y, None, None, None),
                lambda: b.tppo_linear_fwd(x, w, None, 0, None, y[:3], None, None, None),
                lambda: b.tppo_linear_fwd(x.cpu(), w, None, 0, None, y, None, None, None)):
        with pytest.raises(AssertionError):
            bad()
    torch.cuda.synchronize()
    assert bool((y == 7).all())


@pytest.mark.parametrize("M,K,N,act", [(1001, 515, 777, 2), (300, 264, 520, 1), (4100, 520, 2050, 4), (65, 72, 1000, 0)])
def test_buffers_refilled_before_each_call(M, K, N, act):
    """Every operand is written anew, in place, right before each call, which then rewrites its workspace: what
    runs side by side in a call may not see the values that the call before left in these places."""
    from paper_2506_15050_b200 import binding as b
    g = gen(M + K)
    r = lambda *s: [torch.randn(s, generator=g, device=DEV).to(BF) for _ in range(5)]
    sets = list(zip(r(M, N), r(M, K), r(K, N), r(M, N)))
    ws = workspace(M, K, N)
    call = lambda dy, x, w, z, o: b.tppo_linear_bwd(dy, x, w, act, z if act else None, *o, None, ws)
    empty = lambda: (torch.empty((M, K), dtype=BF, device=DEV), torch.empty((K, N), dtype=BF, device=DEV), torch.empty(N, device=DEV))
    want = []
    for s in sets:
        o = empty()
        call(*s, o)
        torch.cuda.synchronize()
        want.append(o)
    mine, got, out = [t.clone() for t in sets[0]], [], empty()
    for _ in range(4):
        for s, w in zip(sets, want):
            for a, t in zip(mine, s):
                a.copy_(t)
            call(*mine, out)
            got.append((tuple(t.clone() for t in out), w))
    torch.cuda.synchronize()
    for o, w in got:
        assert all(torch.equal(a, t) for a, t in zip(o, w))


def test_gradients_without_one_of_the_operands():
    from paper_2506_15050_b200 import binding as b
    for M, K, N in ((40, 64, 72), (33, 130, 2)):
        g = gen(M)
        x, w, dy = whole(g, M, K), whole(g, K, N), whole(g, M, N)
        dx, dw, db, ws = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV), workspace(M, K, N)
        b.tppo_linear_bwd(dy, None, w, b.ACT_NONE, None, dx, None, None, None, ws)
        b.tppo_linear_bwd(dy, x, None, b.ACT_NONE, None, None, dw, db, None, ws)
        assert torch.equal(dx, (dy.double() @ w.double().t()).to(BF)) and torch.equal(dw, (x.double().t() @ dy.double()).to(BF))
        assert torch.equal(db.double(), dy.double().sum(0))
    b.tppo_linear_bwd(dy, None, None, b.ACT_NONE, None, None, None, db.zero_(), None, ws)
    assert torch.equal(db.double(), dy.double().sum(0))


def test_gelu_tails():
    """gelu of -12 .. -1 and its slope, each relative to itself.  Phi(z) is a product of exp(-z^2/2), whose argument
    carries three roundings of a number that it multiplies by z^2 / 2 (1.5 z^2 u) and ex2 four, a polynomial
    in t whose terms add up to 1.8 times its value in magnitude, eight roundings each (15 u), its fit (1.5 u),
    t (4 u) and three more products: 1.5 z^2 + 28 roundings, 32 here."""
    from paper_2506_15050_b200 import binding as b
    z = -(1 + 11 * torch.arange(2001, device=DEV) / 2000).to(BF)
    N = z.numel()
    x, w = torch.ones((1, 1), dtype=BF, device=DEV), z[None, :].contiguous()
    y, ws = torch.empty((1, N), device=DEV), workspace(1, 1, N)
    b.tppo_linear_fwd(x, w, None, b.ACT_GELU, None, y, None, None, ws)
    ref = act64(z.double(), 2)
    rel = (1.5 * z.double() ** 2 + 32) * U32
    err = ((y[0].double() - ref) / ref).abs()
    assert bool((err <= rel).all()), (err / rel).max().item()
    db, dy = torch.empty(N, device=DEV), torch.ones((1, N), device=DEV)
    b.tppo_linear_bwd(dy, x, w, b.ACT_GELU, w, None, None, db, None, ws)
    terms = act64(z.double(), 2).abs() / z.double().abs() + z.double().abs() * torch.exp(-z.double() ** 2 / 2) / math.sqrt(2 * math.pi)
    err = (db.double() - slope64(z.double(), 2)).abs()
    assert bool((err <= rel * terms).all()), (err / (rel * terms)).max().item()


@pytest.mark.parametrize("act", [0, 4])
@pytest.mark.parametrize("M,K,N", [(9000, 5120, 1), (2500, 4100, 3), (1300, 520, 2), (70, 2051, 4), (1, 8, 1)])
def test_fp32_gradients_of_few_columns(M, K, N, act):
    """dz stays in fp32: one rounding of dx, and of dweight after sums of some hundred fp32 additions.  Rows that are
    not 16-byte aligned, from 2^23 elements of x on, take the tensor cores, as the header says: their dz is rounded
    to bf16 once, which adds half a step of it through both products."""
    from paper_2506_15050_b200 import binding as b
    g = gen(M + N)
    x, w = torch.randn((M, K), generator=g, device=DEV).to(BF), torch.randn((K, N), generator=g, device=DEV).to(BF)
    dy, z = torch.randn((M, N), generator=g, device=DEV), torch.randn((M, N), generator=g, device=DEV).to(BF)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(N, device=DEV)
    b.tppo_linear_bwd(dy, x, w, act, z if act else None, dx, dw, db, None, workspace(M, K, N))
    slope = slope64(z.double(), act) if act else torch.ones_like(dy).double()
    dz = dy.double() * slope
    e_dz = 24 * U32 * dy.double().abs() * (1 + z.double().abs()) if act else 0 * dz
    if K % 8 and M * K > 1 << 23:
        e_dz = e_dz + half_step(BF) * dz.abs()
    wd, xd = w.double(), x.double()
    for got, ref, mag, e in ((dx, dz @ wd.t(), dz.abs() @ wd.abs().t(), e_dz @ wd.abs().t()),
                             (dw, xd.t() @ dz, xd.abs().t() @ dz.abs(), xd.abs().t() @ e_dz)):
        tol = (half_step(BF) + U32) * ref.abs() + 320 * U32 * mag + 1.01 * e
        assert bool(((got.double() - ref).abs() <= tol).all()), ((got.double() - ref).abs() / tol).max().item()


@pytest.mark.parametrize("left,right", [(0, 0), (8, 8), (3, 2)])
@pytest.mark.parametrize("M,K,N", [(40, 64, 64), (70, 2050, 1), (300, 520, 3), (200, 130, 77), (4100, 4000, 2008)])
def test_one_rule_for_gradients_that_are_not_finite(M, K, N, left, right):
    """A NaN or an infinity in dy counts as 0 where dz is made (an activation, or fp32), and makes what it enters 0 where
    a bf16 dy is the operand itself -- whatever the sizes and alignments choose beneath."""
    from paper_2506_15050_b200 import binding as b
    g = gen(M + N)
    x, w, dy, z = whole(g, M, K), whole(g, K, N), whole(g, M, N), whole(g, M, N)
    rows, cols = torch.tensor([3, M - 1], device=DEV), torch.tensor([N // 2, N - 1], device=DEV)
    dy[rows[0], cols[0]], dy[rows[1], cols[1]] = float("nan"), -float("inf")
    d = torch.where(torch.isfinite(dy), dy, 0.0).double()
    x, w, dy, z = (strided(t, left, right) for t in (x, w, dy, z))
    ws = workspace(M, K, N, 1)
    for act, grad, through in ((b.ACT_NONE, dy, True), (b.ACT_NONE, dy.float(), False), (b.ACT_RELU, dy, False)):
        dx, dw, db = (torch.empty(s, dtype=BF, device=DEV) for s in ((M, K), (K, N), (N,)))
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        b.tppo_linear_bwd(grad, x, w, act, z if act else None, dx, dw, db, status, ws)
        dz = d * (z.double() > 0) if act else d
        rx, rw = dz @ w.double().t(), x.double().t() @ dz
        if through:
            rx[rows], rw[:, cols] = 0.0, 0.0
        assert torch.equal(dx, rx.to(BF)) and torch.equal(dw, rw.to(BF)) and torch.equal(db, dz.sum(0).to(BF))
        assert int(status) == b.DEV_NONFINITE


@pytest.mark.parametrize("left,right", [(0, 0), (8, 8), (3, 2)])
@pytest.mark.parametrize("M,K,N", [(2100, 5120, 1), (9000, 2048, 1), (1, 64, 1), (5000, 4104, 4), (700, 2056, 2), (20000, 512, 3)])
def test_value_head_in_its_own_workspace(M, K, N, left, right):
    """The bytes that the query asks for and no more, at any alignment; what lies behind them stays as it is."""
    from paper_2506_15050_b200 import binding as b
    g = gen(M + K + N)
    x, w, dy = whole(g, M, K, top=2), whole(g, K, N), whole(g, M, N, top=2)
    rx, rw, rb = (dy.double() @ w.double().t()).to(BF), (x.double().t() @ dy.double()).to(BF), dy.double().sum(0)
    y = x.double() @ w.double()
    x, w, dy = (strided(t, left, right) for t in (x, w, dy))
    n = b.tppo_workspace_bytes(b.OP_LINEAR, M, K, 0, N)
    room = torch.full((n + 1024,), 0xff, dtype=torch.uint8, device=DEV)
    out, dx, dw, db = torch.empty((M, N), device=DEV), Guarded(M, K, BF, left, right), Guarded(K, N, BF, right, left), torch.empty(N, device=DEV)
    b.tppo_linear_fwd(x, w, None, b.ACT_NONE, None, out, None, None, room[:n])
    b.tppo_linear_bwd(dy, x, w, b.ACT_NONE, None, dx.t, dw.t, db, None, room[:n])
    assert torch.equal(out.double(), y) and torch.equal(dx.t, rx) and torch.equal(dw.t, rw) and torch.equal(db.double(), rb)
    dx.check()
    dw.check()
    assert bool((room[n:] == 0xff).all())


def test_weight_gradient_over_rows_beyond_32_bits():
    """dweight contracts 530001 rows of a dz of more than 2^31 elements; sums of whole numbers below 2^24."""
    from paper_2506_15050_b200 import binding as b
    M, K, N, g = 530_001, 64, 4096, gen(12)
    x, w, z = whole(g, M, K), whole(g, K, N), torch.empty((M, N), dtype=BF, device=DEV)
    for m in range(0, M, 50_000):
        z[m:m + 50_000] = whole(g, min(50_000, M - m), N)
    dy = torch.ones((M, N), dtype=BF, device=DEV)
    dw, db = torch.empty_like(w), torch.empty(N, device=DEV)
    b.tppo_linear_bwd(dy, x, w, b.ACT_RELU, z, None, dw, db, None, workspace(M, K, N))
    ref, cols = torch.zeros((K, N), dtype=F64, device=DEV), torch.zeros(N, dtype=F64, device=DEV)
    for m in range(0, M, 50_000):
        on = (z[m:m + 50_000] > 0).double()
        ref += x[m:m + 50_000].double().t() @ on
        cols += on.sum(0)
    assert torch.equal(dw, ref.to(BF)) and torch.equal(db.double(), cols)


@pytest.mark.parametrize("M,K,N,act", [(4200, 1000, 2056, 2), (8200, 1030, 1030, 4)])
def test_long_streams_one_behind_the_other(M, K, N, act):
    """From 2^23 elements of dz on, what follows a stream starts at its end."""
    assert M * N > 1 << 23
    test_calls_one_behind_the_other(M, K, N, act)
