"""tppo_layer_norm_fwd / _bwd against the float64 formulas.

Tolerances.  u = 2^-24.  A sum over a row runs over at most 16 elements in a thread (N / 1024 of them
in the kernel for long rows), five shuffle levels, at most 32 warps in five more: fewer than D(N) =
32 + N / 1024 roundings lie between an element and the sum, so its error is at most D u times the
sum of magnitudes.  With d = x - mean:
  mean: D u mean|x|, the division's u |mean| included in D;
  d:    the mean's error and u |d|;
  var:  relative (D + 3) u from the sum and the squares, and twice the relative error of d, which is at
        most (mean's error) / sqrt(var) in the rms sense; rstd half of that, plus 2 u of rsqrtf;
  y:    |gamma| (|h| times rstd's relative error + rstd times d's error + 3 u |h|) + u |y| + half a step
        of the output type."""
import pytest
import torch

from dense_util import BF, DEV, F32, Guarded, U32, gen, half_step, norm64, norm64_bwd, strided

pytestmark = pytest.mark.gpu


def depth(N):
    return 32 + N / 1024


def make(M, N, dtype, seed, offset=0.5):
    g = gen(seed)
    x = (torch.randn((M, N), generator=g, device=DEV) * torch.exp(torch.randn(N, generator=g, device=DEV)) + offset).to(dtype)
    dy = torch.randn((M, N), generator=g, device=DEV).to(dtype)
    gamma = 1 + 0.3 * torch.randn(N, generator=g, device=DEV)
    beta = 0.2 * torch.randn(N, generator=g, device=DEV)
    return x, dy, gamma, beta


def stat_errors(x, h, mean, rstd, N):
    """Bounds of the errors of mean, d = x - mean, and (relative) rstd, per row."""
    D = depth(N)
    e_mean = D * U32 * x.double().abs().mean(1)
    e_rstd = 0.5 * ((D + 3) * U32 + 2 * e_mean * rstd) + 3 * U32
    return e_mean, e_rstd


def check_fwd(x, gamma, beta, eps, y, mean, rstd):
    N = x.shape[1]
    ry, rm, rr, h = norm64(x, gamma, beta, eps)
    e_mean, e_rstd = stat_errors(x, h, rm, rr, N)
    assert bool(((mean.double() - rm).abs() <= e_mean + 1e-30).all())
    assert bool(((rstd.double() - rr).abs() <= e_rstd * rr).all())
    g = 1.0 if gamma is None else gamma.double().abs()
    tol = g * (h.abs() * (e_rstd + 4 * U32)[:, None] + (rr * e_mean)[:, None]) + ry.abs() * (U32 + half_step(y.dtype)) + 1e-30
    assert bool(((y.double() - ry).abs() <= tol).all()), ((y.double() - ry).abs() / tol).max().item()


SIZES = [(1, 1), (1, 8), (3, 7), (5, 33), (64, 64), (33, 100), (257, 256), (7, 1000), (9, 1024), (130, 1283), (4, 4096),
         (3, 5120), (2, 8200), (3, 8191), (2, 16384), (2, 16385), (2, 33000), (1, 70001)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N", SIZES)
def test_forward(M, N, dtype):
    from paper_2506_15050_b200 import binding as b
    x, _, gamma, beta = make(M, N, dtype, 1 + N)
    for params, (gm, bt) in enumerate(((gamma.to(dtype), beta.to(dtype)), (gamma, beta), (gamma.to(BF), None), (None, None))):
        y = Guarded(M, N, dtype)
        mean, rstd = torch.full((M,), float("nan"), device=DEV), torch.full((M,), float("nan"), device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        b.tppo_layer_norm_fwd(x, gm, bt, 1e-5, y.t, mean, rstd, status)
        check_fwd(x, gm, bt, 1e-5, y.t, mean, rstd)
        y.check()
        assert int(status) == 0
    z = x.clone()
    b.tppo_layer_norm_fwd(z, None, None, 1e-5, z, None, None, None)          # in place, nothing else wanted
    assert torch.equal(z, y.t)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("left,right", [(0, 8), (8, 8), (1, 0), (0, 1), (3, 6)])
@pytest.mark.parametrize("N", [64, 200, 201, 2048])
def test_strided_rows_of_any_alignment(N, left, right, dtype):
    from paper_2506_15050_b200 import binding as b
    M = 37
    x, dy, gamma, beta = make(M, N, dtype, 7 * N + left)
    xs, ds = strided(x, left, right), strided(dy, right, left)
    y, dx = Guarded(M, N, dtype, left, right), Guarded(M, N, dtype, right, left)
    out = []
    for args in ((x, dy, torch.empty_like(x), torch.empty_like(x)), (xs, ds, y.t, dx.t)):
        mean, rstd = (torch.empty(M, device=DEV) for _ in range(2))
        dg, db = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
        b.tppo_layer_norm_fwd(args[0], gamma, beta, 1e-6, args[2], mean, rstd, None)
        b.tppo_layer_norm_bwd(args[1], args[0], gamma, mean, rstd, args[3], dg, db, None, b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV))
        check_fwd(args[0], gamma, beta, 1e-6, args[2], mean, rstd)
        check_bwd(args[1], args[0], gamma, mean, rstd, args[3], dg, db)
    y.check()
    dx.check()


def check_bwd(dy, x, gamma, mean, rstd, dx, dgamma, dbeta):
    """mean and rstd are inputs here, so h = (x - mean) rstd carries 2 u |h| + u rstd |x| (the rounding of
    the difference is relative to it; u |x| covers nothing being cancelled).  a = dy gamma: u |a|.
    c1, c2: (D + 4) u times the mean magnitudes.  dx: rstd times the terms' errors + 4 u of the terms +
    half a step.  Column sums: M terms in at most M + 40 additions, each u of the sum of magnitudes."""
    M, N = x.shape
    D = depth(N)
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    rx, rg, rb = norm64_bwd(dy, h, rstd.double(), gamma)
    a = dy.double() * (1.0 if gamma is None else gamma.double())
    r = rstd.double()[:, None]
    if dx is not None:
        m1, m2 = a.abs().mean(1, keepdim=True), (a * h).abs().mean(1, keepdim=True)
        terms = a.abs() + (D + 4) * m1 + h.abs() * (D + 8) * m2
        tol = r * terms * 5 * U32 + rx.abs() * half_step(dx.dtype) + 1e-30
        assert bool(((dx.double() - rx).abs() <= tol).all()), ((dx.double() - rx).abs() / tol).max().item()
    for got, ref, mag in ((dgamma, rg, (dy.double() * h).abs().sum(0)), (dbeta, rb, dy.double().abs().sum(0))):
        if got is not None:
            tol = (min(M, 200) + 44) * U32 * mag + ref.abs() * half_step(got.dtype) + 1e-30
            assert bool(((got.double() - ref).abs() <= tol).all()), ((got.double() - ref).abs() / tol).max().item()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N", SIZES + [(3000, 64), (5000, 33), (1500, 520)])
def test_backward(M, N, dtype):
    from paper_2506_15050_b200 import binding as b
    x, dy, gamma, _ = make(M, N, dtype, 3 + N, offset=0.0)
    ws = b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV)
    _, m, r, _ = norm64(x, None, None, 1e-5)
    mean, rstd = m.float(), r.float()
    for gm, pt in ((gamma.to(dtype), dtype), (gamma, F32), (gamma.to(BF), BF), (None, F32)):
        ws.fill_(0xff)                                      # NaN patterns: the call may read only what it wrote
        dx = Guarded(M, N, dtype)
        dg, db = torch.full((N,), float("nan"), dtype=pt, device=DEV), torch.full((N,), float("nan"), dtype=pt, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        b.tppo_layer_norm_bwd(dy, x, gm, mean, rstd, dx.t, dg, db, status, ws)
        check_bwd(dy, x, gm, mean, rstd, dx.t, dg, db)
        dx.check()
        assert int(status) == 0
    again = [torch.empty_like(t) for t in (dx.t, dg, db)]
    b.tppo_layer_norm_bwd(dy, x, gm, mean, rstd, again[0], again[1], None, None, ws)       # any subset of the outputs
    assert torch.equal(again[0], dx.t) and torch.equal(again[1], dg)
    b.tppo_layer_norm_bwd(dy, x, gm, mean, rstd, None, None, again[2], None, ws)
    assert torch.equal(again[2], db)
    b.tppo_layer_norm_bwd(dy, x, gm, mean, rstd, again[0].zero_(), None, None, None, None)
    assert torch.equal(again[0], dx.t)
    d = dy.clone()
    b.tppo_layer_norm_bwd(d, x, gm, mean, rstd, d, again[1], again[2], None, ws)           # dx over dy
    assert torch.equal(d, dx.t) and torch.equal(again[1], dg) and torch.equal(again[2], db)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N", [(1000, 1024), (601, 2056), (900, 5120), (700, 8192), (620, 10248), (611, 12288), (600, 16384), (597, 20480),
                                 (1000, 1023), (601, 2051), (900, 5121), (600, 10243), (595, 16383), (593, 20001), (3000, 515)])
@pytest.mark.parametrize("left,right", [(0, 0), (3, 2)])
def test_many_long_rows(M, N, left, right, dtype):
    """Rows brought in by bulk copies, several per block; NaN between strided rows that must not count."""
    from paper_2506_15050_b200 import binding as b
    x, dy, gamma, beta = make(M, N, dtype, N)
    x[M // 3, 5] = float("nan")
    if left + right:
        x, dy = strided(x, left, right), strided(dy, right, left)
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV)
    keep = torch.arange(M, device=DEV) != M // 3
    for gm, bt, pt in ((gamma, beta, F32), (gamma.to(BF), None, BF), (None, beta, F32)):
        b.tppo_layer_norm_fwd(x, gm, bt, 1e-5, y, mean, rstd, status)
        check_fwd(x[keep], gm, bt, 1e-5, y[keep], mean[keep], rstd[keep])
        assert not y[M // 3].any() and float(rstd[M // 3]) == 0
        ws.fill_(0xff)
        dx, dg, db = torch.empty_like(x), torch.empty(N, dtype=pt, device=DEV), torch.empty(N, dtype=pt, device=DEV)
        b.tppo_layer_norm_bwd(dy, x, gm, mean, rstd, dx, dg, db, status, ws)
        check_bwd(dy[keep], x[keep], gm, mean[keep], rstd[keep], dx[keep], dg, db)
        assert not dx[M // 3].any() and int(status) == b.DEV_NONFINITE
        d = dy.clone()
        b.tppo_layer_norm_bwd(d, x, gm, mean, rstd, d, None, None, None, None)
        assert torch.equal(d, dx)
    z = strided(x, left, right) if left + right else x.clone()      # in place, at the same alignment
    b.tppo_layer_norm_fwd(z, None, beta, 1e-5, z, None, None, None)
    assert torch.equal(z, y)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N", [(148, 512), (149, 640), (295, 1536), (593, 768), (1185, 520), (2369, 512), (5001, 2048), (150, 6144), (447, 7168),
                                 (297, 4608)])
def test_last_rows_of_a_walk(M, N, dtype):
    """Blocks whose last trip holds some of its rows only, aligned rows inside a wider matrix of NaN."""
    from paper_2506_15050_b200 import binding as b
    x, dy, gamma, _ = make(M, N, dtype, M + N, offset=0.0)
    _, m, r, _ = norm64(x, None, None, 1e-5)
    mean, rstd = m.float(), r.float()
    x, dy, dx = strided(x, 8, 16), strided(dy, 16, 8), Guarded(M, N, dtype, 8, 8)
    ws, status = b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws.fill_(0xff)
    dg, db = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    b.tppo_layer_norm_bwd(dy, x, gamma, mean, rstd, dx.t, dg, db, status, ws)
    check_bwd(dy, x, gamma, mean, rstd, dx.t, dg, db)
    dx.check()
    assert int(status) == 0
    one = [torch.empty_like(t) for t in (dg, db)]
    b.tppo_layer_norm_bwd(dy, x, gamma, mean, rstd, None, *one, status, ws)
    assert torch.equal(one[0], dg) and torch.equal(one[1], db)


def test_gradient_against_differences():
    """<gradient, direction> against the central difference of <dy, y> in float64: its step 1e-4 leaves an
    error of order 1e-8, the fp32 gradients one of N M u at most relative to the sum of magnitudes."""
    from paper_2506_15050_b200 import binding as b
    M, N, eps = 40, 96, 1e-5
    x, dy, gamma, beta = make(M, N, F32, 5)
    mean, rstd, y = torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.empty_like(x)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    b.tppo_layer_norm_fwd(x, gamma, beta, eps, y, mean, rstd, None)
    b.tppo_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dg, db, None, b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV))
    f = lambda x, g, b_: (dy.double() * norm64(x, g, b_, eps)[0]).sum()
    g = gen(6)
    for k, grad in enumerate((dx, dg, db)):
        args = [x.double(), gamma.double(), beta.double()]
        v = torch.randn(args[k].shape, generator=g, device=DEV, dtype=torch.float64)
        lo, hi = list(args), list(args)
        lo[k], hi[k] = args[k] - 1e-4 * v, args[k] + 1e-4 * v
        want, got = (f(*hi) - f(*lo)) / 2e-4, (grad.double() * v).sum()
        assert abs(want - got) <= 1e-5 * (grad.double() * v).abs().sum()


@pytest.mark.parametrize("dtype,N", [(BF, 64), (BF, 5120), (F32, 201), (BF, 33000)])
def test_rows_without_statistics(dtype, N):
    from paper_2506_15050_b200 import binding as b
    M = 12
    x, dy, gamma, beta = make(M, N, dtype, 9)
    x[1, N // 2], x[3, 0], x[4, N - 1] = float("nan"), float("inf"), -float("inf")
    x[6] = 2.5                                              # no variance: y = beta
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device=DEV), torch.empty(M, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_layer_norm_fwd(x, gamma, beta, 1e-5, y, mean, rstd, status)
    assert int(status) == b.DEV_NONFINITE
    bad = torch.tensor([1, 3, 4], device=DEV)
    good = torch.tensor([r for r in range(M) if r not in (1, 3, 4)], device=DEV)
    assert not y[bad].any() and not mean[bad].any() and not rstd[bad].any()
    check_fwd(x[good], gamma, beta, 1e-5, y[good], mean[good], rstd[good])
    status.zero_()
    dy[8, N // 3] = float("inf")
    dx, dg, db = torch.empty_like(x), torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    ws = b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV)
    b.tppo_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dg, db, status, ws)
    assert int(status) == b.DEV_NONFINITE
    keep = good[good != 8]
    assert not dx[bad].any() and not dx[8].any()
    check_bwd(dy[keep], x[keep], gamma, mean[keep], rstd[keep], dx[keep], dg, db)
    # with eps = 0 a row without variance has no statistics either
    status.zero_()
    b.tppo_layer_norm_fwd(x, gamma, beta, 0.0, y, mean, rstd, status)
    assert int(status) == b.DEV_NONFINITE and not y[6].any() and float(rstd[6]) == 0
    # no rows: empty sums
    b.tppo_layer_norm_bwd(dy[:0], x[:0], gamma, mean[:0], rstd[:0], dx[:0], dg, db, None, ws)
    assert not dg.any() and not db.any()
    b.tppo_layer_norm_fwd(x[:0], gamma, beta, 1e-5, y[:0], None, None, None)


def test_row_offsets_beyond_32_bits():
    """A row stride that puts the last rows past 2^31 elements."""
    from paper_2506_15050_b200 import binding as b
    M, N, ld = 3, 264, 1 << 30
    big = torch.empty(2 * ld + N, dtype=BF, device=DEV)
    x, _, gamma, beta = make(M, N, BF, 11)
    v = big.as_strided((M, N), (ld, 1))
    v.copy_(x)
    mean, rstd, y = torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.empty_like(x)
    b.tppo_layer_norm_fwd(v, gamma, beta, 1e-5, y, mean, rstd, None)
    check_fwd(x, gamma, beta, 1e-5, y, mean, rstd)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N", [(2100, 5120), (2500, 4096), (2049, 8192), (2100, 3001), (2048, 4100), (2600, 2571)])
@pytest.mark.parametrize("left,right", [(0, 0), (8, 8), (1, 2)])
def test_forward_of_many_rows(M, N, left, right, dtype):
    """Two to four blocks per SM, each with its own ring, and several rows per block; the first and the last
    row of a matrix at any alignment hold elements that no bulk copy brings, and their stages are used again."""
    from paper_2506_15050_b200 import binding as b
    x, _, gamma, beta = make(M, N, dtype, M + N)
    if left + right:
        x = strided(x, left, right)
    for gm, bt in ((gamma, beta), (gamma.to(BF), None)):
        y = Guarded(M, N, dtype, left, right)
        mean, rstd, status = torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        b.tppo_layer_norm_fwd(x, gm, bt, 1e-5, y.t, mean, rstd, status)
        check_fwd(x, gm, bt, 1e-5, y.t, mean, rstd)
        y.check()
        assert int(status) == 0


@pytest.mark.parametrize("dtype,M,N", [(BF, 2100, 5192), (BF, 2100, 2565), (F32, 2100, 9236), (F32, 2100, 4657), (BF, 620, 10384)])
def test_rows_of_one_value(dtype, M, N):
    """Eight bits times at most 2^14 columns: every partial sum is exact, so the mean is the value, y = beta, and with
    eps = 0 the row has no statistics."""
    from paper_2506_15050_b200 import binding as b
    c = (torch.arange(M, device=DEV) % 128 + 128).to(dtype) / 128
    x = c[:, None].expand(M, N).contiguous()
    beta = torch.randn(N, generator=gen(N), device=DEV)
    y, mean, rstd, status = torch.empty_like(x), torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_layer_norm_fwd(x, None, beta, 1e-5, y, mean, rstd, status)
    assert torch.equal(mean, c.float()) and torch.equal(y, beta.to(dtype).expand(M, N)) and int(status) == 0
    b.tppo_layer_norm_fwd(x, None, beta, 0.0, y, mean, rstd, status)
    assert not y.any() and not mean.any() and not rstd.any() and int(status) == b.DEV_NONFINITE


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("M,N", [(1, 64), (3, 520), (147, 5120), (150, 640), (600, 16384), (10, 16385), (200, 20001)])
def test_gradients_in_a_workspace_of_the_size_asked_for(M, N, dtype):
    from paper_2506_15050_b200 import binding as b
    x, dy, gamma, _ = make(M, N, dtype, M + N, offset=0.0)
    _, m, r, _ = norm64(x, None, None, 1e-5)
    n = b.tppo_workspace_bytes(b.OP_LAYER_NORM, M, 0, 0, N)
    room = torch.full((n + 4096,), 0xff, dtype=torch.uint8, device=DEV)
    dx, dg, db = torch.empty_like(x), torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    b.tppo_layer_norm_bwd(dy, x, gamma, m.float(), r.float(), dx, dg, db, None, room[:n])
    check_bwd(dy, x, gamma, m.float(), r.float(), dx, dg, db)
    assert bool((room[n:] == 0xff).all())


@pytest.mark.parametrize("M,N,ld,left", [(530_001, 4104, 4104, 0), (530_001, 4101, 4104, 3), (262_200, 8200, 8200, 0)])
def test_more_than_2_to_31_elements(M, N, ld, left):
    """Whole matrices past 32 bits through the kernels that walk over rows: the first rows, those around 2^31 elements
    and the last ones, and the gradients' sums over all rows (M / 148 additions in a block at most, then fp64)."""
    from paper_2506_15050_b200 import binding as b
    assert M * ld > 1 << 31
    g = gen(N)
    x, dy = (torch.empty((M, ld), dtype=BF, device=DEV)[:, left:left + N] for _ in range(2))
    for m in range(0, M, 60_000):
        for t in (x, dy):
            t[m:m + 60_000] = torch.randn((min(60_000, M - m), N), generator=g, device=DEV).to(BF)
    gamma = 1 + 0.3 * torch.randn(N, generator=g, device=DEV)
    mean, rstd, y, dx = torch.empty(M, device=DEV), torch.empty(M, device=DEV), torch.empty_like(x), torch.empty_like(x)
    dg, db, status = torch.empty(N, device=DEV), torch.empty(N, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_layer_norm_fwd(x, gamma, None, 1e-5, y, mean, rstd, status)
    b.tppo_layer_norm_bwd(dy, x, gamma, mean, rstd, dx, dg, db, status, b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV))
    edge = (1 << 31) // ld
    for s in (slice(0, 300), slice(edge - 150, edge + 150), slice(M - 300, M)):
        check_fwd(x[s], gamma, None, 1e-5, y[s], mean[s], rstd[s])
        check_bwd(dy[s], x[s], gamma, mean[s], rstd[s], dx[s], None, None)
    sums = [torch.zeros(N, dtype=torch.float64, device=DEV) for _ in range(4)]
    for m in range(0, M, 60_000):
        s = slice(m, m + 60_000)
        d, h = dy[s].double(), (x[s].double() - mean[s, None].double()) * rstd[s, None].double()
        for k, t in enumerate((d * h, d)):
            sums[k] += t.sum(0)
            sums[k + 2] += t.abs().sum(0)
    for got, ref, mag in zip((dg, db), sums[:2], sums[2:]):
        assert bool(((got.double() - ref).abs() <= (M / 148 + 44) * U32 * mag + ref.abs() * half_step(F32)).all())
    assert int(status) == 0
