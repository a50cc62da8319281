"""tppo_fp8_quantize bit by bit against its definition in float64, and tppo_fp8_matmul against float64 products of the values
that its operands stand for.  Products of two four-bit numbers are exact in fp32, so a sum of K of them is within 2 (K + 2)
roundings of 2^-24 of the sum of magnitudes; the output's rounding is half a step of its type."""
import pytest
import torch

from dense_util import BF, DEV, F32, F64, U32, Guarded, gen, half_step, strided
from fp8_shapes import LONG, RAGGED, TOKENS

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn
ROWS, SQUARE = 1, 2


def block_scales(x, rows, cols):
    """Exponents of the blocks' scales, from the definition."""
    M, K = x.shape
    mb, kb = -(-M // rows), -(-K // cols)
    p = torch.zeros((mb * rows, kb * cols), dtype=F64, device=DEV)
    p[:M, :K] = x.double().abs()
    top = p.view(mb, rows, kb, cols).amax((1, 3))
    e = torch.full_like(top, -126)
    for _ in range(260):                                   # the least e with top <= 448 * 2^e
        e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    return torch.where(top > 0, torch.exp2(e), 1.0)


def spread(s, rows, cols, M, K):
    return s.double().repeat_interleave(rows, 0)[:M].repeat_interleave(cols, 1)[:, :K]


def round_e4m3(v):
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step                    # half to even


def quantize(x, block, status=None, transposed=True, plain=True):
    from paper_2506_15050_b200 import binding as b
    M, K = x.shape
    whole = [torch.full((r + 2, -(-c // 16) * 16 + 16), 0x55, dtype=torch.uint8, device=DEV).view(F8) for r, c in ((M, K), (K, M))]
    q, qt = whole[0][1:M + 1, :K], whole[1][1:K + 1, :M]
    s, st = b.fp8_scales(M, K, block, DEV), b.fp8_scales(K, M, block, DEV)
    s.fill_(float("nan")), st.fill_(float("nan"))
    b.tppo_fp8_quantize(x, block, q if plain else None, s if plain else None, qt if transposed else None, st if transposed else None, status)
    for w, r, c in ((whole[0], M, K), (whole[1], K, M)):   # nothing around them is written
        u = w.view(torch.uint8).clone()
        u[1:r + 1, :c] = 0x55
        assert bool((u == 0x55).all())
    return q, s, qt, st


def expected(x, block):
    """(values, scales as stored) of x and of its transpose."""
    out = []
    for y in (x, x.t()):
        rows, cols = (1, 128) if block == ROWS else (128, 128)
        s = block_scales(y, rows, cols)
        out += [round_e4m3(y.double() / spread(s, rows, cols, *y.shape)), s.t() if block == ROWS else s]
    return out


def check_quantized(x, block):
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    got, want = quantize(x, block, st), expected(x, block)
    for g, w in zip(got, want):
        assert torch.equal(g.to(F64), w)
    assert int(st) == 0
    # each layout by itself
    assert torch.equal(quantize(x, block, transposed=False)[0].to(F64), want[0])
    assert torch.equal(quantize(x, block, plain=False)[2].to(F64), want[2])
    return got


def sample(M, K, dtype, seed=0, spread_by=2.0):
    g = gen(seed + 3 * M + K)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)
    return (r(M, K) * torch.exp(spread_by * r(M, K))).to(dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [ROWS, SQUARE])
@pytest.mark.parametrize("M,K", [(1, 1), (1, 128), (7, 5), (128, 128), (129, 127), (200, 300), (1, 5120), (513, 1), (640, 1283), (16, 4096)])
def test_quantizer_bit_by_bit(M, K, block, dtype):
    check_quantized(sample(M, K, dtype), block)


@pytest.mark.parametrize("left,right", [(1, 0), (3, 4), (8, 8)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_quantizer_strides(left, right, dtype):
    check_quantized(strided(sample(150, 333, dtype), left, right), ROWS)
    check_quantized(strided(sample(150, 256, dtype), left, right), SQUARE)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [ROWS, SQUARE])
def test_quantizer_at_the_ends_of_the_range(dtype, block):
    """Zeros, the largest and smallest numbers, maxima on and beside 448 * 2^e, ties of the rounding."""
    x = torch.zeros((260, 256), dtype=F32, device=DEV)
    x[1] = 3.3e38
    x[2] = 1e-38
    x[3] = 2.0 ** -133
    x[4, 5] = 2.0 ** -126 * 448
    x[5, 5], x[6, 5], x[7, 5] = 448.0, 449.0, 447.0
    x[8, :16] = torch.arange(16, device=DEV) + 0.5         # ties at a step of 1
    x[8, 100] = 256.0
    x[9, :64] = (torch.arange(64, device=DEV) + 0.5) * 2.0 ** -9
    x[9, 100] = 448.0
    x[10] = -1e30
    x[130:200] = torch.randn((70, 256), generator=gen(1), device=DEV) * 1e-3
    check_quantized(x.to(dtype), block)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [ROWS, SQUARE])
def test_what_is_not_finite_counts_as_zero(dtype, block):
    from paper_2506_15050_b200 import binding as b
    x = sample(140, 270, dtype)
    x[3, 7], x[100, 200], x[139, 269] = float("nan"), float("inf"), float("-inf")
    clean = torch.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    got, want = quantize(x, block, st), expected(clean, block)
    assert int(st) == b.DEV_NONFINITE
    for g, w in zip(got, want):
        assert torch.equal(g.to(F64), w)


def operand(M, K, block, seed=0, dtype=BF):
    from paper_2506_15050_b200 import binding as b
    x = sample(M, K, dtype, seed, 0.7)
    q, s = b.fp8_empty(M, K, DEV), b.fp8_scales(M, K, block, DEV)
    b.tppo_fp8_quantize(x, block, q, s, None, None, None)
    rows, cols = (1, 128) if block == ROWS else (128, 128)
    return q, s, q.to(F64) * spread(s.t() if block == ROWS else s, rows, cols, M, K)


def check_product(M, N, K, block, dtype, left=0, right=0, seed=0):
    from paper_2506_15050_b200 import binding as b
    a, sa, A = operand(M, K, ROWS, seed)
    w, sw, W = operand(N, K, block, seed + 1)
    y, st = Guarded(M, N, dtype, left, right), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_fp8_matmul(a, sa, w, sw, block, y.t, st)
    assert int(st) == 0
    ref, mag = A @ W.t(), A.abs() @ W.abs().t()
    d = (y.t.double() - ref).abs()
    tol = 2 * (K + 2) * U32 * mag + half_step(dtype) * ref.abs()
    assert bool((d <= tol).all()), (d / tol.clamp_min(1e-300)).max().item()
    y.check()
    return y.t


SHAPES = [(1, 1, 1), (1, 5120, 5120), (2, 3, 130), (16, 128, 128), (17, 300, 129), (33, 4000, 515), (64, 512, 4096), (65, 129, 640), (128, 128, 1),
          (130, 777, 1283), (300, 2000, 260), (1001, 777, 515), (1025, 1000, 777), (2048, 2048, 128), (2049, 2047, 1153), (5000, 257, 2048),
          (3000, 2500, 520)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [ROWS, SQUARE])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_products(M, N, K, block, dtype):
    check_product(M, N, K, block, dtype)


@pytest.mark.parametrize("dtype,left,right", [(BF, 1, 2), (BF, 8, 8), (F32, 1, 0), (F32, 4, 4), (BF, 0, 3)])
@pytest.mark.parametrize("M,N,K", [(40, 257, 300), (2100, 1999, 140)])
def test_strided_outputs(M, N, K, dtype, left, right):
    check_product(M, N, K, SQUARE, dtype, left, right)


@pytest.mark.parametrize("M,N", [(70, 90), (2200, 1900)])
def test_every_block_has_its_own_scales(M, N):
    """Scales far apart from row to row and block to block, of both operands: each product meets the right ones."""
    from paper_2506_15050_b200 import binding as b
    K, g = 128 * 9 + 40, gen(11)
    kb = 10
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    one = lambda r: torch.randint(1, 4, (r, K), generator=g, device=DEV).float().to(F8)
    pow2 = lambda *s: torch.exp2(torch.randint(-20, 21, s, generator=g, device=DEV).float())
    def put(q):
        p = b.fp8_empty(*q.shape, DEV)
        p.copy_(q)
        return p
    a, w = put(one(M)), put(one(N))
    sa, sw, sq = pow2(kb, M), pow2(kb, N), pow2(-(-N // 128), kb)
    A = a.to(F64) * spread(sa.t(), 1, 128, M, K)
    for s, block, W in ((sw, ROWS, w.to(F64) * spread(sw.t(), 1, 128, N, K)), (sq, SQUARE, w.to(F64) * spread(sq, 128, 128, N, K))):
        y = torch.empty((M, N), device=DEV)
        b.tppo_fp8_matmul(a, sa, w, s, block, y, st)
        ref = A @ W.t()                                    # all terms positive
        assert bool(((y.double() - ref).abs() <= 2 * (K + 2) * U32 * ref).all())
    assert int(st) == 0


@pytest.mark.parametrize("M,N,K", [(8, 200, 300), (1500, 1400, 300)])
def test_bad_scales_values_and_overflow(M, N, K):
    from paper_2506_15050_b200 import binding as b
    for dtype in (BF, F32):
        a, sa, A = operand(M, K, ROWS, 5)
        w, sw, W = operand(N, K, SQUARE, 6)
        y, st = torch.empty((M, N), dtype=dtype, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        call = lambda: b.tppo_fp8_matmul(a, sa, w, sw, SQUARE, y, st)
        call()
        good = y.clone()
        keep = sa.clone()
        for bad in (3.0, 0.0, -1.0, float("nan"), float("inf"), 2.0 ** -130):
            st.zero_()
            sa[1, 3] = bad
            call()
            assert int(st) == b.DEV_NONFINITE and not bool(y[3].any())
            assert torch.equal(y[:3], good[:3]) and torch.equal(y[4:], good[4:])
            sa.copy_(keep)
        a.view(torch.uint8)[5, 2] = 0x7f                   # e4m3's NaN
        st.zero_()
        call()
        assert int(st) == b.DEV_NONFINITE and not bool(y[5].any()) and torch.equal(y[6:], good[6:])
        a, sa, _ = operand(M, K, ROWS, 5)
        sa[:, 2] = 2.0 ** 120
        sw.fill_(2.0 ** 20)
        st.zero_()
        call()
        assert int(st) == b.DEV_NONFINITE and not bool(y[2].any())


def test_empty_products_and_repeatability():
    from paper_2506_15050_b200 import binding as b
    e = lambda r, c: b.fp8_empty(r, c, DEV)
    y, st = Guarded(5, 9, F32, 1, 1), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_fp8_matmul(e(5, 0), b.fp8_scales(5, 0, ROWS, DEV), e(9, 0), b.fp8_scales(9, 0, SQUARE, DEV), SQUARE, y.t, st)
    assert not bool(y.t.any())
    y.check()
    b.tppo_fp8_matmul(e(0, 130), b.fp8_scales(0, 130, ROWS, DEV), e(9, 130), b.fp8_scales(9, 130, SQUARE, DEV), SQUARE,
                      torch.empty((0, 9), device=DEV), st)
    x = torch.empty((0, 40), dtype=BF, device=DEV)
    b.tppo_fp8_quantize(x, ROWS, e(0, 40), b.fp8_scales(0, 40, ROWS, DEV), e(40, 0), b.fp8_scales(40, 0, ROWS, DEV), st)
    assert int(st) == 0
    for M, N, K in ((3, 1000, 2000), (2500, 2300, 900)):
        first = check_product(M, N, K, ROWS, F32).clone()
        for _ in range(3):
            assert torch.equal(check_product(M, N, K, ROWS, F32), first)


@pytest.mark.parametrize("M,K,N", [(300, 520, 390), (37, 1283, 250)])
def test_gradients_of_a_projection(M, K, N):
    """x W, dy W^T and x^T dy from one quantisation of each, against the gradients of the quantised product in float64."""
    from paper_2506_15050_b200 import binding as b
    x, w, dy = sample(M, K, BF, 1, 0.7), sample(K, N, F32, 2, 0.5), sample(M, N, BF, 3, 0.5)
    xq, xs, xt, xts = quantize(x, ROWS)
    wq, ws, wt, wts = quantize(w, SQUARE)
    dq, ds, dt, dts = quantize(dy, ROWS)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    y, dx, dw = (torch.empty(s, device=DEV) for s in ((M, N), (M, K), (K, N)))
    b.tppo_fp8_matmul(xq, xs, wt, wts, SQUARE, y, st)
    b.tppo_fp8_matmul(dq, ds, wq, ws, SQUARE, dx, st)
    b.tppo_fp8_matmul(xt, xts, dt, dts, ROWS, dw, st)
    X, W = xq.to(F64) * spread(xs.t(), 1, 128, M, K), wq.to(F64) * spread(ws, 128, 128, K, N)
    D, X2, D2 = dq.to(F64) * spread(ds.t(), 1, 128, M, N), xt.to(F64) * spread(xts.t(), 1, 128, K, M), dt.to(F64) * spread(dts.t(), 1, 128, N, M)
    for got, p, q in ((y, X, W), (dx, D, W.t()), (dw, X2, D2.t())):
        k = p.shape[1]
        assert bool(((got.double() - p @ q).abs() <= 2 * (k + 2) * U32 * (p.abs() @ q.abs())).all())
    # the quantised values are within half a step of what they stand for: 2^-4 of it, or of the smallest step of the block
    for t, v, s in ((x, X, spread(xs.t(), 1, 128, M, K)), (w, W, spread(ws, 128, 128, K, N))):
        assert bool(((t.double() - v).abs() <= 2.0 ** -4 * t.double().abs() + 2.0 ** -10 * s).all())
    assert int(st) == 0


def test_refusals_of_the_binding():
    from paper_2506_15050_b200 import binding as b
    a, s, _ = operand(20, 100, ROWS)
    w, sw, _ = operand(30, 100, SQUARE)
    y = torch.empty((20, 30), device=DEV)
    with pytest.raises(AssertionError):
        b.tppo_fp8_matmul(a, s, w, sw[:, :0], SQUARE, y, None)
    with pytest.raises(AssertionError):
        b.tppo_fp8_matmul(a, s, w, sw, SQUARE, y[:, :29], None)
    with pytest.raises(b.TppoError):
        b.tppo_fp8_matmul(a.contiguous(), s, w, sw, SQUARE, y, None)              # rows of 100 bytes
    with pytest.raises(AssertionError):
        b.tppo_fp8_matmul(a.view(torch.uint8), s, w, sw, SQUARE, y, None)
    with pytest.raises(b.TppoError):
        b.tppo_fp8_quantize(torch.zeros((4, 8), device=DEV), 3, None, None, None, None, None)


def test_more_than_two_to_the_31_elements():
    from paper_2506_15050_b200 import binding as b
    M, K, N = (1 << 21) + 77, 1040, 24
    x = torch.zeros((M, K), dtype=BF, device=DEV)
    x[-300:] = sample(300, K, BF, 4, 0.7)
    q, s = b.fp8_empty(M, K, DEV), b.fp8_scales(M, K, ROWS, DEV)
    qt, ts = b.fp8_empty(K, M, DEV), b.fp8_scales(K, M, ROWS, DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_fp8_quantize(x, ROWS, q, s, qt, ts, st)
    first = M // 128 * 128 - 128                            # whole blocks of rows from here on
    want = expected(x[first:], ROWS)
    assert torch.equal(q[first:].to(F64), want[0]) and torch.equal(s[:, first:].double(), want[1])
    assert torch.equal(qt[:, first:].to(F64), want[2]) and torch.equal(ts[first // 128:].double(), want[3])
    w, sw, W = operand(N, K, SQUARE, 6)
    y = torch.empty((M, N), device=DEV)
    b.tppo_fp8_matmul(q, s, w, sw, SQUARE, y, st)
    A = want[0] * spread(want[1].t(), 1, 128, M - first, K)
    assert bool(((y[first:].double() - A @ W.t()).abs() <= 2 * (K + 2) * U32 * (A.abs() @ W.abs().t())).all())
    assert not bool(y[:M - 300].any()) and int(st) == 0
    # contraction over the long side: what is not 0 begins 300 rows from its end, within 256 rows of `first`
    dw = torch.empty((K, K), device=DEV)
    b.tppo_fp8_matmul(qt, ts, qt, ts, ROWS, dw, st)
    T = want[2] * spread(want[3].t(), 1, 128, K, M - first)
    h0 = expected(x[first - 256:first], ROWS)
    H = h0[2] * spread(h0[3].t(), 1, 128, K, 256)
    ref, mag = T @ T.t() + H @ H.t(), T.abs() @ T.abs().t() + H.abs() @ H.abs().t()
    assert bool(((dw.double() - ref).abs() <= 2 * (600 + 2) * U32 * mag).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [ROWS, SQUARE])
@pytest.mark.parametrize("M,N,K", list(RAGGED.values()) + TOKENS)
def test_every_cut_of_the_product(M, N, K, block, dtype):
    check_product(M, N, K, block, dtype)


@pytest.mark.parametrize("M,N,K", LONG)
def test_precision_of_long_contractions(M, N, K):
    """fp32 outputs, by norms.  The tensor cores round (or cut) once per step of 32 elements, 32 times in each of S = K / 1024
    segments, whose sums are added up in registers.  An error of at most a step of 2^-23 of the running sum is 2^-23 / sqrt(3) of it
    (cut) or half of that (rounded); running sums of n parts have half of the variance of n whole ones on average.  So the result
    is within 2^-23 sqrt(32 / 2 / 3 + S / 2 / 12) of its norm: 2.9e-7 at 16384, where sums left in the tensor cores have 1.2e-6."""
    from paper_2506_15050_b200 import binding as b
    g, ops = gen(K), []
    for rows in (M, N):
        x = torch.randn((rows, K), generator=g, device=DEV)
        q, s = b.fp8_empty(rows, K, DEV), b.fp8_scales(rows, K, ROWS, DEV)
        b.tppo_fp8_quantize(x, ROWS, q, s, None, None, None)
        ops.append((q, s, q.to(F64) * spread(s.t(), 1, 128, rows, K)))
    (a, sa, A), (w, sw, W) = ops
    y, st = torch.empty((M, N), device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    b.tppo_fp8_matmul(a, sa, w, sw, ROWS, y, st)
    ref, S = A @ W.t(), -(-K // 1024)
    err = float((y.double() - ref).norm() / ref.norm())
    print(f"{M} x {N} x {K}: {err:.2e}")
    assert int(st) == 0 and err <= 2.0 ** -23 * (32 / 6 + S / 24) ** 0.5


@pytest.mark.parametrize("M,N", [(9, 200), (1500, 1400)])
@pytest.mark.parametrize("e", [-126, -100, -60, 60, 100, 126])
def test_scales_at_the_ends_of_their_range(M, N, e):
    """2^e in one operand, 2^-e in the other: small whole numbers, exact."""
    from paper_2506_15050_b200 import binding as b
    K, g = 300, gen(e + 200)
    a, w = b.fp8_empty(M, K, DEV), b.fp8_empty(N, K, DEV)
    for t in (a, w):
        t.copy_(torch.randint(-3, 4, t.shape, generator=g, device=DEV).float().to(F8))
    sa, sw, st = b.fp8_scales(M, K, ROWS, DEV), b.fp8_scales(N, K, SQUARE, DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    sa.fill_(2.0 ** e), sw.fill_(2.0 ** -e)
    y = torch.empty((M, N), device=DEV)
    b.tppo_fp8_matmul(a, sa, w, sw, SQUARE, y, st)
    assert int(st) == 0 and torch.equal(y.double(), a.to(F64) @ w.to(F64).t())
