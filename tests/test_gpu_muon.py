"""tppo_muon_orthogonalize against the float64 recursion.

Tolerances.  h = 2^-11 is half a step of fp16.  A rounded operand M is off by at most h |M|_F in the
Frobenius norm, and by h / sqrt(3) |M|_F with rounding errors spread evenly over a step.  With singular
values of X below 1.21 and, after the last step, above 0.68, one step passes on
  B's rounding:  |dB X| <= 1.21 * 2.81 sqrt(m) h'             -> 5.0 h' of |X|
  A's rounding:  |b + 2 c A| <= 4.78, |A| <= 1.45 sqrt(m)     -> 12.3 h'
  X's rounding:  through B X 5.0 h', through A = X X^T twice A's gain, 24.6 h'
in all 28.4 h' = 8.0e-3 with h' = h / sqrt(3); the steps before enter through a polynomial whose slope is
at most 0.72 in magnitude around 1, so all steps together stay below sqrt(1 / (1 - 0.72^2)) = 1.44 times
that: 1.16e-2 of the norm.  Matrices with orthogonal rows and one singular value s leave only errors of
s, which are followed step by step in `scalar_error`.  The bf16 output adds half a step, 2^-8."""
import math

import pytest
import torch

from dense_util import BF, DEV, F32, F64, Guarded, U32, gen, half_step, strided

pytestmark = pytest.mark.gpu
NS = (3.4445, -4.7750, 2.0315)
H16 = 2.0 ** -11


def reference(u, steps, eps):
    x = u.double()
    x = x / (x.norm() + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    for _ in range(steps):
        a = x @ x.t()
        x = NS[0] * x + (NS[1] * a + NS[2] * a @ a) @ x
    return x.t() if flip else x


def call(grad, momentum=None, mu=0.95, nesterov=True, eps=1e-7, steps=5, scale=1.0, update=None, status=None, want=0):
    from paper_2506_15050_b200 import binding as b
    R, C = grad.shape
    ws = b.workspace(b.OP_MUON, R, 0, 0, C, DEV)
    ws.fill_(0xff)
    update = torch.empty((R, C), dtype=BF, device=DEV) if update is None else update
    status = torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status
    b.tppo_muon_orthogonalize(grad, momentum, mu, nesterov, eps, steps, scale, update, status, ws)
    assert int(status) == want
    return update


def near(update, ref, steps=5):
    tol = 1.16e-2 * ref.norm() + half_step(BF) * ref.norm()
    return (update.double() - ref).norm() <= tol


SIZES = [(1, 1), (1, 50), (50, 1), (2, 3), (8, 8), (16, 64), (33, 20), (64, 64), (65, 64), (100, 700), (130, 129), (700, 100),
         (257, 300), (515, 515), (24, 5000), (5000, 24), (1030, 519), (640, 1500)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("R,C", SIZES)
def test_random_matrices(R, C, dtype):
    g = gen(R + 3 * C)
    grad = (1e-3 * torch.randn((R, C), generator=g, device=DEV)).to(dtype)
    u = Guarded(R, C, BF)
    call(grad, update=u.t)
    u.check()
    assert near(u.t, reference(grad, 5, 1e-7))
    # momentum, both forms
    for nesterov in (True, False):
        m0 = 1e-2 * torch.randn((R, C), generator=g, device=DEV)
        m = m0.clone()
        up = call(grad, m, 0.9, nesterov, scale=1.5)
        mu = float(torch.tensor(0.9, dtype=F32))
        mref = mu * m0.double() + grad.double()
        assert bool(((m.double() - mref).abs() <= 2 * U32 * (mref.abs() + grad.double().abs())).all())
        uref = grad.double() + mu * m.double() if nesterov else m.double()
        assert near(up, 1.5 * reference(uref, 5, 1e-7))


@pytest.mark.parametrize("R,C", [(2500, 2300), (2300, 5200), (5000, 2310)])
def test_many_tiles(R, C):
    """Sizes whose products take the persistent kernel and its mirrored tiles."""
    g = gen(R)
    grad = torch.randn((R, C), generator=g, device=DEV).to(BF)
    assert near(call(grad), reference(grad, 5, 1e-7))
    again = call(grad)
    assert torch.equal(again, call(grad))


def hadamard(n):
    h = torch.ones((1, 1), dtype=F64, device=DEV)
    while h.shape[0] < n:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h


def scalar_error(s, m, steps):
    """(result, bound of its relative error) for a matrix with m equal singular values s: per step A = s^2 and B
    carry h each while their diagonals are operands, the operand X carries h into B X and twice into A."""
    err = 0.0
    for k in range(steps):
        a = s * s
        b = NS[1] * a + NS[2] * a * a
        out = NS[0] * s + b * s
        apart = m <= 64 or k >= steps - 3
        da = 2 * err + (0 if apart else H16) + 2 * H16            # relative to a; X's rounding enters twice
        db = abs(NS[1] + 2 * NS[2] * a) * a * da + (0 if apart else H16 * abs(b))
        err = (abs(NS[0] + b) * s * err + db * s + (0 if apart else abs(b) * s * H16)) / abs(out) + 1e-6
        s = out
    return s, err


@pytest.mark.parametrize("R,C", [(16, 64), (64, 64), (128, 128), (128, 256), (256, 128), (512, 1024), (2048, 2048), (2048, 4096),
                                 (4096, 2048)])
@pytest.mark.parametrize("steps", [1, 2, 5])
def test_orthogonal_rows(R, C, steps):
    """Rows of a Hadamard matrix: dense products whose result is the same matrix, scaled."""
    m, n = min(R, C), max(R, C)
    h = hadamard(n)[torch.randperm(n, generator=gen(n), device=DEV)[:m]]
    x = h.t().contiguous() if R > C else h
    s0 = math.sqrt(n) / math.sqrt(m * n)                          # |row| / |matrix|
    s, err = scalar_error(s0, m, steps)
    up = call(x.to(BF), eps=0.0, steps=steps)
    ref = x * (s / math.sqrt(n))
    assert bool(((up.double() - ref).abs() <= (err + half_step(BF)) * ref.abs()).all()), \
        (((up.double() - ref) / ref).abs().max().item(), err)


@pytest.mark.parametrize("R,C", [(40, 40), (150, 333), (333, 150), (2400, 2600), (2600, 2400)])
def test_scaled_permutations(R, C):
    """One element per row and column: zeros stay exactly 0, each element follows the scalar recursion.
    Gains per step as at the top: 28.4 h of the largest possible value, here per element."""
    g = gen(R)
    m = min(R, C)
    rows, cols = torch.randperm(R, generator=g, device=DEV)[:m], torch.randperm(C, generator=g, device=DEV)[:m]
    x = torch.zeros((R, C), dtype=F64, device=DEV)
    x[rows, cols] = (1 + 3 * torch.rand(m, generator=g, device=DEV, dtype=F64)).to(BF).double()
    up = call(x.to(BF))
    ref = reference(x, 5, 1e-7)
    on = x != 0
    assert not up[~on].any()
    assert bool(((up.double() - ref)[on].abs() <= (28.4 * 1.44 * H16 + half_step(BF)) * 1.21).all())


def test_low_rank_plus_noise():
    """A spectrum over four orders of magnitude: the small directions do not drown in roundings."""
    g = gen(4)
    x = torch.randn((100, 8), generator=g, device=DEV) @ torch.randn((8, 700), generator=g, device=DEV)
    x += 0.01 * torch.randn((100, 700), generator=g, device=DEV)
    ref = reference(x, 5, 1e-7)
    assert near(call(x), ref) and near(call(x.t().contiguous()), ref.t())


@pytest.mark.parametrize("left,right", [(8, 8), (1, 0), (0, 3), (4, 4)])
@pytest.mark.parametrize("R,C", [(96, 160), (75, 33), (2400, 2408)])
def test_strided_rows_of_any_alignment(R, C, left, right):
    g = gen(left + C)
    grad, m = torch.randn((R, C), generator=g, device=DEV).to(BF), torch.randn((R, C), generator=g, device=DEV)
    mine, out = strided(m, right, left), Guarded(R, C, BF, left, right)
    plain_m = m.clone()
    plain = call(grad, plain_m, 0.9, True)
    call(strided(grad, left, right), mine, 0.9, True, update=out.t)
    out.check()
    assert torch.equal(mine, plain_m)
    # the norm may be summed in another order: one fp32 step of it moves roundings, no more
    assert (out.t.double() - plain.double()).norm() <= 2e-3 * plain.double().norm()
    over = grad.clone()                                     # the update over the gradient
    call(over, m.clone(), 0.9, True, update=over)
    assert torch.equal(over, plain)


def test_extreme_values():
    from paper_2506_15050_b200 import binding as b
    z = torch.zeros((40, 70), dtype=BF, device=DEV)
    for eps in (0.0, 1e-7):
        assert not call(z, eps=eps).any()
    g = gen(8)
    x = torch.randn((40, 70), generator=g, device=DEV)
    for f in (1e-34, 1e30):                                  # squares leave the range of fp32
        y = (x * f)
        assert near(call(y, eps=0.0), reference(y.double(), 5, 0.0))
    y = x.clone()
    y[3, 4], y[5, 6] = float("nan"), float("inf")
    m = torch.randn((40, 70), generator=g, device=DEV)
    m[7, 8] = float("nan")
    m0 = m.clone()
    up = call(y, m, 0.5, False, want=b.DEV_NONFINITE)
    ref = 0.5 * torch.nan_to_num(m0.double(), nan=0.0) + torch.where(torch.isfinite(y), y, 0.0).double()
    ref[7, 8] = 0.0
    assert bool(torch.isfinite(m).all()) and near(up, reference(ref, 5, 1e-7))
    call(x[:0], update=torch.empty((0, 70), dtype=BF, device=DEV))


@pytest.mark.parametrize("R,C", [(16, 24), (300, 120)])
@pytest.mark.parametrize("power", [-149, 120])
def test_norms_at_the_ends_of_the_range(R, C, power):
    """Whole numbers times a power of two that leaves them exact in fp32; the reciprocal of the norm is not
    representable there, the quotient is that of the whole numbers."""
    x = torch.randint(-120, 121, (R, C), generator=gen(R + power + 200), device=DEV).float()
    ref = reference(x, 5, 0.0)
    y = (x.double() * 2.0 ** power).float()
    assert torch.equal(y.double() * 2.0 ** -power, x.double())
    assert near(call(y, eps=0.0), ref)


@pytest.mark.parametrize("R,C", [(256, 1024), (1030, 519), (700, 100), (2500, 2300), (2300, 5200), (5000, 2310)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_documented_precision(R, C, dtype):
    """Five steps on random matrices: X within about 1e-3 of its norm (1.5e-3 here), then one rounding whose error is
    at most half a step, evenly spread: 2^-8 / sqrt(3) of the norm.  Together 2.71e-3."""
    grad = torch.randn((R, C), generator=gen(R * C), device=DEV).to(dtype)
    ref = reference(grad, 5, 1e-7)
    assert (call(grad).double() - ref).norm() <= math.hypot(1.5e-3, half_step(BF) / math.sqrt(3)) * ref.norm()


@pytest.mark.parametrize("tall", [True, False])
def test_more_than_2_to_31_elements(tall):
    """A long side of 2^22 and a bit.  X after each step is U times a polynomial of U^T U, so the reference needs
    the small side's products only; some columns (rows) of it are compared, at the bound of `near` each."""
    n, m, g = (1 << 22) + 77, 520, gen(31)
    assert n * m > 1 << 31
    u = torch.empty((n, m) if tall else (m, n), dtype=BF, device=DEV)
    gram, step = torch.zeros((m, m), dtype=F64, device=DEV), 1 << 18
    mix = torch.randn((m, m), generator=g, device=DEV) * m ** -0.5 + torch.eye(m, device=DEV)
    part = lambda k: u[k:k + step] if tall else u[:, k:k + step].t()
    for k in range(0, n, step):
        part(k).copy_(torch.randn((min(step, n - k), m), generator=g, device=DEV) @ mix)
        gram += part(k).double().t() @ part(k).double()
    norm = gram.trace().sqrt()
    p = torch.eye(m, dtype=F64, device=DEV) / norm          # X = U p, A = p^T gram p
    for _ in range(5):
        a = p.t() @ gram @ p
        p = p @ (NS[0] * torch.eye(m, dtype=F64, device=DEV) + NS[1] * a + NS[2] * a @ a)
    up = torch.empty_like(u)
    call(u, eps=0.0, update=up)
    edge = (1 << 31) // m if tall else 0
    for k in (0, edge, n - 500):
        got = up[k:k + 500] if tall else up[:, k:k + 500].t()
        ref = (u[k:k + 500] if tall else u[:, k:k + 500].t()).double() @ p
        assert near(got, ref), float((got.double() - ref).norm() / ref.norm())
