"""Host side of the residual join, the 8-bit products and the gradient norm without a GPU: workspace sizes and refusals before any
launch."""
import ctypes

import pytest

from test_dense_abi import F32, I32, I64, INVALID, SZ, UNSUPPORTED, VP, WORKSPACE, p, refused  # noqa: F401

RESIDUAL_NORM, GRAD_NORM = 8, 9


class Tensor(ctypes.Structure):
    _fields_ = [("data", VP), ("n", I64), ("dtype", I32), ("reserved", I32)]


@pytest.fixture(scope="module")
def lib():
    from paper_2506_15050_b200 import build
    b = ctypes.CDLL(build.build())
    b.tppo_workspace_bytes.restype = SZ
    b.tppo_workspace_bytes.argtypes = [ctypes.c_int, I64, I32, I64, I32]
    b.tppo_residual_norm_fwd.argtypes = [VP, I64, VP, I64, VP, I64, I32, I64, I32, VP, VP, I32, F32, F32, I32, VP, I64, VP, I64, VP, VP, VP, VP]
    b.tppo_residual_norm_bwd.argtypes = [VP, I64, VP, I64, VP, I64, VP, I64, VP, I64, I32, I64, I32, VP, VP, I32, VP, VP, F32, I32, VP, I64, VP,
                                         I64, VP, I64, VP, VP, VP, VP, SZ, VP]
    b.tppo_fp8_quantize.argtypes = [VP, I32, I64, I64, I64, I32, VP, I64, VP, I64, VP, I64, VP, I64, VP, VP]
    b.tppo_fp8_matmul.argtypes = [VP, I64, VP, I64, VP, I64, VP, I64, I32, I64, I64, I64, VP, I32, I64, VP, VP]
    b.tppo_grad_norm.argtypes = [VP, I32, VP, VP, VP, VP, SZ, VP]
    b.tppo_grad_clip.argtypes = [VP, I32, VP, ctypes.c_double, VP, VP, VP, VP]
    return b


def test_workspace_sizes(lib):
    w = lib.tppo_workspace_bytes
    for m, n in ((0, 5), (1, 1), (100, 64), (16384, 5120)):
        assert w(RESIDUAL_NORM, m, 0, 0, n) % 256 == 0 and w(RESIDUAL_NORM, m, 0, 0, n) >= 16 * m + 8 * n
    assert w(RESIDUAL_NORM, -1, 0, 0, 64) == 0 and w(RESIDUAL_NORM, 4, 0, 0, 0) == 0
    assert w(RESIDUAL_NORM, 1 << 30, 0, 0, 1 << 30) > 2 * 256 * 4 << 30
    assert 0 < w(GRAD_NORM, 0, 0, 0, 0) <= w(GRAD_NORM, 1000, 0, 0, 0) < w(GRAD_NORM, 100000, 0, 0, 0)


def test_residual_norm_refusals(lib, p):  # noqa: F811
    a = p[1]
    args = "z ldz res ldr gate ldg dtype M N gp gn pdtype alpha eps norms h ldh n ldn r1 r2 status stream".split()
    good = dict(z=a, ldz=16, res=a, ldr=16, gate=a, ldg=16, dtype=0, M=4, N=16, gp=a, gn=a, pdtype=1, alpha=1.0, eps=1e-6, norms=3, h=a, ldh=16,
                n=a, ldn=16, r1=a, r2=a, status=a, stream=None)
    big = (1 << 30) + 1
    refused(lib.tppo_residual_norm_fwd, args, good, [
        (dict(z=None), INVALID), (dict(res=None), INVALID), (dict(h=None), INVALID), (dict(n=None), INVALID), (dict(M=-1), INVALID),
        (dict(N=0), INVALID), (dict(ldz=15), INVALID), (dict(ldr=15), INVALID), (dict(ldh=15), INVALID), (dict(ldn=15), INVALID),
        (dict(ldg=15), INVALID), (dict(dtype=2), INVALID), (dict(pdtype=2), INVALID), (dict(norms=4), INVALID), (dict(norms=-1), INVALID),
        (dict(alpha=float("nan")), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("inf")), INVALID), (dict(z=a + 1), INVALID),
        (dict(gp=a + 2), INVALID), (dict(r1=a + 2), INVALID), (dict(status=a + 1), INVALID),
        (dict(norms=1), INVALID), (dict(norms=2), INVALID), (dict(norms=1, n=None, gn=None), INVALID), (dict(norms=1, n=None, r2=None), INVALID),
        (dict(norms=2, gp=None), INVALID), (dict(M=big), UNSUPPORTED), (dict(N=big, ldz=big, ldr=big, ldh=big, ldn=big, ldg=big), UNSUPPORTED)])
    nothing = dict(good, M=0, z=None, res=None, h=None, n=None)
    assert lib.tppo_residual_norm_fwd(*[nothing[k] for k in args]) == 0
    args = ("dh lddh dn lddn z ldz h ldh gate ldg dtype M N gp gn pdtype r1 r2 alpha norms dz lddz dres lddr dg lddg dgp dgn status ws bytes "
            "stream").split()
    good = dict(dh=a, lddh=16, dn=a, lddn=16, z=a, ldz=16, h=a, ldh=16, gate=a, ldg=0, dtype=1, M=4, N=16, gp=a, gn=a, pdtype=1, r1=a, r2=a, alpha=1.0,
                norms=3, dz=a, lddz=16, dres=a, lddr=16, dg=a, lddg=0, dgp=a, dgn=a, status=a, ws=a, bytes=1 << 30, stream=None)
    need = lib.tppo_workspace_bytes(RESIDUAL_NORM, 4, 0, 0, 16)
    refused(lib.tppo_residual_norm_bwd, args, good, [
        (dict(z=None), INVALID), (dict(dn=None), INVALID), (dict(h=None), INVALID), (dict(r1=None), INVALID), (dict(r2=None), INVALID),
        (dict(lddh=15), INVALID), (dict(lddn=15), INVALID), (dict(ldz=15), INVALID), (dict(ldh=15), INVALID), (dict(lddz=15), INVALID),
        (dict(lddr=15), INVALID), (dict(ldg=17, lddg=15), INVALID), (dict(ldg=15, lddg=17), INVALID), (dict(gate=None), INVALID),
        (dict(norms=1), INVALID), (dict(norms=2), INVALID), (dict(norms=8), INVALID), (dict(dtype=3), INVALID), (dict(M=-1), INVALID),
        (dict(N=0), INVALID), (dict(alpha=float("inf")), INVALID), (dict(dz=a + 2), INVALID), (dict(dgp=a + 1), INVALID),
        (dict(ws=None), WORKSPACE), (dict(ws=a + 16), WORKSPACE), (dict(bytes=need - 1), WORKSPACE),
        (dict(M=(1 << 30) + 1), UNSUPPORTED)])


def test_fp8_refusals(lib, p):  # noqa: F811
    a = p[1]
    args = "x dtype ldx M K block q ldq s lds qt ldqt st ldst status stream".split()
    good = dict(x=a, dtype=0, ldx=40, M=20, K=40, block=1, q=a, ldq=48, s=a, lds=20, qt=a, ldqt=32, st=a, ldst=40, status=a, stream=None)
    refused(lib.tppo_fp8_quantize, args, good, [
        (dict(x=None), INVALID), (dict(x=a + 1), INVALID), (dict(ldx=39), INVALID), (dict(dtype=2), INVALID), (dict(block=0), INVALID),
        (dict(block=3), INVALID), (dict(M=-1), INVALID), (dict(K=-1), INVALID), (dict(q=a + 8), INVALID), (dict(ldq=40), INVALID),
        (dict(ldq=32), INVALID), (dict(s=None), INVALID), (dict(q=None), INVALID), (dict(qt=None), INVALID), (dict(st=None), INVALID),
        (dict(lds=19), INVALID), (dict(ldst=39), INVALID), (dict(ldqt=20), INVALID), (dict(qt=a + 4), INVALID), (dict(s=a + 2), INVALID),
        (dict(status=a + 2), INVALID), (dict(M=(1 << 30) + 1), UNSUPPORTED), (dict(K=(1 << 30) + 1), UNSUPPORTED)])
    for k in ("M", "K"):
        assert lib.tppo_fp8_quantize(*[dict(good, **{k: 0})[n] for n in args]) == 0
    nothing = dict(good, q=None, s=None, qt=None, st=None)
    assert lib.tppo_fp8_quantize(*[nothing[n] for n in args]) == 0
    args = "a lda sa ldas b ldb sb ldbs block M N K y ydtype ldy status stream".split()
    good = dict(a=a, lda=144, sa=a, ldas=20, b=a, ldb=144, sb=a, ldbs=30, block=1, M=20, N=30, K=140, y=a, ydtype=0, ldy=30, status=a, stream=None)
    refused(lib.tppo_fp8_matmul, args, good, [
        (dict(a=None), INVALID), (dict(sa=None), INVALID), (dict(b=None), INVALID), (dict(sb=None), INVALID), (dict(y=None), INVALID),
        (dict(lda=140), INVALID), (dict(ldb=128), INVALID), (dict(a=a + 8), INVALID), (dict(b=a + 1), INVALID), (dict(ldas=19), INVALID),
        (dict(ldbs=29), INVALID), (dict(block=2, ldbs=1), INVALID), (dict(block=4), INVALID), (dict(ydtype=2), INVALID), (dict(ldy=29), INVALID),
        (dict(y=a + 1), INVALID), (dict(M=-1), INVALID), (dict(N=-1), INVALID), (dict(K=-1), INVALID), (dict(status=a + 3), INVALID),
        (dict(sa=a + 2), INVALID), (dict(M=(1 << 30) + 1), UNSUPPORTED), (dict(N=(1 << 30) + 1), UNSUPPORTED), (dict(K=(1 << 30) + 1), UNSUPPORTED)])
    for k in ("M", "N"):
        assert lib.tppo_fp8_matmul(*[dict(good, **{k: 0})[n] for n in args]) == 0


def test_grad_norm_refusals(lib, p):  # noqa: F811
    a = p[1]
    def tensors(*t):
        return (Tensor * len(t))(*[Tensor(d, n, k, 0) for d, n, k in t])
    ok = tensors((a, 5, 0), (a, 7, 1), (None, 0, 1))
    need = lib.tppo_workspace_bytes(GRAD_NORM, 3, 0, 0, 0)
    norm = lambda t=ok, count=3, sq=a, norm=a, st=a, ws=a, size=1 << 20: lib.tppo_grad_norm(t, count, sq, norm, st, ws, size, None)
    clip = lambda t=ok, count=3, sq=a, m=1.0, out=None, coef=a, st=a: lib.tppo_grad_clip(t, count, sq, m, out, coef, st, None)
    for f in (norm, clip):
        assert f(t=None) == INVALID and f(count=-1) == INVALID and f(sq=None) == INVALID and f(sq=a + 4) == INVALID and f(st=a + 1) == INVALID
        for bad in ((None, 5, 0), (a, -1, 0), (a, 5, 2), (a + 1, 5, 0), (a + 2, 5, 1)):
            assert f(t=tensors((a, 5, 0), bad), count=2) == INVALID
        assert f(t=tensors((a, 1 << 43, 0)), count=1) == UNSUPPORTED
    assert norm(ws=None) == WORKSPACE and norm(ws=a + 8) == WORKSPACE and norm(size=need - 1) == WORKSPACE and norm(norm=a + 2) == INVALID
    for m in (-1.0, float("nan"), float("inf")):
        assert clip(m=m) == INVALID
    assert clip(coef=a + 1) == INVALID
    assert clip(out=tensors((a, 5, 1), (a, 6, 1), (None, 0, 0))) == INVALID        # lengths differ
    assert clip(out=tensors((a, 5, 1), (None, 7, 1), (None, 0, 0))) == INVALID


@pytest.mark.parametrize("more", [0, 100, 1200])
def test_clipping_refuses_outputs_at_the_place_of_another_tensor(lib, p, more):  # noqa: F811
    """An element has one writer and no other reader.  Refused before anything is launched, in lists of any length."""
    a, launched = p[1], 4                                  # TPPO_ERR_CUDA: past all checks, without a GPU
    rest = [(a + 65536 + 256 * i, 8, 1) for i in range(more)]
    def tensors(*t):
        t = [*t[:1], *rest, *t[1:]]
        return (Tensor * len(t))(*[Tensor(d, n, k, 0) for d, n, k in t])
    clip = lambda g, out: lib.tppo_grad_clip(g, len(g), a, 1.0, out, None, None, None)
    one, two, far = (a, 64, 1), (a + 256, 64, 1), (a + 4096, 64, 1)
    for bad in ((one, (a, 63, 1)), (one, (a, 128, 0)), (one, two, one, (a + 256, 1, 1))):
        assert clip(tensors(*bad), None) == INVALID and clip(tensors(*bad), tensors(*bad)) == INVALID
    assert clip(tensors(one, two), tensors(one, one)) == INVALID                   # an output that is another entry's gradient
    assert clip(tensors(one, one), tensors(one, far)) == INVALID
    assert clip(tensors(one, one), tensors(far, one)) == INVALID
    assert clip(tensors((a, 64, 1)), tensors((a, 64, 0))) == INVALID               # its own gradient in another type
    if not __import__("torch").cuda.is_available():
        for good in ((one, two), (two, one), (one, one), (one, two, one, two), (one, (None, 0, 0), (a, 0, 1), two)):
            assert clip(tensors(*good), None) == launched
        assert clip(tensors(one, one), tensors(two, far)) == launched and clip(tensors(two, one), tensors(two, far)) == launched


def test_sizes_of_the_product_tests_take_every_cut(lib):
    """The sizes that test_gpu_fp8.py multiplies, by how the library cuts them."""
    from fp8_shapes import LONG, RAGGED, TOKENS
    cut = lib.tppo_test_fp8_cut
    cut.argtypes = [I64, I64, I64, I32, I32]
    assert set(RAGGED) == {(0, 1)} | {(bn, s) for bn in (16, 32, 64, 128) for s in range(1, 9)}
    for dtype, e in ((0, 2), (1, 4)):
        for (bn, splits), (m, n, k) in RAGGED.items():
            assert n * e % 16 and cut(m, n, k, dtype, 0) == 16 * bn + splits, (m, n, k)
        tiles = {cut(m, n, k, dtype, 1) // 16 for m, n, k in TOKENS}
        assert {16, 64, 128} <= tiles
    long = [cut(m, n, k, 1, 1) // 16 for m, n, k in LONG]
    assert 0 in long and len(set(long)) >= 3
    assert cut(0, 1, 1, 0, 1) == -1 and cut(1, 1, (1 << 30) + 1, 0, 1) == -1
