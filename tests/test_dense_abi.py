"""The dense operators' host side without a GPU: workspace sizes and refusals before any launch."""
import ctypes

import pytest

VP, I32, I64, F32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
INVALID, WORKSPACE, UNSUPPORTED = 1, 2, 3
LAYER_NORM, LINEAR, MUON = 5, 6, 7


@pytest.fixture(scope="module")
def lib():
    from paper_2506_15050_b200 import build
    b = ctypes.CDLL(build.build())
    b.tppo_workspace_bytes.restype = SZ
    b.tppo_workspace_bytes.argtypes = [ctypes.c_int, I64, I32, I64, I32]
    b.tppo_layer_norm_fwd.argtypes = [VP, I32, I64, I32, I64, VP, VP, I32, F32, VP, I64, VP, VP, VP, VP]
    b.tppo_layer_norm_bwd.argtypes = [VP, VP, I32, I64, I32, I64, I64, VP, I32, VP, VP, VP, I64, VP, VP, VP, VP, SZ, VP]
    b.tppo_linear_fwd.argtypes = [VP, I64, VP, I64, I64, I32, I32, VP, I32, I32, VP, I64, VP, I32, I64, VP, I64, VP, VP, SZ, VP]
    b.tppo_linear_bwd.argtypes = [VP, I32, I64, VP, I64, VP, I64, I64, I32, I32, I32, VP, I64, VP, I64, VP, I64, VP, I32, VP,
                                  VP, SZ, VP]
    b.tppo_muon_orthogonalize.argtypes = [VP, I32, I64, VP, I64, I64, I32, F32, I32, F32, I32, F32, VP, I64, VP, VP, SZ, VP]
    return b


@pytest.fixture(scope="module")
def p():
    buf = (ctypes.c_char * 8192)()
    at = (ctypes.addressof(buf) + 255) // 256 * 256
    return buf, at


def refused(call, args, good, bad):
    """Each change of `good` alone gives its status."""
    for change, status in bad:
        a = dict(good)
        a.update(change)
        assert call(*[a[k] for k in args]) == status, change


def test_workspace_sizes(lib):
    w = lib.tppo_workspace_bytes
    for op in (LAYER_NORM, LINEAR, MUON):
        small, big = w(op, 100, 64, 0, 64), w(op, 16384, 5120, 0, 5120)
        assert 0 < small <= big and small % 256 == 0 and big % 256 == 0
        assert w(op, -1, 64, 0, 64) == 0 and w(op, 100, 64, 0, 0) == 0
    # operand copies are counted where rows do not make whole lines, or on request
    assert w(LINEAR, 100, 72, 0, 64) > w(LINEAR, 100, 64, 0, 64) + 100 * 72 * 2
    assert w(LINEAR, 100, 64, 1, 64) >= w(LINEAR, 100, 64, 0, 64) + 2 * (100 * 64 + 64 * 64)
    # offsets beyond 32 bits
    assert w(MUON, 100000, 0, 0, 50000) > 8 * 100000 * 50000
    assert w(LINEAR, 1 << 20, 8192, 1, 8192) > 4 * (1 << 20) * 8192


def test_layer_norm_refusals(lib, p):
    a = p[1]
    args = "x dtype M N ldx gamma beta pdtype eps y ldy mean rstd status stream".split()
    good = dict(x=a, dtype=0, M=4, N=16, ldx=16, gamma=a, beta=a, pdtype=1, eps=1e-5, y=a, ldy=16, mean=a, rstd=a, status=a, stream=None)
    refused(lib.tppo_layer_norm_fwd, args, good, [
        (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(ldx=15), INVALID),
        (dict(ldy=15), INVALID), (dict(dtype=2), INVALID), (dict(pdtype=2), INVALID), (dict(eps=-1e-5), INVALID),
        (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(x=a + 1), INVALID), (dict(gamma=a + 2), INVALID),
        (dict(mean=a + 2), INVALID), (dict(status=a + 1), INVALID), (dict(M=(1 << 30) + 1), UNSUPPORTED),
        (dict(N=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31), UNSUPPORTED)])
    assert lib.tppo_layer_norm_fwd(*[dict(good, M=0, x=None, y=None)[k] for k in args]) == 0
    args = "dy x dtype M N lddy ldx gamma pdtype mean rstd dx lddx dgamma dbeta status ws bytes stream".split()
    good = dict(dy=a, x=a, dtype=1, M=4, N=16, lddy=16, ldx=16, gamma=a, pdtype=1, mean=a, rstd=a, dx=a, lddx=16, dgamma=a, dbeta=a,
                status=a, ws=a, bytes=1 << 30, stream=None)
    refused(lib.tppo_layer_norm_bwd, args, good, [
        (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(mean=None), INVALID), (dict(rstd=None), INVALID), (dict(N=0), INVALID),
        (dict(lddx=15), INVALID), (dict(lddy=3), INVALID), (dict(dtype=5), INVALID), (dict(pdtype=-1), INVALID), (dict(M=-2), INVALID),
        (dict(dx=a + 2), INVALID), (dict(dgamma=a + 1), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=a + 16), WORKSPACE),
        (dict(bytes=100), WORKSPACE), (dict(bytes=lib.tppo_workspace_bytes(LAYER_NORM, 4, 0, 0, 16) - 1), WORKSPACE)])
    nothing = dict(good, dx=None, dgamma=None, dbeta=None, ws=None, bytes=0)
    assert lib.tppo_layer_norm_bwd(*[nothing[k] for k in args]) == 0


def test_linear_refusals(lib, p):
    a = p[1]
    args = "x ldx w ldw M K N bias bdtype act residual ldr y ydtype ldy pre ldp status ws bytes stream".split()
    good = dict(x=a, ldx=16, w=a, ldw=24, M=4, K=16, N=24, bias=a, bdtype=0, act=2, residual=a, ldr=24, y=a, ydtype=0, ldy=24, pre=a, ldp=24,
                status=a, ws=None, bytes=0, stream=None)
    refused(lib.tppo_linear_fwd, args, good, [
        (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID), (dict(M=-1), INVALID), (dict(K=0), INVALID),
        (dict(N=0), INVALID), (dict(ldx=15), INVALID), (dict(ldw=23), INVALID), (dict(ldy=23), INVALID), (dict(ldr=23), INVALID),
        (dict(ldp=23), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID), (dict(ydtype=2), INVALID), (dict(bdtype=2), INVALID),
        (dict(x=a + 1), INVALID), (dict(y=a + 2, ydtype=1), INVALID), (dict(bias=a + 2, bdtype=1), INVALID), (dict(status=a + 2), INVALID),
        (dict(x=a + 2), WORKSPACE), (dict(ldw=25), WORKSPACE), (dict(ldw=25, ws=a, bytes=256), WORKSPACE),
        (dict(ldw=25, ws=a + 8, bytes=1 << 30), WORKSPACE), (dict(M=1 << 31), UNSUPPORTED), (dict(K=(1 << 30) + 8, ldx=1 << 31), UNSUPPORTED)])
    assert lib.tppo_linear_fwd(*[dict(good, M=0, x=None, w=None, y=None)[k] for k in args]) == 0
    args = "dy dtype lddy x ldx w ldw M K N act pre ldp dx lddx dw lddw db bdtype status ws bytes stream".split()
    good = dict(dy=a, dtype=0, lddy=24, x=a, ldx=16, w=a, ldw=24, M=4, K=16, N=24, act=2, pre=a, ldp=24, dx=a, lddx=16, dw=a, lddw=24, db=a,
                bdtype=1, status=a, ws=a, bytes=1 << 30, stream=None)
    refused(lib.tppo_linear_bwd, args, good, [
        (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(pre=None), INVALID), (dict(act=7), INVALID),
        (dict(lddy=20), INVALID), (dict(ldp=20), INVALID), (dict(lddx=15), INVALID), (dict(lddw=20), INVALID), (dict(K=0), INVALID),
        (dict(dtype=3), INVALID), (dict(bdtype=3), INVALID), (dict(dy=a + 2, dtype=1), INVALID), (dict(db=a + 2), INVALID),
        (dict(ws=None), WORKSPACE), (dict(bytes=64), WORKSPACE), (dict(ws=a + 1), WORKSPACE), (dict(ldx=17, bytes=0), WORKSPACE)])
    nothing = dict(good, dx=None, dw=None, db=None, ws=None, bytes=0)
    assert lib.tppo_linear_bwd(*[nothing[k] for k in args]) == 0


def test_muon_refusals(lib, p):
    a = p[1]
    args = "g dtype ldg m ldm R C mu nesterov eps steps scale u ldu status ws bytes stream".split()
    good = dict(g=a, dtype=0, ldg=24, m=a, ldm=24, R=4, C=24, mu=0.9, nesterov=1, eps=1e-7, steps=5, scale=1.0, u=a, ldu=24, status=a, ws=a,
                bytes=1 << 30, stream=None)
    refused(lib.tppo_muon_orthogonalize, args, good, [
        (dict(g=None), INVALID), (dict(u=None), INVALID), (dict(R=-1), INVALID), (dict(C=0), INVALID), (dict(ldg=23), INVALID),
        (dict(ldm=23), INVALID), (dict(ldu=23), INVALID), (dict(steps=0), INVALID), (dict(steps=17), INVALID), (dict(eps=-1.0), INVALID),
        (dict(eps=float("nan")), INVALID), (dict(mu=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(dtype=2), INVALID),
        (dict(g=a + 1), INVALID), (dict(m=a + 2), INVALID), (dict(u=a + 1), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=a + 64), WORKSPACE),
        (dict(bytes=4096), WORKSPACE), (dict(bytes=lib.tppo_workspace_bytes(MUON, 4, 0, 0, 24) - 1), WORKSPACE)])
    assert lib.tppo_muon_orthogonalize(*[dict(good, R=0, g=None, u=None)[k] for k in args]) == 0


def test_muon_scale_is_bounded(lib, p):
    a = p[1]
    for scale in (1.1e38, -3e38, float("inf")):               # times a singular value it could leave bf16
        assert lib.tppo_muon_orthogonalize(a, 0, 24, None, 0, 4, 24, 0.0, 0, 1e-7, 5, scale, a, 24, None, a, 1 << 30, None) == INVALID


def test_other_types_are_refused():
    import torch

    from paper_2506_15050_b200 import binding as b
    with pytest.raises(AssertionError, match="bfloat16 or torch.float32"):
        b._type_of(torch.ones(3, dtype=torch.float16))


def test_linear_backward_without_an_operand(lib, p):
    """x is not needed without dweight, weight not without dx: neither they nor their strides are looked at."""
    a = p[1]
    args = "dy dtype lddy x ldx w ldw M K N act pre ldp dx lddx dw lddw db bdtype status ws bytes stream".split()
    good = dict(dy=a, dtype=0, lddy=24, x=None, ldx=0, w=None, ldw=0, M=0, K=16, N=24, act=0, pre=None, ldp=0, dx=None, lddx=0, dw=None, lddw=0,
                db=None, bdtype=1, status=None, ws=None, bytes=0, stream=None)
    for change in (dict(), dict(x=a, ldx=16), dict(w=a, ldw=24), dict(M=4), dict(M=4, x=a, ldx=16)):
        assert lib.tppo_linear_bwd(*[dict(good, **change)[k] for k in args]) == 0
    refused(lib.tppo_linear_bwd, args, dict(good, M=4), [
        (dict(x=a, ldx=15), INVALID), (dict(w=a, ldw=23), INVALID), (dict(dx=a, lddx=16), INVALID), (dict(dw=a, lddw=24), INVALID)])


def test_workspaces_follow_the_path(lib):
    """Rows beyond the kernels that walk over them take 64 partial rows, no call more partial rows than rows, and a
    value head only its partial sums; a workspace of the largest sizes serves the smaller ones of the same kind."""
    w = lib.tppo_workspace_bytes
    assert w(LAYER_NORM, 16384, 0, 0, 70001) <= 3 * 148 * 2 * 4 * 16384 + 4 * 16384 + 512      # what 16384 columns take
    assert w(LAYER_NORM, 64, 0, 0, 70001) <= 64 * 2 * 4 * 70001 + 4 * 64 + 512
    assert w(LAYER_NORM, 1, 0, 0, 5120) <= 2 * 4 * 5120 + 512
    assert w(LAYER_NORM, 16384, 0, 0, 16384) >= 148 * 2 * 4 * 16384
    assert 4 << 20 <= w(LINEAR, 16384, 5120, 0, 1) <= 6 << 20
    assert w(LINEAR, 1, 5120, 0, 4) <= 1 << 18
    assert w(LINEAR, 16384, 5120, 1, 1) >= 2 * 16384 * 5120                # misaligned views on request: operand copies
    assert w(LINEAR, 16384, 5121, 0, 1) >= 2 * 16384 * 5121 and w(LINEAR, 16384, 5120, 0, 5) >= 2 * 16384 * 5120
    for N in (1, 2, 3, 4):
        sizes = [w(LINEAR, 16384, K, 0, N) for K in (8, 64, 2048, 2056, 5120, 8192)]
        assert sizes == sorted(sizes)
        sizes = [w(LINEAR, M, 2048, 0, N) for M in (1, 4, 100, 1000, 10000, 100000)]
        assert sizes == sorted(sizes)
    for M in (1, 100, 600, 16384):
        sizes = [w(LAYER_NORM, M, 0, 0, N) for N in (1, 511, 512, 513, 2048, 2049, 16384, 16385, 70001, 1 << 20)]
        assert sizes == sorted(sizes)
