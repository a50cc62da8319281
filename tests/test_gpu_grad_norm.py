"""tppo_grad_norm / tppo_grad_clip against float64 sums.

Tolerances: a sum of squares adds 32 of them in fp32 (eight in a chain of fused multiply-adds, four chains joined: ten
roundings of positive terms, 10 U with U = 2^-24) and the rest in 64 bits, so the norm is within 5 U of itself before its rounding
to fp32; a coefficient within 6 U; a clipped element within 2 U more and half a step of its type."""
import math

import pytest
import torch

from dense_util import BF, DEV, F32, U32, gen, half_step

pytestmark = pytest.mark.gpu
U = U32


def tensors(sizes, types, seed=0, pad=0, scale=1.0):
    """Tensors inside buffers whose other elements are guarded; `pad` elements in front of each."""
    g = gen(seed)
    whole = [torch.full((n + pad + 3,), float("nan"), dtype=t, device=DEV) for n, t in zip(sizes, types)]
    out = [w[pad:pad + n] for w, n in zip(whole, sizes)]
    for t in out:
        t.copy_(scale * torch.randn(t.shape, generator=g, device=DEV))
    return whole, out


def guard(whole, views):
    for w, v in zip(whole, views):
        a = v.storage_offset()
        assert bool(torch.isnan(w[:a]).all()) and bool(torch.isnan(w[a + v.numel():]).all()), "written outside"


def norm64(ts):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in ts))


def call(ts, max_norm, out=None):
    from paper_2506_15050_b200 import binding as b
    grads = b.tensor_list(ts)
    outs = None if out is None else b.tensor_list(out)
    sq, norm = torch.full((1,), -1.0, dtype=torch.float64, device=DEV), torch.full((1,), -1.0, device=DEV)
    coef, st = torch.full((1,), -1.0, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = b.workspace(b.OP_GRAD_NORM, len(ts), 0, 0, 0, DEV)
    ws.fill_(0xff)
    b.tppo_grad_norm(grads, sq, norm, st, ws)
    b.tppo_grad_clip(grads, sq, max_norm, outs, coef, st)
    return float(sq), float(norm), float(coef), int(st)


def check(ts, max_norm, out=None):
    before = [t.clone() for t in ts]
    sq, norm, coef, st = call(ts, max_norm, out)
    ref = norm64(before)
    assert st == 0
    assert abs(sq - ref * ref) <= 11 * U * ref * ref and abs(norm - ref) <= 7 * U * ref
    c = min(1.0, max_norm / ref) if ref > 0 else 1.0
    assert abs(coef - c) <= 8 * U * c
    for o, g in zip(ts if out is None else out, before):
        r = g.double() * c
        tol = (10 * U + half_step(o.dtype)) * r.abs() + (0 if c == 1 and o.dtype == g.dtype else 2.0 ** -133)
        assert bool(((o.double() - r).abs() <= tol).all())
    return coef


SETS = {"one": [1], "few": [5, 0, 1, 17, 8192, 8191, 8193], "cluster": [3000] * 40, "edge": [8192 * 128, 1], "beyond": [8192 * 128, 8193, 3],
        "many": [i % 97 for i in range(1100)], "large": [3_000_001, 40_000_000, 7, 999_999]}


@pytest.mark.parametrize("pad", [0, 1, 5])
@pytest.mark.parametrize("kind", ["bf16", "f32", "mix"])
@pytest.mark.parametrize("name", SETS)
def test_sizes_types_and_alignment(name, kind, pad):
    sizes = SETS[name]
    types = [{"bf16": BF, "f32": F32}.get(kind, (BF, F32)[i % 2]) for i in range(len(sizes))]
    whole, ts = tensors(sizes, types, len(sizes), pad)
    ref = norm64(ts)
    # into other buffers, of the same type and of the other
    for flip in (False, True):
        to = [(F32 if t == BF else BF) if flip else t for t in types]
        ow, out = tensors(sizes, to, 1, pad)
        keep = [t.clone() for t in ts]
        check(ts, 0.3 * ref, out)
        guard(ow, out)
        assert all(torch.equal(a, b) for a, b in zip(keep, ts))
    # nothing to clip, then clipped, both in place
    keep = [t.clone() for t in ts]
    assert check(ts, 1.5 * ref) == 1.0
    assert all(torch.equal(a, b) for a, b in zip(keep, ts))
    check(ts, 0.3 * ref)
    guard(whole, ts)


def test_misaligned_pairs():
    """Gradient and output at different places of a 16-byte piece."""
    for a, o in ((0, 1), (1, 0), (2, 3), (4, 0), (0, 4)):
        for ta, to in ((BF, F32), (F32, BF), (BF, BF), (F32, F32)):
            sizes = [20000, 33, 9]
            _, ts = tensors(sizes, [ta] * 3, 3, a)
            ow, out = tensors(sizes, [to] * 3, 4, o)
            check(ts, 0.25 * norm64(ts), out)
            guard(ow, out)


@pytest.mark.parametrize("sizes", [[70000, 3], [8192 * 200, 5]])
@pytest.mark.parametrize("scale", [1e-30, 1e-38, 1e18, 1e30])
def test_range_of_fp32(scale, sizes):
    """Squares below and beyond fp32."""
    _, ts = tensors(sizes, [F32] * 2, 5, 0, scale)
    ref = norm64(ts)
    sq, norm, coef, st = call(ts, ref / 2, [torch.empty_like(t) for t in ts])
    assert st == 0 and abs(sq - ref * ref) <= 12 * U * ref * ref
    assert abs(norm - ref) <= 7 * U * ref + 2.0 ** -149 and abs(coef - 0.5) <= 4 * U
    # a few large ones among many small ones
    ts[0][:7] = 1e20
    ref = norm64(ts)
    assert abs(call(ts, 1.0, [torch.empty_like(t) for t in ts])[0] - ref * ref) <= 12 * U * ref * ref


def test_very_small_coefficients_keep_their_precision():
    ts = [torch.full((100,), 3e38, device=DEV), torch.full((50,), -1e37, device=DEV)]
    ref = norm64(ts)
    out = [torch.empty_like(t) for t in ts]
    sq, norm, coef, st = call(ts, 0.05, out)
    assert st == 0 and math.isinf(norm) and abs(sq - ref * ref) <= 11 * U * ref * ref
    for o, t in zip(out, ts):
        r = t.double() * (0.05 / ref)
        assert bool(((o.double() - r).abs() <= 11 * U * r.abs()).all())


def test_zero_norms_limits_and_empty_lists():
    from paper_2506_15050_b200 import binding as b
    ts = [torch.zeros(5000, device=DEV), torch.zeros(3, dtype=BF, device=DEV)]
    assert call(ts, 1.0) == (0.0, 0.0, 1.0, 0)
    assert call(ts, 0.0) == (0.0, 0.0, 1.0, 0)
    ts = [torch.randn(5000, device=DEV)]
    assert call(ts, 0.0)[2:] == (0.0, 0) and not bool(ts[0].any())
    assert call([], 1.0) == (0.0, 0.0, 1.0, 0)
    assert call([torch.empty(0, device=DEV)], 1.0) == (0.0, 0.0, 1.0, 0)
    # a tensor listed twice counts twice
    t = torch.ones(16, device=DEV)
    assert call([t, t], 100.0)[0] == 32.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("sizes", [[100], [8192 * 300, 11]])
def test_not_finite_leaves_a_step_without_effect(bad, sizes):
    from paper_2506_15050_b200 import binding as b
    for dt in (BF, F32):
        _, ts = tensors(sizes, [dt] * len(sizes), 6)
        ts[-1][sizes[-1] // 2] = bad
        sq, norm, coef, st = call(ts, 1.0)
        assert math.isinf(sq) and sq > 0 and math.isinf(norm) and coef == 0.0 and st == b.DEV_NONFINITE
        assert not any(bool(t.any()) for t in ts)
    st, coef = torch.zeros(1, dtype=torch.int32, device=DEV), torch.empty(1, device=DEV)
    t = torch.ones(40, device=DEV)
    b.tppo_grad_clip(b.tensor_list([t]), torch.tensor([float("nan")], dtype=torch.float64, device=DEV), 1.0, None, coef, st)
    assert int(st) == b.DEV_NONFINITE and not bool(t.any()) and float(coef) == 0


def test_more_tensors_than_a_launch_takes():
    sizes = [1 + (i * 37) % 300 for i in range(2500)]
    _, ts = tensors(sizes, [(BF, F32)[i % 2] for i in range(2500)], 8)
    check(ts, 0.5 * norm64(ts))


def test_repeatable_and_captured():
    from paper_2506_15050_b200 import binding as b
    sizes = [8192 * 40 + 3, 100000, 77] * 20
    _, ts = tensors(sizes, [BF] * 60, 9)
    out = [torch.empty_like(t) for t in ts]
    first = call(ts, 1.0, out)
    for _ in range(5):
        assert call(ts, 1.0, out) == first
    grads, outs = b.tensor_list(ts), b.tensor_list(out)
    sq, norm, coef = torch.zeros(1, dtype=torch.float64, device=DEV), torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
    ws = b.workspace(b.OP_GRAD_NORM, 60, 0, 0, 0, DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        b.tppo_grad_norm(grads, sq, norm, None, ws)
        b.tppo_grad_clip(grads, sq, 1.0, outs, coef, None)
    del grads, outs                      # the captured call keeps the addresses
    graph.replay()
    assert (float(sq), float(norm), float(coef)) == first[:3]
    ts[0].mul_(2)
    graph.replay()
    got, want = [o.clone() for o in out], call(ts, 1.0, out)
    assert float(sq) == want[0] and all(torch.equal(a, o) for a, o in zip(got, out))


def test_refusals_of_the_binding():
    from paper_2506_15050_b200 import binding as b
    with pytest.raises(AssertionError):
        b.tensor_list([torch.zeros(4)])                                           # not on the GPU
    with pytest.raises(AssertionError):
        b.tensor_list([torch.zeros((4, 4), device=DEV).t()[1:]])                  # not contiguous
    with pytest.raises(AssertionError):
        b.tensor_list([torch.zeros(4, dtype=torch.float16, device=DEV)])
    t, sq = b.tensor_list([torch.zeros(4, device=DEV)]), torch.zeros(1, dtype=torch.float64, device=DEV)
    with pytest.raises(b.TppoError):
        b.tppo_grad_clip(t, sq, 1.0, b.tensor_list([torch.zeros(5, device=DEV)]), None, None)
    with pytest.raises(AssertionError):
        b.tppo_grad_clip(t, sq, 1.0, b.tensor_list([]), None, None)
    with pytest.raises(b.TppoError):
        b.tppo_grad_clip(t, sq, -1.0, None, None, None)


def test_more_than_two_to_the_31_elements():
    n = (1 << 31) + 4099
    t = torch.zeros(n, dtype=BF, device=DEV)
    t[:1000], t[-5000:] = 3.0, -0.5
    ref = math.sqrt(9 * 1000 + 0.25 * 5000)
    sq, norm, coef, st = call([t, torch.ones(7, device=DEV)], 1.0)
    whole = math.sqrt(ref * ref + 7)
    assert st == 0 and abs(norm - whole) <= 7 * U * whole
    assert bool(((t[:1000].double() - 3 / whole).abs() <= (10 * U + half_step(BF)) * 3 / whole).all())
    assert bool(((t[-5000:].double() + 0.5 / whole).abs() <= (10 * U + half_step(BF)) * 0.5 / whole).all())
    assert not bool(t[1000:-5000].any())


@pytest.mark.parametrize("sizes", [[], [0], [1], [5, 0, 3], [8192 * 3 + 1], [300] * 64, [3000] * 40, [8192 * 127, 9]])
def test_short_lists_over_and_over(sizes):
    """Lists that one cluster takes, most of its blocks with nothing to read: the same bits every time, alone, replayed back to
    back, and beside the same on a second stream."""
    from paper_2506_15050_b200 import binding as b
    _, ts = tensors(sizes, [(BF, F32)[i % 2] for i in range(len(sizes))], 11)
    grads, ref = b.tensor_list(ts), norm64(ts)
    def buffers():
        return torch.zeros(1, dtype=torch.float64, device=DEV), torch.zeros(1, device=DEV), b.workspace(b.OP_GRAD_NORM, len(ts), 0, 0, 0, DEV)
    (sq, norm, ws), (sq2, norm2, ws2) = buffers(), buffers()
    b.tppo_grad_norm(grads, sq, norm, None, ws)
    first = float(sq), float(norm)
    assert abs(first[0] - ref * ref) <= 11 * U * ref * ref and abs(first[1] - ref) <= 7 * U * ref
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    seen = torch.zeros(200, 2, dtype=torch.float64, device=DEV)
    with torch.cuda.graph(graph):
        for i in range(100):
            b.tppo_grad_norm(grads, sq, norm, None, ws)
            seen[i, 0] = sq[0]
            sq.zero_()
    side.wait_stream(torch.cuda.current_stream())
    graph.replay()
    with torch.cuda.stream(side):
        for i in range(100):
            b.tppo_grad_norm(grads, sq2, norm2, None, ws2)
            seen[100 + i, 0] = sq2[0]
            sq2.zero_()
    torch.cuda.synchronize()
    assert bool((seen[:, 0] == first[0]).all()) and float(norm) == float(norm2) == first[1]


@pytest.mark.parametrize("others", [3, 200, 1500])
def test_a_gradient_listed_twice_in_place_is_scaled_once(others):
    """Tied weights: each occurrence counts for the norm, the tensor is scaled by the coefficient, not by its square -- in one
    launch and where its two places are in different ones."""
    for dt in (BF, F32):
        _, ts = tensors([300] * others + [8192 * 5 + 3], [dt] * (others + 1), 12)
        tied = ts[-1]
        listed = [tied] + ts[:-1] + [tied, tied]
        before, ref = [t.clone() for t in ts], norm64(listed)
        sq, norm, coef, st = call(listed, 0.3 * ref)
        assert st == 0 and abs(norm - ref) <= 7 * U * ref and abs(coef - 0.3) <= 8 * U * 0.3
        for got, t in zip(ts, before):
            r = t.double() * 0.3
            assert bool(((got.double() - r).abs() <= (10 * U + half_step(dt)) * r.abs() + 2.0 ** -133).all())
