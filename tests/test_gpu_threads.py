"""Calls of two host threads, each with its own stream, buffers and workspace: the C entry points hold no
lock and keep no state that one call could take from another."""
import threading

import pytest
import torch

from dense_util import BF, DEV, F32, gen

pytestmark = pytest.mark.gpu

CALLS = 3000


def norm_fwd(M, N, dtype, stream):
    """One call of the C entry point with its arguments prepared, so that the threads meet inside it."""
    from paper_2506_15050_b200 import binding as b
    x = torch.randn((M, N), generator=gen(N), device=DEV).to(dtype)
    y, t = torch.empty_like(x), b._DTYPES[dtype]
    args = (x.data_ptr(), t, M, N, N, None, None, b.F32, 1e-5, y.data_ptr(), N, None, None, None, stream.cuda_stream)
    return lambda: b._lib.tppo_layer_norm_fwd(*args), (y,), (x,)


def norm_bwd(M, N, dtype, stream):
    from paper_2506_15050_b200 import binding as b
    g = gen(N)
    x, dy = (torch.randn((M, N), generator=g, device=DEV).to(dtype) for _ in range(2))
    mean, rstd = x.float().mean(1), x.float().std(1).reciprocal()
    dx, dg, db = torch.empty_like(x), torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    ws = b.workspace(b.OP_LAYER_NORM, M, 0, 0, N, DEV)
    args = (dy.data_ptr(), x.data_ptr(), b._DTYPES[dtype], M, N, N, N, None, b.F32, mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), N,
            dg.data_ptr(), db.data_ptr(), None, ws.data_ptr(), ws.numel(), stream.cuda_stream)
    return lambda: b._lib.tppo_layer_norm_bwd(*args), (dx, dg, db), (x, dy, mean, rstd, ws)


def narrow(M, K, N, stream):
    from paper_2506_15050_b200 import binding as b
    g = gen(K)
    x, w = torch.randn((M, K), generator=g, device=DEV).to(BF), torch.randn((K, N), generator=g, device=DEV).to(BF)
    y = torch.empty((M, N), device=DEV)
    args = (x.data_ptr(), K, w.data_ptr(), N, M, K, N, None, b.F32, b.ACT_NONE, None, 0, y.data_ptr(), b.F32, N, None, 0, None, None, 0,
            stream.cuda_stream)
    return lambda: b._lib.tppo_linear_fwd(*args), (y,), (x, w)


def policy(V, stream):
    from paper_2506_15050_b200 import binding as b
    R, g = 64, gen(V)
    logits = torch.randn((R, V), generator=g, device=DEV).to(BF)
    targets = torch.randint(0, V, (R,), generator=g, device=DEV, dtype=torch.int32)
    old, adv = torch.randn(R, generator=g, device=DEV) - 8, torch.randn(R, generator=g, device=DEV)
    logp, loss, stats = torch.empty(R, device=DEV), torch.empty(1, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV)
    d, ws = torch.empty_like(logits), b.workspace(b.OP_POLICY_LOSS, R, 0, R, V, DEV)

    args = (logits.data_ptr(), b.BF16, R, V, V, targets.data_ptr(), None, None, R, None, old.data_ptr(), adv.data_ptr(), R, 0.2, 0.28, 0.0,
            logp.data_ptr(), None, loss.data_ptr(), stats.data_ptr(), d.data_ptr(), b.DLOGITS_FULL, b.POLICY_CLUSTER_SMEM,
            ws.data_ptr(), ws.numel(), stream.cuda_stream)
    return lambda: b._lib.tppo_policy_loss_fwd_bwd(*args), (logp, loss, d), (logits, targets, old, adv, stats, ws)


# each pair shares one kernel and differs in the shared memory that it asks for
PAIRS = {
    "norm fwd": lambda s, t: (norm_fwd(2048, 4096, BF, s), norm_fwd(2048, 10240, BF, t)),
    "norm fwd, odd": lambda s, t: (norm_fwd(2048, 4101, F32, s), norm_fwd(2048, 8001, F32, t)),
    "norm bwd, one phase": lambda s, t: (norm_bwd(600, 520, F32, s), norm_bwd(600, 5120, F32, t)),
    "norm bwd, two phases": lambda s, t: (norm_bwd(600, 2051, BF, s), norm_bwd(600, 10001, BF, t)),
    "narrow linear": lambda s, t: (narrow(64, 64, 1, s), narrow(64, 48000, 1, t)),
    "policy loss": lambda s, t: (policy(4096, s), policy(150000, t)),
}


@pytest.mark.parametrize("pair", PAIRS)
def test_two_threads(pair):
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    calls = PAIRS[pair](*streams)
    torch.cuda.synchronize()
    want = []
    for call, outs, _ in calls:
        assert call() == 0
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    codes, start = [set(), set()], threading.Barrier(2)

    def loop(k):
        start.wait()
        for _ in range(CALLS):
            codes[k].add(calls[k][0]())

    threads = [threading.Thread(target=loop, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert codes == [{0}, {0}]
    for (_, outs, _), w in zip(calls, want):
        assert all(torch.equal(a, b) for a, b in zip(outs, w))
