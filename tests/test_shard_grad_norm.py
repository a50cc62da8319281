"""The gradient norm of a model whose gradients are spread over ranks: two gloo ranks on CPU, float64 arithmetic in the kernels'
place.  Under test: `shard.global_sum_sq`, after which every rank clips by the norm of all gradients."""
import math
import os
import socket

import numpy as np
import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_2506_15050_b200 import shard


def gradients():
    g = np.random.default_rng(3)
    return [torch.from_numpy(g.standard_normal(n)) for n in (5, 1000, 0, 33, 7)]


def worker(rank, world, port, out, bad):
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    try:
        mine = gradients()[rank::world]
        s = torch.tensor([sum(float((t * t).sum()) for t in mine)], dtype=torch.float64)
        if bad and rank == 1:
            s.fill_(math.inf)
        got = [None] * world
        dist.all_gather_object(got, float(shard.global_sum_sq(s)))
        if rank == 0:
            torch.save(got, out)
    finally:
        dist.destroy_process_group()


def run(tmp_path, bad):
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    out = str(tmp_path / f"norm{bad}.pt")
    mp.spawn(worker, args=(2, port, out, bad), nprocs=2, join=True)
    return torch.load(out)


def test_two_ranks_have_the_norm_of_all_gradients(tmp_path):
    whole = sum(float((t * t).sum()) for t in gradients())
    a, b = run(tmp_path, False)
    assert a == b and abs(a - whole) <= 4 * 2.0 ** -53 * whole          # the same terms in another order


def test_one_rank_that_is_not_finite_stops_all(tmp_path):
    assert run(tmp_path, True) == [math.inf, math.inf]


def test_alone_it_changes_nothing():
    s = torch.tensor([3.0], dtype=torch.float64)
    assert shard.global_sum_sq(s) is s and float(s) == 3.0
