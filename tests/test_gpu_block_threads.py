"""Two host threads, each with its own stream, buffers and workspaces, call the residual join, the 8-bit products, the gradient norm
and clipping at the same time: no call takes state from another's."""
import threading

import pytest
import torch

from test_gpu_block_step import Step, outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [((520, 256), (1, 392)), ((700, 1031), (2100, 640))])
def test_steps_of_two_threads(sizes):
    steps = [Step(m, k, seed=m + k) for m, k in sizes]
    want = []
    for c in steps:
        c.step()
        torch.cuda.synchronize()
        want.append(outputs(c))
    start, failures = threading.Barrier(2), []

    def work(c, w):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                start.wait(30)
                for _ in range(40):
                    c.step()
                torch.cuda.current_stream().synchronize()
            for k, v in w.items():
                if not torch.equal(c.out[k], v):
                    failures.append(k)
        except Exception as e:  # noqa: BLE001 - reported below
            failures.append(repr(e))

    threads = [threading.Thread(target=work, args=a) for a in zip(steps, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not failures and not any(t.is_alive() for t in threads)
