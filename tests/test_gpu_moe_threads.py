"""Plans sorted from two host threads at once, of different numbers of experts: each call as if it were alone."""
import threading

import numpy as np
import pytest
import torch

import _moe as M
from _util import lib

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("tokens", [100, 4000, 40000])  # one CTA, a cluster, chunks
def test_sorts_of_two_threads(N, tokens):
    """Their kernels want 36 and 139 KB of shared memory: neither call's limit is the other's."""
    work = []
    for experts in (260, 1024):
        idx = np.random.default_rng(experts).integers(-1, experts, (tokens, 2)).astype(np.int32)
        work.append((N.MoEPlan(tokens, 2, experts), torch.as_tensor(idx, device="cuda"), M.plan_of(idx, experts)))
    torch.cuda.synchronize()
    failures, start = [], threading.Barrier(len(work))

    def run(plan, idx):
        stream = torch.cuda.Stream()
        start.wait()
        try:
            for _ in range(3000):
                N.moe_sort(plan, idx, stream=stream)
            stream.synchronize()
        except Exception as e:  # a thread's own would be lost
            failures.append(e)
    threads = [threading.Thread(target=run, args=w[:2]) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
    for plan, _, (row_start, rows, row_of) in work:
        assert np.array_equal(plan.row_start.cpu().numpy(), row_start) and np.array_equal(plan.rows.cpu().numpy(), rows)
        assert np.array_equal(plan.row_of.cpu().numpy(), row_of)
    assert N.nvfp4_get_device_status() == 0
