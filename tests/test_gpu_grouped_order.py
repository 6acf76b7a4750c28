"""The experts' linears whatever the order is in which their clusters start: with their tiles in reverse, the clusters that start
first have none (there may be more clusters than tiles) and take those that have."""
import pytest
import torch

import _moe as M
from _util import lib
from test_gpu_linear_grouped import check_linear, check_swiglu, linear

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def lib_():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.fixture
def N(lib_):
    lib_.nvfp4_debug_inject_fault(lib_.FAULT_GROUPED_REVERSED)
    yield lib_
    lib_.nvfp4_debug_inject_fault(lib_.FAULT_NONE)


# Tiles of 64 tokens: at most some 260 on 128 experts, 6 and 10 of them there.  Of 256: 240 on 8 experts, 128 there.  More
# tiles than clusters: 448 of 336.
FEW = {"one of many": [0] * 3 + [128] + [0] * 124, "some of many": [0] * 60 + [100, 1, 0, 31] + [0] * 64}
MANY = {"one": [0, 0, 2000, 0, 0, 0, 0, 0], "two": [0, 900, 0, 0, 0, 0, 0, 700]}


@pytest.mark.parametrize("counts", FEW, ids=lambda c: c)
@pytest.mark.parametrize("k", [256, 768, 1536])  # units asked for three, two and one ahead
@pytest.mark.parametrize("mx", [False, True])
def test_rows_in_small_tiles(N, counts, k, mx):
    check_linear(N, FEW[counts], 272, k, mx)


@pytest.mark.parametrize("counts", MANY, ids=lambda c: c)
@pytest.mark.parametrize("k", [256, 768, 1536])
def test_rows_in_large_tiles(N, counts, k):
    check_linear(N, MANY[counts], 4096, k)


def test_more_tiles_than_clusters(N):
    check_linear(N, [257] * 28, 2048, 256)


@pytest.mark.parametrize("form", ["nvfp4", "mxfp4", "mxfp4 rotated"])
@pytest.mark.parametrize("k", [256, 1536])
def test_swiglu(N, form, k):
    for counts, inner in ((FEW["some of many"], 256), (MANY["two"], 2048)):
        N.nvfp4_debug_inject_fault(N.FAULT_GROUPED_REVERSED)
        check_swiglu(N, counts, inner, k, form != "nvfp4", form.endswith("rotated"), per_expert=False)


@pytest.mark.parametrize("tokens", [100, 4000])
def test_tokens_without_experts(N, tokens):
    """A padded batch: clusters for its choices, no tile."""
    plan = M.make_plan(N, torch.full((tokens, 4), -1, dtype=torch.int32), 64)
    a, w = M.Rows(N, plan, 256, 1), M.Weights(N, 64, 1024, 256, 3)
    out = torch.full((plan.max_rows, 1024), -7.0, dtype=BF, device="cuda")
    for _ in range(2):  # in reverse, and not
        linear(N, plan, a, w, out, 1024, 256, False)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0 and (out == -7).all()
