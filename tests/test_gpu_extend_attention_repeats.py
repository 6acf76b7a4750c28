"""extend_attention_nvfp4 gives the same bits in every run, whatever ran on the SM before it."""
import pytest
import torch

import _paged as P
from _util import lib
from test_gpu_extend_attention import queries, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("tokens,hq", [(33, 5), (27, 6), (45, 5), (70, 3), (40, 4), (130, 1)])
@pytest.mark.parametrize("capacity", [0, 3000])
def test_partly_filled_tiles_after_other_queries(N, tokens, hq, capacity):
    """Tiles of 129 to 255 rows whose last warp is partly filled, between calls whose queries are far larger or not finite
    and leave the shared memory so: a row's rounding goes by its own warp's rows, never by what stood there."""
    large = P.Case(N, [2000], 1, 0, 0, seed=801)  # for calls that occupy every SM
    case = P.Case(N, [700], 1, 0, 0, seed=800, capacity=capacity or 700)
    q = queries(tokens, hq, 60)
    q[0, 0] *= 2.0 ** 20  # the tile's first row alone is rounded in the other order
    first = run(N, case, q, [tokens])
    for spread in (2.0 ** 30, float("nan"), 2.0 ** -40, 1.0):
        other = queries(2000, hq, 61, spread=spread)
        for _ in range(3):
            run(N, large, other, [2000])
            assert torch.equal(first, run(N, case, q, [tokens]))
