"""kv_append_rope_axes_nvfp4 where a token is refused on the device."""
import numpy as np
import pytest
import torch

import _paged as P
from _util import lib
from oracle import nvfp4_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n", [3, 3000])
def test_queries_off_the_rotary_table_are_zero_whatever_they_hold(N, n, bad):
    hq, hkv = 6, 2
    case = P.Case(N, [0], hkv, 64, 0, seed=1, capacity=n)
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(n, h, 128, generator=g, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    q[1, :, ::3] = bad
    q[2, 0, 77] = bad
    rope = np.arange(n, dtype=np.int32)[:, None] % 50
    rope[1] = 50            # one past the table
    rope[2] = -1
    table = torch.from_numpy(O.rope_table(50).astype(np.float32)).cuda()
    q_out = torch.full((n, hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    i32 = lambda a: torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    N.kv_append_rope_axes_nvfp4(case.cache, q, k, v, i32(np.zeros(n)), i32(np.arange(n)), i32(rope), bytes(64), table, q_out,
                                pages=case.pages)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 7
    assert (q_out[1] == 0).all() and (q_out[2] == 0).all()
    assert torch.isfinite(q_out[0].float()).all() and (q_out[0] != 0).any()
