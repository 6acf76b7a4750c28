"""The rotary append's binding looks at the whole shape of its table: rows of 64 (cos, sin) pairs.  No call reaches a GPU."""
import pytest
import torch

from _util import lib


@pytest.fixture(scope="module")
def N():
    return lib()


@pytest.mark.parametrize("shape", [(8,), (8, 2), (8, 64), (8, 32, 2), (8, 64, 1)])
def test_a_rotary_table_of_another_shape_is_refused(N, shape):
    c = N.KVCache(2, 2, 8, 1.0, 1.0, device="cpu")
    k, seq = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    before = N.nvfp4_launch_count()
    with pytest.raises(ValueError, match="rope_table"):
        N.kv_append_rope_axes_nvfp4(c, None, k, k, seq, seq, seq.view(3, 1), bytes(64), torch.zeros(shape), None)
    assert N.nvfp4_launch_count() == before
