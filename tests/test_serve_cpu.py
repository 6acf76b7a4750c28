"""What the serving example refuses before it launches anything."""
import types

import pytest
import torch

from _util import lib


@pytest.fixture(scope="module")
def S():
    lib()
    from paper_2606_15682_gb300 import serve
    return serve


def batch(S, layer):
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    return S.Batch(layer, table, lens, 2, torch.zeros(32, 64, 2))


def layer(k_shift):
    return types.SimpleNamespace(hidden=512, inner=256, heads=10, kv_heads=2, cache=types.SimpleNamespace(capacity=16),
                                 k_shift=k_shift)


@pytest.mark.parametrize("shifted", [0, 1])
def test_a_cap_over_shifted_keys_is_refused(S, shifted):
    layers = [layer(None), layer(None)]
    layers[shifted] = layer(torch.zeros(2, 128))
    b = batch(S, layers[0])
    x = torch.zeros(6, 512, dtype=torch.bfloat16)
    before = S.N.nvfp4_launch_count()
    with pytest.raises(ValueError, match="k_shift"):
        b.run(layers, x, x[0], logit_cap=30.0)
    assert (b.pages.seq_lens == 0).all(), "the sequences are as they were"
    assert S.N.nvfp4_launch_count() == before
