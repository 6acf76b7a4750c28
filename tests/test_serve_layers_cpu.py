"""The serving example's layers with an MLP, which need not know of experts: their calls, in order.  Nothing is launched."""
import types

import pytest
import torch

from _util import lib

MLP = ["residual_norm_nvfp4", "nvfp4_linear", "kv_append_rope_axes_nvfp4", "extend_attention_nvfp4", "nvfp4_quantize",
       "nvfp4_linear", "residual_norm_nvfp4", "nvfp4_linear_swiglu_quantize", "nvfp4_linear"]


def layer(**kw):
    one = torch.zeros(1)
    return types.SimpleNamespace(hidden=512, inner=256, heads=10, kv_heads=2, cache=types.SimpleNamespace(capacity=16),
                                 k_shift=None, g=[one] * 4, norm1=one, norm2=one, qkv=(one,) * 3, o=(one,) * 3,
                                 gate_up=(one,) * 3, down=(one,) * 3, **kw)


def batch(S, layer):
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    return S.Batch(layer, table, lens, 2, torch.zeros(32, 64, 2))


@pytest.fixture
def S(monkeypatch):
    lib()
    from paper_2606_15682_gb300 import serve
    calls = []
    for name in set(MLP):
        monkeypatch.setattr(serve.N, name, lambda *a, _n=name, **k: calls.append(_n))
    serve.calls = calls
    yield serve
    del serve.calls


@pytest.mark.parametrize("kw", [{}, dict(experts=0, top_k=0)], ids=["without experts", "of none"])
def test_the_calls_of_two_layers(S, kw):
    layers = [layer(**kw), layer()]
    b = batch(S, layers[0])
    b.run(layers, torch.zeros(6, 512, dtype=torch.bfloat16), torch.zeros(512))
    assert S.calls == MLP * 2 + ["residual_norm_nvfp4"]


def test_a_layer_of_experts_in_a_batch_of_another_kind_is_refused(S):
    b = batch(S, layer())
    with pytest.raises(ValueError, match="experts"):
        b.run([layer(), layer(experts=16, top_k=2)], torch.zeros(6, 512, dtype=torch.bfloat16), torch.zeros(512))
    assert not S.calls
