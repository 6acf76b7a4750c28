"""A plan without tokens has buffers without rows, whose address is null: the calls on rows do nothing with them, and refuse the
same sizes and steps as with tokens.  No call here reaches a GPU."""
import pytest
import torch

from _util import lib
from test_moe_abi_cpu import LINEARS, ROWS, SHAPE, INVALID, call, plan

EMPTY = dict(x=None, rows=None, codes=None, scales=None, out=None, d_y=None, d_w=None, base=None, weights=None, a_codes=None,
             a_scales=None)


@pytest.fixture(scope="module")
def N():
    return lib()


@pytest.mark.parametrize("name", ROWS[1:] + LINEARS)
def test_empty_buffers(N, name):
    before = N.nvfp4_launch_count()
    assert call(N, name, p=plan(N, n_tokens=0, row_of=None), **EMPTY) == 0
    assert N.nvfp4_launch_count() == before


@pytest.mark.parametrize("name", LINEARS)
def test_sizes_and_steps_are_checked_without_tokens_too(N, name):
    none = plan(N, n_tokens=0, row_of=None)
    wrong = [(dict(k=384), SHAPE), (dict(k=0), SHAPE)]
    wrong += [(dict(inner=192), SHAPE)] if "swiglu" in name else [(dict(n=250), SHAPE), (dict(ld_out=248), SHAPE)]
    wrong += [(dict(a_step=2), INVALID)] if name.startswith("nvfp4") else []
    for kw, code in wrong:
        assert call(N, name, p=none, **EMPTY, **kw) == code, kw


def test_binding(N):
    p, E, n, k = N.MoEPlan(0, 2, 4, device="cpu"), 4, 512, 256

    def u8(*shape):
        return torch.empty(*shape, dtype=torch.uint8)
    a, w, h = (u8(0, k // 2), u8(0)), (u8(E, n, k // 2), u8(E * n * k // 16)), (u8(0, n // 4), u8(0))
    g, gw, out = torch.ones(1), torch.ones(E), torch.empty(0, n, dtype=torch.bfloat16)
    assert out.data_ptr() == 0 and a[0].data_ptr() == 0
    before = N.nvfp4_launch_count()
    N.nvfp4_linear_grouped(p, *a, g, *w, gw, out, n, k, stream=0)
    N.mxfp4_linear_grouped(p, *a, *w, out, n, k, stream=0)
    N.nvfp4_linear_grouped_swiglu_quantize(p, *a, g, *w, gw, n // 2, k, g, *h, stream=0)
    N.mxfp4_linear_grouped_swiglu_quantize(p, *a, *w, n // 2, k, *h, stream=0)
    assert N.nvfp4_launch_count() == before
