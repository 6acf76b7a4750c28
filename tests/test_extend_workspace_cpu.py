"""extend_attention_nvfp4 refuses a workspace that is missing, too short or misaligned, for each of its kernels.

Host only: no call here reaches a GPU.
"""
import pytest

from _util import lib
from test_operators_abi_cpu import ALIGN, INVALID, OK_PTR, SHAPE, cache, call_attention, pages, ptr


@pytest.fixture(scope="module")
def N():
    return lib()


# (batch, tokens, query heads, KV heads, capacity, pages a sequence): up to 8 rows a sequence and KV head, up to 16, 24
# and 32, tiles; all with so few tiles that the keys are split.
FORMS = [(1, 1, 8, 2, 16384, 0), (4, 8, 8, 1, 8192, 0), (2, 8, 12, 2, 64, 200), (2, 8, 8, 1, 4096, 0),
         (1, 100, 4, 1, 16384, 0), (2, 200, 4, 2, 64, 300)]


@pytest.mark.parametrize("batch,tokens,hq,hkv,capacity,per", FORMS)
def test_a_split_call_needs_its_workspace(N, batch, tokens, hq, hkv, capacity, per):
    context = capacity * (per or 1)
    need = N.extend_attention_nvfp4_workspace_size(batch, tokens, hq, hkv, context)
    assert need > 0
    rows = tokens // batch * (hq // hkv)
    # At least two parts of every row: 128 sums and two numbers more, in fp32.
    assert need >= 2 * batch * hkv * rows * 130 * 4
    c = cache(N, batch=9, num_kv_heads=hkv, capacity=capacity)
    pg = pages(N, batch=batch, pages_per_seq=per) if per else None
    if not per:
        c.batch = batch

    def call(**kw):
        return call_attention(N, c=c, pg=pg, n=tokens, hq=hq, ld_q=hq * 128, **kw)
    for start in (None, ptr()):
        assert call(start=start, ws=None, ws_bytes=need) == INVALID
        assert call(start=start, ws=None, ws_bytes=0) == INVALID
        assert call(start=start, ws_bytes=need - 1) == SHAPE
        assert call(start=start, ws_bytes=0) == SHAPE
        for off in (4, 8, 12):
            assert call(start=start, ws=ptr(OK_PTR + off), ws_bytes=need) == ALIGN
