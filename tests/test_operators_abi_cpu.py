"""Host-only checks of the operators around the linears: what they refuse
before anything is launched.  No call here reaches a GPU."""
import ctypes
import itertools

import pytest
import torch

from _util import lib

OK_PTR = 0x10000  # aligned, never dereferenced: validation fails first
INVALID, SHAPE, ALIGN = 1, 2, 3


@pytest.fixture(scope="module")
def N():
    return lib()


def ptr(v=OK_PTR):
    return ctypes.c_void_p(v)


def cache(N, **kw):
    c = dict(k_codes=OK_PTR, k_scales=OK_PTR, v_codes=OK_PTR, v_scales=OK_PTR, seq_lens=OK_PTR, batch=4, num_kv_heads=2,
             head_dim=128, capacity=64, k_gscale=0.1, v_gscale=0.1, kv_format=0)
    c.update(kw)
    return N.KVCacheStruct(**c)


def pages(N, **kw):
    p = dict(table=OK_PTR, seq_lens=OK_PTR, batch=2, pages_per_seq=2)
    p.update(kw)
    return N.KVPagesStruct(**p)


BAD_CACHES = [(dict(k_codes=None), INVALID), (dict(v_scales=None), INVALID), (dict(k_gscale=0.0), INVALID),
              (dict(v_gscale=float("nan")), INVALID), (dict(kv_format=2), INVALID), (dict(head_dim=64), SHAPE),
              (dict(batch=0), SHAPE), (dict(capacity=0), SHAPE), (dict(num_kv_heads=-1), SHAPE),
              (dict(k_codes=OK_PTR + 8), ALIGN), (dict(v_scales=OK_PTR + 4), ALIGN)]
BAD_PAGES = [(dict(table=None), INVALID), (dict(batch=0), SHAPE), (dict(pages_per_seq=0), SHAPE),
             (dict(pages_per_seq=1 << 30), SHAPE), (dict(table=OK_PTR + 2), ALIGN)]


def call_append(N, c=None, pg=None, **kw):
    a = dict(q=ptr(), ld_q=1280, hq=4, k=ptr(), ld_k=256, v=ptr(), ld_v=256, seq=ptr(), pos=ptr(), rope_pos=ptr(), axes=1,
             axis=bytes(64), n=2, table=ptr(), positions=64, shift=None, out=ptr())
    a.update(kw)
    return N._lib.kv_append_rope_axes_nvfp4(
        None if c is False else ctypes.byref(c or cache(N)), None if pg is None else ctypes.byref(pg), a["q"], a["ld_q"],
        a["hq"], a["k"], a["ld_k"], a["v"], a["ld_v"], a["seq"], a["pos"], a["rope_pos"], a["axes"], a["axis"], a["n"],
        a["table"], a["positions"], a["shift"], a["out"], ctypes.c_void_p(0))


def call_read(N, c=None, pg=None, **kw):
    a = dict(seq=ptr(), pos=ptr(), n=2, k=ptr(), v=ptr())
    a.update(kw)
    return N._lib.kv_read_nvfp4(None if c is False else ctypes.byref(c or cache(N)), None if pg is None else ctypes.byref(pg),
                                a["seq"], a["pos"], a["n"], a["k"], a["v"], ctypes.c_void_p(0))


def call_attention(N, c=None, pg=None, opt=None, **kw):
    a = dict(q=ptr(), ld_q=512, n=4, hq=4, start=None, out=ptr(), ws=ptr(), ws_bytes=1 << 40)
    a.update(kw)
    o = dict(softmax_scale=0.1, logit_cap=0.0, slopes=None, window=0, prefix_lens=None, doc_start=None)
    o.update(opt or {})
    o = N.AttentionOptionsStruct(**o)
    return N._lib.extend_attention_nvfp4(
        None if c is False else ctypes.byref(c or cache(N)), None if pg is None else ctypes.byref(pg), a["q"], a["ld_q"],
        a["n"], a["hq"], a["start"], ctypes.byref(o) if opt is not False else None, a["out"], a["ws"], a["ws_bytes"],
        ctypes.c_void_p(0))


def call_norm(N, **kw):
    a = dict(x=ptr(), ld_x=256, y=ptr(), ld_y=256, rows=2, cols=256, post=None, gate=None, per=1, alpha=1.0, w=ptr(),
             eps=1e-6, r=ptr(), h=ptr(), g=None, codes=None, scales=None)
    a.update(kw)
    return N._lib.residual_norm_nvfp4(a["x"], a["ld_x"], a["y"], a["ld_y"], a["rows"], a["cols"], a["post"], a["gate"],
                                      a["per"], a["alpha"], a["w"], a["eps"], a["r"], a["h"], a["g"], a["codes"],
                                      a["scales"], ctypes.c_void_p(0))


def test_cache_and_pages_are_checked_by_every_call(N):
    for call in (call_append, call_read, call_attention):
        assert call(N, c=False) == INVALID
        for kw, code in BAD_CACHES:
            assert call(N, c=cache(N, **kw)) == code, (call.__name__, kw)
        for kw, code in BAD_PAGES:
            assert call(N, pg=pages(N, **kw)) == code, (call.__name__, kw)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(seq=None), INVALID), (dict(pos=None), INVALID),
    (dict(rope_pos=None), INVALID), (dict(table=None), INVALID), (dict(out=None), INVALID), (dict(axis=None), INVALID),
    (dict(axis=bytes([0] * 63 + [1])), INVALID), (dict(axes=0), SHAPE), (dict(axes=5), SHAPE), (dict(hq=0), SHAPE),
    (dict(ld_q=504), SHAPE), (dict(ld_k=128), SHAPE), (dict(ld_v=128), SHAPE), (dict(n=-1), SHAPE),
    (dict(positions=0), SHAPE), (dict(n=1 << 40), SHAPE), (dict(ld_q=1284), ALIGN), (dict(ld_k=260), ALIGN),
    (dict(q=ptr(OK_PTR + 2)), ALIGN), (dict(out=ptr(OK_PTR + 8)), ALIGN), (dict(shift=ptr(OK_PTR + 4)), ALIGN),
    (dict(table=ptr(OK_PTR + 8)), ALIGN), (dict(pos=ptr(OK_PTR + 2)), ALIGN)])
def test_append_refusals(N, kw, code):
    assert call_append(N, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(seq=None), INVALID), (dict(pos=None), INVALID), (dict(k=None, v=None), INVALID), (dict(n=-1), SHAPE),
    (dict(n=1 << 31), SHAPE), (dict(k=ptr(OK_PTR + 8)), ALIGN), (dict(seq=ptr(OK_PTR + 1)), ALIGN)])
def test_read_refusals(N, kw, code):
    assert call_read(N, **kw) == code


@pytest.mark.parametrize("kw,opt,code", [
    ({}, False, INVALID), (dict(q=None), None, INVALID), (dict(out=None), None, INVALID),
    ({}, dict(softmax_scale=0.0), INVALID), ({}, dict(softmax_scale=float("inf")), INVALID),
    ({}, dict(logit_cap=-1.0), INVALID), ({}, dict(logit_cap=float("nan")), INVALID), ({}, dict(window=-1), INVALID),
    (dict(hq=3), None, SHAPE), (dict(hq=0), None, SHAPE), (dict(n=5), None, SHAPE), (dict(n=-4), None, SHAPE),
    (dict(ld_q=504), None, SHAPE), (dict(q=ptr(OK_PTR + 8)), None, ALIGN), (dict(out=ptr(OK_PTR + 8)), None, ALIGN),
    (dict(ld_q=516), None, ALIGN), (dict(start=ptr(OK_PTR + 2)), None, ALIGN), ({}, dict(slopes=OK_PTR + 2), ALIGN),
    ({}, dict(prefix_lens=OK_PTR + 1), ALIGN), ({}, dict(doc_start=OK_PTR + 3), ALIGN)])
def test_attention_refusals(N, kw, opt, code):
    assert call_attention(N, opt=opt, **kw) == code


def test_attention_needs_lengths_and_its_workspace(N):
    assert call_attention(N, c=cache(N, seq_lens=None)) == INVALID
    assert call_attention(N, pg=pages(N, seq_lens=None)) == INVALID
    need = N.extend_attention_nvfp4_workspace_size(4, 4, 4, 2, 64)
    if need:
        assert call_attention(N, ws=None) == INVALID
        assert call_attention(N, ws_bytes=need - 1) == SHAPE
        assert call_attention(N, ws=ptr(OK_PTR + 8)) == ALIGN


def test_workspace_size_covers_every_size(N):
    """Non-negative, zero for nothing, and never beyond what a workspace can reasonably be."""
    size = N.extend_attention_nvfp4_workspace_size
    for bad in ((0, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 0, 2, 64), (1, 1, 4, 0, 64), (1, 1, 4, 2, 0), (1, -1, 4, 2, 64)):
        assert size(*bad) == 0
    for b, n, (hq, hk), ctx in itertools.product((1, 3, 64, 1000), (1, 5, 4096), ((1, 1), (40, 8), (64, 8)), (1, 700, 1 << 20)):
        assert 0 <= size(b, n, hq, hk, ctx) < 1 << 32


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVALID), (dict(r=None, h=None), INVALID), (dict(w=None), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(alpha=float("inf")), INVALID), (dict(codes=ptr()), INVALID),
    (dict(codes=ptr(), scales=ptr()), INVALID), (dict(g=ptr(), scales=ptr()), INVALID),
    (dict(y=None, h=None), INVALID), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=12), SHAPE),
    (dict(cols=32776, ld_x=40000, ld_y=40000), SHAPE), (dict(ld_x=248), SHAPE), (dict(ld_y=248), SHAPE),
    (dict(gate=ptr(), per=0), SHAPE), (dict(cols=40, codes=ptr(), scales=ptr(), g=ptr()), SHAPE),
    (dict(x=ptr(OK_PTR + 8)), ALIGN), (dict(y=ptr(OK_PTR + 8)), ALIGN), (dict(ld_x=260), ALIGN), (dict(w=ptr(OK_PTR + 2)), ALIGN),
    (dict(gate=ptr(OK_PTR + 8)), ALIGN), (dict(r=ptr(OK_PTR + 4)), ALIGN),
    (dict(codes=ptr(), scales=ptr(OK_PTR + 2), g=ptr()), ALIGN)])
def test_norm_refusals(N, kw, code):
    assert call_norm(N, **kw) == code


def test_binding_checks_its_tensors(N):
    """The binding refuses what the C entry point cannot see: types, shapes, strides."""
    bf, i32 = torch.bfloat16, torch.int32
    x = torch.zeros(4, 64, dtype=bf)
    c = N.KVCache(2, 2, 8, 1.0, 1.0, device="cpu")
    seq = torch.zeros(3, dtype=i32)
    rope = torch.zeros(8, 64, 2)
    k = torch.zeros(3, 2, 128, dtype=bf)
    with pytest.raises(ValueError):
        N.KVPages(torch.zeros(2, 3), torch.zeros(2, dtype=i32))
    with pytest.raises(ValueError):
        N.KVPages(torch.zeros(2, 3, dtype=i32), torch.zeros(3, dtype=i32))
    with pytest.raises(ValueError):
        N.kv_append_rope_axes_nvfp4(c, None, k, k, seq, seq, seq.view(3, 1), [0] * 63, rope, None)
    with pytest.raises(ValueError):
        N.kv_append_rope_axes_nvfp4(c, None, k.float(), k, seq, seq, seq.view(3, 1), [0] * 64, rope, None)
    with pytest.raises(ValueError):
        N.kv_append_rope_axes_nvfp4(c, None, k[:, :1], k, seq, seq, seq.view(3, 1), [0] * 64, rope, None)
    with pytest.raises(ValueError):
        N.kv_append_rope_axes_nvfp4(c, k, k, k, seq, seq, seq.view(3, 1), [0] * 64, rope, None)
    with pytest.raises(ValueError):
        N.kv_read_nvfp4(c, seq, seq.long(), k, None)
    with pytest.raises(ValueError):
        N.kv_read_nvfp4(c, seq, seq, k[:2], None)
    with pytest.raises(ValueError):
        N.extend_attention_nvfp4(c, k.transpose(0, 1), 1.0, k, None)
    with pytest.raises(ValueError):
        N.extend_attention_nvfp4(c, k, 1.0, k, None, slopes=torch.zeros(3))
    with pytest.raises(ValueError):
        N.residual_norm_nvfp4(x, x.float(), x, x, x[0])
    with pytest.raises(ValueError):
        N.residual_norm_nvfp4(x, x, x, x, x[0], gate=x, rows_per_gate=2)
