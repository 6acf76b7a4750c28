"""extend_attention_nvfp4 against the plain form in 64 bits.

Tolerance, per output: half a bf16 ulp for the output's own rounding, plus
2^-10 of sum(weight * |v|).  The softmax weights are rounded to f16 (2^-11 of
each); the rest of the 2^-10 covers what is held in fp32: scores (some 2^-22 of
a few hundred), exp2 (2^-22), the sums over at most a few thousand keys
(2^-13 if every addition erred one way).  Q, K and V are exact in f16.
"""
import math

import numpy as np
import pytest
import torch

import _paged as P
from _util import lib

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


def run(N, case, q, news, uniform=False, out=None, **kw):
    n, hq = q.shape[0], q.shape[1]
    start = None if uniform else torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
    B = len(news)
    nbytes = N.extend_attention_nvfp4_workspace_size(B, n, hq, case.hkv, case.context)
    ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda") if nbytes else None  # NaN to who reads it
    out = torch.full((n, hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    N.extend_attention_nvfp4(case.cache, q, kw.pop("scale", SCALE), out, ws, q_start=start, pages=case.pages, **kw)
    return out


def queries(n, hq, seed, ld=None, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.randn(n, ld or hq, 128, generator=g, device="cuda") * spread
    return wide.to(torch.bfloat16)[:, :hq]


def check(N, case, q, news, uniform=False, **kw):
    dev = {k: (torch.as_tensor(v, device="cuda") if k in ("slopes", "prefix_lens", "doc_start") and v is not None else v)
           for k, v in kw.items()}
    out = run(N, case, q, news, uniform, **dev)
    torch.cuda.synchronize()
    ref, mass, empty = P.attention64(case, q, news, kw.get("scale", SCALE), kw.get("logit_cap", 0.0), kw.get("window", 0),
                                     kw.get("slopes"), kw.get("prefix_lens"), kw.get("doc_start"))
    y = out.double().cpu().numpy()
    assert np.isfinite(y).all()
    assert (y[empty] == 0).all(), "a query that sees nothing gets zeros"
    over = np.abs(y - ref) - (P.half_ulp(ref) * (1 + 2.0 ** -6) + 2.0 ** -10 * mass)
    assert over.max() <= 0, f"worst excess {over.max():.3e} at {np.unravel_index(over.argmax(), over.shape)}"
    return out


# heads, kv heads: groups of 1, 5, 6, 8, 16
LAYOUTS = [(2, 2), (5, 1), (12, 2), (8, 1), (16, 1)]


@pytest.mark.parametrize("hq,hkv", LAYOUTS)
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("page", [0, 16, 37])
def test_one_token_each(N, hq, hkv, fmt, page):
    lens = [1, 2, 15, 16, 17, 127, 128, 129, 300, 0, 1025, 64]
    case = P.Case(N, lens, hkv, page, fmt, seed=1 + hq)
    check(N, case, queries(len(lens), hq, 5), [1] * len(lens), uniform=True)
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("hq,hkv", LAYOUTS)
@pytest.mark.parametrize("news,lens", [
    ([4, 4, 4], [100, 4, 777]),
    ([3, 0, 7, 1], [3, 50, 130, 1]),
    ([16, 2], [400, 200]),
    ([33, 9], [129, 260]),
    ([130, 61], [130, 300]),
    ([257], [600]),
])
def test_several_tokens(N, hq, hkv, news, lens):
    for fmt, page in ((0, 0), (1, 48)):
        case = P.Case(N, lens, hkv, page, fmt, seed=3)
        check(N, case, queries(sum(news), hq, 6), news)
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("new,length", [(1, 1), (2, 2), (127, 127), (128, 128), (129, 129), (255, 511), (300, 1100)])
@pytest.mark.parametrize("hq,hkv", [(2, 1), (5, 1)])
def test_prompt_lengths_at_tile_edges(N, new, length, hq, hkv):
    case = P.Case(N, [length], hkv, 0, 0, seed=length)
    check(N, case, queries(new, hq, new), [new], uniform=True)


OPTIONS = [
    dict(logit_cap=5.0),
    dict(window=1),
    dict(window=70),
    dict(slopes="alibi"),
    dict(prefix_lens=[40, 500, 0]),
    dict(doc_start="docs"),
    dict(logit_cap=20.0, window=90, slopes="alibi", prefix_lens=[100, 0, 64], doc_start="docs"),
    dict(scale=1.7, slopes="steep"),
]


@pytest.mark.parametrize("opt", range(len(OPTIONS)))
@pytest.mark.parametrize("news", [[1, 1, 1], [5, 3, 8], [150, 90, 200]])
@pytest.mark.parametrize("page,fmt", [(0, 0), (24, 1)])
def test_scores_and_masks(N, opt, news, page, fmt):
    lens, hq, hkv = [333, 90, 201], 10, 2
    kw = dict(OPTIONS[opt])
    rng = np.random.default_rng(opt)
    if kw.get("slopes") == "alibi":
        kw["slopes"] = (2.0 ** (-8 * np.arange(1, hq + 1) / hq)).astype(np.float32)
    elif kw.get("slopes") == "steep":
        kw["slopes"] = np.linspace(-0.01, 40.0, hq).astype(np.float32)
    if "prefix_lens" in kw:
        kw["prefix_lens"] = np.array(kw["prefix_lens"], np.int32)
    if "doc_start" in kw:
        start = []
        for n, length in zip(news, lens):
            for p in range(length - n, length):
                start.append(p // 61 * 61 if rng.random() < 0.9 else length + 5)  # some queries see nothing
        kw["doc_start"] = np.array(start, np.int32)
    case = P.Case(N, lens, hkv, page, fmt, seed=11)
    check(N, case, queries(sum(news), hq, 8), news, **kw)
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("news", [[1, 1, 1], [40, 2, 100]])
def test_absent_pages_and_lengths_out_of_range(N, news):
    lens = [200, 130, 100]
    case = P.Case(N, lens, 2, 16, 0, seed=21)
    table = case.table.copy()
    table[0, :5] = -1          # left behind by a window
    table[1, 2] = case.rows    # past the pool
    table[2, :] = 1 << 30      # nothing there at all
    case.set_table(table)
    check(N, case, queries(sum(news), 10, 3), news)
    assert N.nvfp4_get_device_status() == 0
    # A length above the capacity is clamped and reported; more queries than tokens see nothing at first.
    case = P.Case(N, [64, 3], 1, 0, 0, seed=22, capacity=64)
    case.lens_dev.copy_(torch.tensor([1000, 3], dtype=torch.int32))
    q = queries(sum([2, 10]), 4, 4)
    out = run(N, case, q, [2, 10])
    ref, _, empty = P.attention64(case, q, [2, 10], SCALE)
    assert (out.double().cpu().numpy()[empty] == 0).all() and empty.sum() == 7
    assert N.nvfp4_get_device_status() == 7
    # q_start beyond the tokens: clamped and reported, nothing out of place is written.
    case = P.Case(N, [64, 30], 1, 0, 0, seed=23)
    out = torch.full((4, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    bad = torch.tensor([0, 2, 90], dtype=torch.int32, device="cuda")
    nbytes = N.extend_attention_nvfp4_workspace_size(2, 3, 4, 1, 64)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
    N.extend_attention_nvfp4(case.cache, q[:3], SCALE, out[:3], ws, q_start=bad)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 7
    assert torch.isfinite(out).all() and (out[3] == 7).all()


@pytest.mark.parametrize("news", [[1], [40], [300]])
def test_extreme_scores_and_queries(N, news):
    """Large and tiny queries: rows of 2^15 and of 2^-60, and a row of zeros (a plain mean of V)."""
    case = P.Case(N, [500], 2, 0, 0, seed=31)
    for spread in (200.0, 2.0 ** -60, 0.0):
        check(N, case, queries(news[0], 4, 9, spread=spread), news)
    # One query row with channels 2^20 apart: the small ones count only as much as they can.
    q = queries(news[0], 4, 10)
    q[:, :, ::2] *= 2.0 ** -20
    check(N, case, q, news)


@pytest.mark.parametrize("news", [[1, 1], [6, 3], [140, 129]])
def test_strided_queries_other_stream_and_repeats(N, news):
    case = P.Case(N, [700, 260], 2, 32, 0, seed=41)
    q = queries(sum(news), 10, 11, ld=14)  # queries cut from a wider projection output
    assert not q.is_contiguous()
    first = check(N, case, q, news)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = run(N, case, q, news)
    s.synchronize()
    assert torch.equal(first, again)
    for _ in range(5):
        assert torch.equal(first, run(N, case, q, news))


def test_matches_decode_attention_within_rounding(N):
    """One token per sequence without options is what decode_attention_nvfp4 computes."""
    lens = [1500, 7, 1024, 2048]
    case = P.Case(N, lens, 2, 0, 0, seed=51, capacity=2048)
    q = queries(4, 10, 12)
    out = run(N, case, q, [1] * 4, uniform=True)
    ws = torch.empty(N.decode_attention_nvfp4_workspace_size(4, 10, 2048), dtype=torch.uint8, device="cuda")
    ref = torch.empty_like(out)
    N.decode_attention_nvfp4(case.cache, q, SCALE, ref, ws)
    _, mass, _ = P.attention64(case, q, [1] * 4, SCALE)
    d = np.abs((out.double() - ref.double()).cpu().numpy())
    assert (d <= 2 * P.half_ulp(ref.double().cpu().numpy()) + 2.0 ** -9 * mass).all()


@pytest.mark.parametrize("new", [1, 64])
def test_rows_past_32_bit_offsets(N, new):
    """A pool whose codes end past 2^32 bytes, the sequence's pages at both ends of it."""
    page, hkv = 64, 8
    rows = (1 << 32) // (hkv * page * 64) + 40
    case = P.Case(N, [256], hkv, page, 0, seed=61)
    small, pool = case.cache, N.KVCache(1, hkv, 2, P.GK, P.GV)
    pool.batch, pool.capacity, pool.seq_lens = rows, page, case.lens_dev
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        src = getattr(small, name)
        big = torch.empty((rows,) + tuple(src.shape[1:]), dtype=torch.uint8, device="cuda")
        setattr(pool, name, big)
    where = np.array([[rows - 1, 0, rows - 2, 5]], np.int32)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        for i in range(4):
            getattr(pool, name)[int(where[0, i])].copy_(getattr(small, name)[int(case.table[0, i])])
    q = queries(new, 16, 13)
    want = run(N, case, q, [new])
    case.cache = pool
    case.rows = rows
    pages = N.KVPages(torch.from_numpy(where).cuda(), case.lens_dev)
    case.pages = pages
    got = run(N, case, q, [new])
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0
    assert torch.equal(want, got)


def test_no_tokens_is_a_no_op(N):
    case = P.Case(N, [10], 1)
    before = N.nvfp4_launch_count()
    q = torch.empty(0, 4, 128, dtype=torch.bfloat16, device="cuda")
    N.extend_attention_nvfp4(case.cache, q, SCALE, q, None)
    assert N.nvfp4_launch_count() == before


@pytest.mark.parametrize("news", [[1, 1], [70, 5]])
def test_captures_in_a_graph(N, news):
    case = P.Case(N, [300, 90], 2, 16, 0, seed=71)
    q = queries(sum(news), 4, 14)
    want = run(N, case, q, news)
    start = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device="cuda")
    nbytes = N.extend_attention_nvfp4_workspace_size(2, sum(news), 4, 2, case.context)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
    out = torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        N.extend_attention_nvfp4(case.cache, q, SCALE, out, ws, q_start=start, pages=case.pages)
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
