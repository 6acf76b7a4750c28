"""extend_attention_nvfp4 over contexts of more than 512 keys, against the plain form in 64 bits.

Tolerance, per output: half a bf16 ulp for the output's own rounding; 2^-10 of
sum(weight * |v|) for the weights' rounding to f16 (2^-11 of each) and for what
is held in fp32; and 2^-29 of (largest weight) * sum(|v|) over the visible keys.
The last is f16's underflow: the largest weight is held at 2^4 or more, and
half a subnormal step is 2^-25.
"""
import math

import numpy as np
import pytest
import torch

import _paged as P
from _util import lib
from test_gpu_extend_attention import queries, run

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


def reference(case, q, news, scale=SCALE, logit_cap=0.0, window=0, slopes=None, prefix_lens=None, doc_start=None):
    """(out, bound without the output's rounding, rows that see nothing), in 64 bits on the GPU."""
    dev = q.device
    hq = q.shape[1]
    group = hq // case.hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    bound, empty = torch.zeros_like(out), torch.ones(q.shape[0], dtype=torch.bool, device=dev)
    first = 0
    for b, n in enumerate(news):
        length = min(case.lens[b], case.context)
        if n == 0 or length == 0:
            first += n
            continue
        (k, here), (v, _) = case.rows_of("k", b), case.rows_of("v", b)
        k, v = (torch.from_numpy(x).to(dev) for x in (k, v))
        t = torch.arange(length, device=dev)
        p = length - n + torch.arange(n, device=dev)[:, None]
        see = t <= p
        if prefix_lens is not None:
            see = see | (t < int(prefix_lens[b]))
        see = see & (p >= 0) & torch.from_numpy(here).to(dev)
        if window:
            see = see & (t > p - window)
        if doc_start is not None:
            see = see & (t >= torch.as_tensor(doc_start[first:first + n], device=dev)[:, None])
        some = see.any(1)
        empty[first:first + n] = ~some
        for h in range(hq):
            s = scale * float(np.float32(P.GK)) * (q[first:first + n, h].double() @ k[h // group].T)
            if logit_cap:
                s = logit_cap * torch.tanh(s / logit_cap)
            if slopes is not None:
                s = s - float(slopes[h]) * (p - t).abs()
            s = s.masked_fill(~see, -math.inf)
            w = torch.softmax(s, 1)[some]
            vv = v[h // group] * float(np.float32(P.GV))
            rows = torch.arange(first, first + n, device=dev)[some]
            out[rows, h] = w @ vv
            bound[rows, h] = 2.0 ** -10 * (w @ vv.abs()) + 2.0 ** -29 * w.amax(1, keepdim=True) * (
                see[some].double() @ vv.abs())
        first += n
    return out.cpu().numpy(), bound.cpu().numpy(), empty.cpu().numpy()


def check(N, case, q, news, uniform=False, skip=None, **kw):
    dev = {k: (torch.as_tensor(v, device="cuda") if k in ("slopes", "prefix_lens", "doc_start") and v is not None else v)
           for k, v in kw.items()}
    out = run(N, case, q, news, uniform, **dev)
    torch.cuda.synchronize()
    ref, bound, empty = reference(case, q, news, **kw)
    y = out.double().cpu().numpy()
    keep = np.ones(len(y), bool)
    if skip is not None:
        keep[skip] = False
    assert np.isfinite(y[keep]).all()
    assert (y[empty] == 0).all(), "a query that sees nothing gets zeros"
    over = (np.abs(y - ref) - (P.half_ulp(ref) * (1 + 2.0 ** -6) + bound))[keep]
    assert over.max() <= 0, f"worst excess {over.max():.3e} at {np.unravel_index(over.argmax(), over.shape)}"
    return out


def options(name, hq, news, lens, seed=0):
    """A fresh set of options; lens long enough for their numbers to matter."""
    rng = np.random.default_rng(seed)
    alibi = (2.0 ** (-8 * np.arange(1, hq + 1) / hq)).astype(np.float32)
    docs = []
    for n, length in zip(news, lens):
        for p in range(length - n, length):
            docs.append(p // 701 * 701 if rng.random() < 0.9 else length + 5)  # some queries see nothing
    docs = np.array(docs, np.int32)
    prefix = np.array([(977 * (b + 1)) % 1500 if b % 3 else 0 for b in range(len(news))], np.int32)
    return {
        "plain": {},
        "cap": dict(logit_cap=8.0),
        "window": dict(window=333),
        "window_one": dict(window=1),
        "bias": dict(slopes=alibi),
        "prefix": dict(prefix_lens=prefix),
        "prefix_window": dict(prefix_lens=prefix, window=600),
        "docs": dict(doc_start=docs),
        "all": dict(logit_cap=20.0, window=900, slopes=alibi, prefix_lens=prefix, doc_start=docs),
    }[name]


# Few rows of a sequence and KV head (8, 16, 24, 32), then tiles of 256.
FEW = [
    ([1] * 6, (5, 1)), ([1] * 6, (8, 2)), ([1] * 6, (2, 2)),   # 8
    ([2] * 6, (6, 1)), ([1] * 6, (16, 1)),                     # 16
    ([4] * 6, (10, 2)), ([3, 9, 0, 1, 2, 7], (6, 1)),          # 24
    ([4] * 6, (8, 1)), ([1] * 6, (26, 1)),                     # 32
]
LENS = [513, 3000, 1, 1153, 2047, 700]


@pytest.mark.parametrize("opt", ["plain", "cap", "window", "window_one", "bias", "prefix", "prefix_window", "docs", "all"])
@pytest.mark.parametrize("which", range(len(FEW)))
@pytest.mark.parametrize("page,fmt", [(0, 0), (37, 1), (64, 0)])
def test_few_rows(N, which, opt, page, fmt):
    news, (hq, hkv) = FEW[which]
    case = P.Case(N, LENS, hkv, page, fmt, seed=100 + which)
    check(N, case, queries(sum(news), hq, which), news, uniform=len(set(news)) == 1 and page != 64,
          **options(opt, hq, news, LENS, which))
    assert N.nvfp4_get_device_status() == 0


# (new tokens, lengths, heads): several tiles a sequence, tiles cut into parts, sequences of very different lengths.
MANY = [
    ([60], [2000], (5, 1)),
    ([129, 3, 260], [1500, 2600, 700], (4, 2)),
    ([700], [700], (3, 1)),
    ([40] * 12, [600 + 130 * i for i in range(12)], (12, 2)),
]


@pytest.mark.parametrize("opt", ["plain", "cap", "window", "window_one", "bias", "prefix", "prefix_window", "docs", "all"])
@pytest.mark.parametrize("which", range(len(MANY)))
@pytest.mark.parametrize("page,fmt", [(0, 1), (48, 0)])
def test_many_rows(N, which, opt, page, fmt):
    news, lens, (hq, hkv) = MANY[which]
    case = P.Case(N, lens, hkv, page, fmt, seed=200 + which)
    check(N, case, queries(sum(news), hq, which), news, uniform=len(set(news)) == 1, **options(opt, hq, news, lens, which))
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("news", [[1, 1, 1], [3, 3, 3], [50, 70, 90]])
@pytest.mark.parametrize("page", [16, 100])
def test_absent_pages(N, news, page):
    lens = [1700, 900, 600]
    case = P.Case(N, lens, 2, page, 0, seed=300)
    table = case.table.copy()
    table[0, : 900 // page] = -1      # left behind by a window
    table[1, 3] = case.rows           # past the pool
    table[1, 5] = -7
    table[2, :] = 1 << 30             # nothing there at all
    case.set_table(table)
    check(N, case, queries(sum(news), 10, 3), news)
    check(N, case, queries(sum(news), 10, 3), news, window=400)
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("news", [[1, 1], [4, 4], [150, 20]])
def test_spread_scores(N, news):
    """Large, tiny and zero queries, scores that rise and that fall along the keys."""
    case = P.Case(N, [2500, 800], 2, 0, 0, seed=310)
    for spread in (200.0, 2.0 ** -60, 0.0):
        check(N, case, queries(sum(news), 10, 9, spread=spread), news)
    for slope in (-0.05, 0.05, 30.0, -30.0):
        check(N, case, queries(sum(news), 10, 9), news, slopes=np.full(10, slope, np.float32))


@pytest.mark.parametrize("news", [[1, 1], [4, 4], [150, 20]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite_harms_no_other(N, news, bad):
    case = P.Case(N, [1500, 800], 2, 32, 0, seed=320)
    q = queries(sum(news), 10, 9).contiguous()
    q[0, :, 5] = bad
    check(N, case, q, news, skip=[0])
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("news", [[1] * 5, [2] * 5, [40] * 5])
def test_same_bits_in_any_order_and_stream(N, news):
    case = P.Case(N, [600, 2100, 40, 1300, 999], 2, 16, 0, seed=330)
    q = queries(sum(news), 10, 9)
    first = run(N, case, q, news, True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = [run(N, case, q, news, True) for _ in range(4)]
    s.synchronize()
    assert all(torch.equal(first, x) for x in again)


@pytest.mark.parametrize("news", [[1, 1], [3, 3], [60, 60]])
def test_length_above_the_capacity_is_clamped_and_reported(N, news):
    case = P.Case(N, [800, 700], 2, 0, 0, seed=340, capacity=800)
    case.lens_dev.copy_(torch.tensor([5000, 700], dtype=torch.int32))
    q = queries(sum(news), 8, 4)
    out = run(N, case, q, news, True)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 7
    ref, bound, _ = reference(case, q, news)
    assert (np.abs(out.double().cpu().numpy() - ref) <= P.half_ulp(ref) * (1 + 2.0 ** -6) + bound).all()


@pytest.mark.parametrize("seed", range(3))
def test_maxima_that_move_by_little(N, seed):
    """Scores whose running maxima pass the threshold for a new one by roundings: a biased draft over many keys."""
    news, lens = [4] * 12, [4001 - 97 * i for i in range(12)]
    case = P.Case(N, lens, 2, 128, 1, seed=350 + seed)
    slopes = np.concatenate([2.0 ** (-8 * np.arange(1, 6) / 5), -(2.0 ** (-8 * np.arange(1, 6) / 5))]).astype(np.float32)
    check(N, case, queries(48, 10, seed), news, uniform=True, slopes=slopes)
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("news", [[1, 1], [4, 4], [150, 20]])
@pytest.mark.parametrize("log_spread", [16, 24, 30, 40])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_scores_past_fp32s_integers(N, news, log_spread, cap):
    """Queries so large that scores are far apart; finite everywhere, and the file's tolerance where the largest key is
    clear of the others by 40 and by the scores' error (2^-18 of the sum of their terms, more than fp32 sums of 128
    exact products can lose)."""
    case = P.Case(N, [1500, 800], 2, 0, 0, seed=360)
    q = queries(sum(news), 10, 9, spread=2.0 ** log_spread)
    out = run(N, case, q, news, logit_cap=cap)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    if cap:
        return
    clear, first = np.zeros((len(q), 10), bool), 0
    for b, n in enumerate(news):
        k = torch.from_numpy(case.rows_of("k", b)[0]).cuda() * float(np.float32(P.GK)) * SCALE
        t = torch.arange(case.lens[b], device="cuda")
        hidden = t > (case.lens[b] - n + torch.arange(n, device="cuda"))[:, None]
        for h in range(10):
            qq, kk = q[first:first + n, h].double(), k[h // 5]
            top = (qq @ kk.T).masked_fill(hidden, -math.inf).topk(2, dim=1).values
            error = 2.0 ** -18 * (qq.abs() @ kk.abs().T).amax(1)
            clear[first:first + n, h] = (top[:, 0] - top[:, 1] > 2 * error + 40).cpu().numpy()
        first += n
    assert clear.any()
    ref, bound, _ = reference(case, q, news)
    over = np.abs(out.double().cpu().numpy() - ref) - (P.half_ulp(ref) * (1 + 2.0 ** -6) + bound)
    assert over[clear].max() <= 0
