"""kv_append_rope_axes_nvfp4 and kv_read_nvfp4: rotation, quantized append and
read-back over contiguous and paged caches, bit for bit against the oracle."""
import numpy as np
import pytest
import torch

import _paged as P
from _util import f32, lib, u8
from oracle import nvfp4_oracle as O

pytestmark = pytest.mark.gpu
TABLE = 97  # rotary positions


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


AXES = {1: [0] * 64, 2: [0] * 40 + [1] * 24, 3: [0] * 16 + [1] * 24 + [2] * 24,
        4: [(i * 7 + i // 9) % 4 for i in range(64)]}  # the last one interleaved


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device="cuda")


def append(N, hq, hkv, places, axes, page, fmt, seed, batch=3, context=120, shift=True, wide=False, rope_pos=None):
    """Append rows at `places` [(sequence, position)] and compare the whole cache and the rotated queries."""
    rng = np.random.default_rng(seed)
    n = len(places)
    case = P.Case(N, [0] * batch, hkv, page, fmt, seed=seed, capacity=context)
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (torch.randn(n, hq + 2 * hkv + (3 if wide else 0), 128, generator=g, device="cuda") * 2).to(torch.bfloat16)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:hq + 2 * hkv]
    if not wide:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    seq, pos = (np.array([p[i] for p in places], np.int32) for i in range(2))
    if rope_pos is None:
        rope_pos = rng.integers(0, TABLE, (n, axes)).astype(np.int32)
    table = O.rope_table(TABLE).astype(np.float32)
    m = rng.standard_normal((hkv, 128)).astype(np.float32) if shift else None
    q_out = torch.full((n, hq, 128), float("nan"), dtype=torch.bfloat16, device="cuda") if hq else None
    N.kv_append_rope_axes_nvfp4(case.cache, q if hq else None, k, v, i32(seq), i32(pos), i32(rope_pos), AXES[axes],
                                torch.from_numpy(table).cuda(), q_out,
                                k_shift=None if m is None else torch.from_numpy(m).cuda(), pages=case.pages)
    torch.cuda.synchronize()
    # The oracle's rotation takes one table row per token: make that row of each token's axes.
    ok_rope = ((rope_pos >= 0) & (rope_pos < TABLE)).all(1)
    rows = np.stack([table[np.where(ok_rope, rope_pos[:, AXES[axes][c]], 0), c] for c in range(64)], 1)
    own = np.arange(n)
    if hq:
        want = np.where(ok_rope[:, None, None], P.bf16(O.rope_f32(f32(q), own, rows)), 0)
        assert np.array_equal(f32(q_out), want)
    kr = O.rope_f32(f32(k), own, rows)
    if shift:
        kr = (kr - m).astype(np.float32)
    element = "e1m2" if fmt else "e2m1"
    kept = np.ones(n, bool)
    for name, x, gs in (("k", kr, P.GK), ("v", f32(v), P.GV)):
        codes, scales = O.quantize(x.reshape(-1, 128), gs, element)
        codes, scales = codes.reshape(n, hkv, 64), scales.reshape(n, hkv, 8)
        want_c, want_s = (a.copy() for a in case.data[name])
        for i in range(n):
            inside = 0 <= seq[i] < batch and 0 <= pos[i] < case.context
            page_i = case.table[seq[i], pos[i] // case.size] if inside else -1
            kept[i] = ok_rope[i] and 0 <= page_i < case.rows
            if kept[i]:
                want_c[page_i, :, pos[i] % case.size] = codes[i]
                want_s[page_i, :, pos[i] % case.size] = scales[i]
        assert np.array_equal(u8(getattr(case.cache, name + "_codes")), want_c), name
        assert np.array_equal(u8(getattr(case.cache, name + "_scales")), want_s), name
    assert N.nvfp4_get_device_status() == (0 if kept.all() else 7)
    return case


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
@pytest.mark.parametrize("page,fmt", [(0, 0), (1, 0), (16, 1), (37, 0)])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (10, 2), (0, 3), (5, 5)])
def test_append_bit_exact(N, axes, page, fmt, hq, hkv):
    places = [(0, 0), (2, 5), (1, 119), (0, 36), (0, 37), (2, 64), (1, 15), (1, 16)]
    append(N, hq, hkv, places, axes, page, fmt, seed=axes + hq, shift=hq != 4, wide=hq == 10)


@pytest.mark.parametrize("n", [1, 3, 70, 3000])
def test_append_sizes(N, n):
    """From one token to enough for the form with several heads per lane group."""
    places = [(i % 3, i // 3) for i in range(n)]
    append(N, 14, 2, places, 3, 64, 0, seed=n, context=max(120, n // 3 + 1), wide=True)


def test_append_outside_is_skipped_and_reported(N):
    good = [(0, 1), (1, 2)]
    append(N, 4, 2, good + [(3, 0)], 1, 16, 0, seed=1)          # no such sequence
    append(N, 4, 2, good + [(-1, 0)], 1, 16, 0, seed=2)
    append(N, 4, 2, good + [(0, 128)], 1, 16, 0, seed=3)        # context is 8 pages of 16
    append(N, 4, 2, good + [(0, -2)], 1, 0, 0, seed=4)
    rope = np.array([[0, 5, 6], [3, TABLE, 1], [1, 2, -1], [4, 4, 4]], np.int32)  # off the table
    append(N, 4, 2, good + [(2, 9), (2, 10)], 3, 16, 0, seed=5, rope_pos=rope)


def test_append_to_an_absent_page(N):
    case = P.Case(N, [0, 0], 1, 8, 0, seed=9, capacity=40)
    table = case.table.copy()
    table[1, 2] = -1
    case.set_table(table)
    x = torch.ones(2, 1, 128, dtype=torch.bfloat16, device="cuda")
    rope = torch.from_numpy(O.rope_table(50).astype(np.float32)).cuda()
    N.kv_append_rope_axes_nvfp4(case.cache, None, x, x, i32([0, 1]), i32([17, 17]), i32([[17], [17]]), AXES[1], rope, None,
                                pages=case.pages)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 7
    codes = u8(case.cache.k_codes)
    changed = {p for p in range(case.rows) if not np.array_equal(codes[p], case.data["k"][0][p])}
    assert changed == {case.table[0, 2]}


def test_one_axis_is_the_plain_append(N):
    """Contiguous cache, one axis whose position is the place: kv_append_rope_nvfp4's bytes."""
    n, hkv, cap = 40, 2, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(n, hkv, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    seq, pos = i32(np.arange(n) % 4), i32(np.arange(n))
    table = torch.empty(cap, 64, 2, device="cuda")
    N.nvfp4_rope_table(table)
    shift = torch.randn(hkv, 128, generator=g, device="cuda")
    for fmt in (0, 1):
        a, b = (N.KVCache(4, hkv, cap, P.GK, P.GV, kv_format=fmt) for _ in range(2))
        N.kv_append_rope_nvfp4(a, k, v, seq, pos, table, k_shift=shift)
        N.kv_append_rope_axes_nvfp4(b, None, k, v, seq, pos, pos.view(n, 1), AXES[1], table, None, k_shift=shift)
        for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name


@pytest.mark.parametrize("page,fmt,hkv", [(0, 0, 1), (16, 0, 3), (37, 1, 2), (1, 1, 8)])
def test_read_bit_exact(N, page, fmt, hkv):
    lens = [130, 1, 77]
    case = P.Case(N, lens, hkv, page, fmt, seed=4, scale_range=(0, 0x7F))
    rng = np.random.default_rng(5)
    seq = rng.integers(0, 3, 301).astype(np.int32)
    pos = np.array([rng.integers(0, lens[b]) for b in seq], np.int32)
    for want_k, want_v in ((True, True), (True, False), (False, True)):
        outs = [torch.full((301, hkv, 128), float("nan"), dtype=torch.bfloat16, device="cuda") if w else None
                for w in (want_k, want_v)]
        N.kv_read_nvfp4(case.cache, i32(seq), i32(pos), *outs, pages=case.pages)
        torch.cuda.synchronize()
        for name, out, g in (("k", outs[0], P.GK), ("v", outs[1], P.GV)):
            if out is None:
                continue
            codes, scales = case.data[name]
            at = case.table[seq, pos // case.size], slice(None), pos % case.size
            exact = P.values(codes[at], scales[at], fmt).astype(np.float32)  # exact in 32 bits
            want = P.bf16(exact * np.float32(g))
            assert np.array_equal(f32(out).view(np.int32) & 0x7FFFFFFF, want.view(np.int32) & 0x7FFFFFFF)
            assert np.array_equal(f32(out), want)
    assert N.nvfp4_get_device_status() == 0


def test_read_outside_gives_zeros(N):
    case = P.Case(N, [40, 20], 2, 8, 0, seed=6)
    table = case.table.copy()
    table[0, 1] = case.rows + 1
    case.set_table(table)
    seq, pos = i32([0, 0, 2, 1, -1, 1]), i32([3, 9, 0, 40, 0, 19])  # row 1 absent, 2 and 4 no sequence, 3 past the end
    k = torch.full((6, 2, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    N.kv_read_nvfp4(case.cache, seq, pos, k, v, pages=case.pages)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 7
    for out in (k, v):
        zero = (out == 0).all(-1).all(-1).tolist()
        assert zero == [False, True, True, True, True, False]


def test_append_then_read_round_trip(N):
    """What comes back is within the format's rounding of what went in: a quarter of the block's largest value."""
    n, hkv = 50, 2
    case = P.Case(N, [0], hkv, 16, 0, seed=7, capacity=64)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(n, hkv, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    zero = i32(np.zeros(n))
    table = torch.empty(64, 64, 2, device="cuda")
    N.nvfp4_rope_table(table)
    N.kv_append_rope_axes_nvfp4(case.cache, None, k, v, zero, i32(np.arange(n)), i32(np.zeros((n, 1))), AXES[1], table, None,
                                pages=case.pages)  # position 0: no rotation
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    N.kv_read_nvfp4(case.cache, zero, i32(np.arange(n)), ko, vo, pages=case.pages)
    for x, y in ((k, ko), (v, vo)):
        top = x.float().unflatten(-1, (8, 16)).abs().amax(-1, keepdim=True)
        assert ((x.float() - y.float()).unflatten(-1, (8, 16)).abs() <= 0.25 * top).all()
