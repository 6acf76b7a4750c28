"""residual_norm_nvfp4 against the plain form in 64 bits.

Tolerance, per output: half a bf16 ulp (1 + 2^-6 of it, for results at a binade's
edge) plus 2^-19 of the magnitudes added: r is a handful of fp32 operations, h
also a sum of up to 32768 squares in fp32 in at least 8 x 32 partial sums (some
2^-17 of the sum if all errors agreed, half of that after the square root) and
rsqrt (2^-22); h is therefore given 2^-17."""
import numpy as np
import pytest
import torch

import _paged as P
from _util import f32, lib, u8
from oracle import nvfp4_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


def rand(rows, cols, seed, scale=1.0, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, ld or cols, generator=g, device="cuda") * scale).to(torch.bfloat16)[:, :cols]


def plain(x, y, w, post=None, gate=None, per=1, alpha=1.0, eps=1e-6):
    x = x.double().cpu().numpy()
    mag = np.abs(x)
    if y is not None:
        z = y.double().cpu().numpy()
        if post is not None:
            z = z / np.sqrt((z * z).mean(1, keepdims=True) + eps) * post.double().cpu().numpy()
        if gate is not None:
            z = z * gate.double().cpu().numpy()[np.arange(len(x)) // per]
        mag = mag + np.abs(alpha * z)
        x = x + float(np.float32(alpha)) * z
    inv = 1 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    wn = w.double().cpu().numpy() if w is not None else 1.0
    return x, mag, x * inv * wn, mag * inv * np.abs(wn)


def close(got, want, mag, rel):
    y = got.double().cpu().numpy()
    assert np.isfinite(y).all()
    over = np.abs(y - want) - P.half_ulp(want) * (1 + 2.0 ** -6) - rel * mag
    assert over.max() <= 0, over.max()


COLS = [8, 64, 136, 512, 1536, 5120, 8192, 16384, 16392, 32768]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("rows", [1, 5])
@pytest.mark.parametrize("post,gate", [(False, 0), (True, 0), (False, 1), (True, 2), (True, 100)])
def test_norms_and_sum(N, cols, rows, post, gate):
    x, y = rand(rows, cols, 1, 3.0), rand(rows, cols, 2, 0.5)
    w, wp = rand(1, cols, 3)[0], rand(1, cols, 4)[0]
    g = rand(-(-rows // gate), cols, 5) if gate else None
    r, h = (torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    N.residual_norm_nvfp4(x, y, r, h, w, eps=1e-5, w_post=wp if post else None, gate=g, rows_per_gate=gate or 1, alpha=0.37)
    torch.cuda.synchronize()
    want_r, mag_r, want_h, mag_h = plain(x, y, w, wp if post else None, g, gate or 1, 0.37, 1e-5)
    close(r, want_r, mag_r, 2.0 ** -19 if not post else 2.0 ** -17)
    close(h, want_h, mag_h, 2.0 ** -17)


@pytest.mark.parametrize("rows,cols", [(1, 64), (3, 192), (127, 1536), (130, 5120), (257, 512), (300, 16448)])
def test_nvfp4_output_is_the_quantized_bf16_output(N, rows, cols):
    x, y, w = rand(rows, cols, 1, 3.0), rand(rows, cols, 2), rand(1, cols, 3)[0]
    x[:, 5] *= 40
    h = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    r = torch.empty_like(h)
    N.residual_norm_nvfp4(x, y, r, h, w)
    gs = float(O.tensor_scale(f32(h)))
    g = torch.tensor([gs], dtype=torch.float32, device="cuda")
    codes, scales = [], []
    for _ in range(3):
        codes.append(torch.full((rows, cols // 2), 0xAA, dtype=torch.uint8, device="cuda"))
        scales.append(torch.full((N.nvfp4_scales_bytes(rows, cols, N.SCALES_MMA),), 0xAA, dtype=torch.uint8, device="cuda"))
    N.nvfp4_quantize(h, g, codes[0], scales[0], N.SCALES_MMA)
    r2, h2 = torch.empty_like(h), torch.empty_like(h)
    N.residual_norm_nvfp4(x, y, r2, h2, w, g_out=g, codes=codes[1], scales=scales[1])
    N.residual_norm_nvfp4(x, y, r2, None, w, g_out=g, codes=codes[2], scales=scales[2])
    torch.cuda.synchronize()
    assert torch.equal(h, h2) and torch.equal(r, r2)
    for i in (1, 2):
        assert torch.equal(codes[0], codes[i]) and torch.equal(scales[0], scales[i])
    oc, os_ = O.quantize(f32(h), np.float32(gs))
    assert np.array_equal(u8(codes[1]), oc)
    assert np.array_equal(u8(scales[1]), O.scales_to_mma(os_).reshape(-1))
    assert N.nvfp4_get_device_status() == 0


def test_forms_without_some_inputs_or_outputs(N):
    rows, cols = 9, 264
    x, y, w = rand(rows, cols, 1), rand(rows, cols, 2), rand(1, cols, 3)[0]
    r, h, h2 = (torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    N.residual_norm_nvfp4(x, None, None, h, w)                 # a plain norm
    _, _, want, mag = plain(x, None, w)
    close(h, want, mag, 2.0 ** -17)
    N.residual_norm_nvfp4(x, y, r, None, None, alpha=-2.0)     # a sum alone
    want, mag, _, _ = plain(x, y, None, alpha=-2.0)
    close(r, want, mag, 2.0 ** -19)
    N.residual_norm_nvfp4(x, y, None, h, w)                    # no residual out
    N.residual_norm_nvfp4(x, y, r, h2, w)
    assert torch.equal(h, h2)
    inplace = x.clone()
    N.residual_norm_nvfp4(inplace, y, inplace, h, w)           # residual updated where it stands
    assert torch.equal(inplace, r) and torch.equal(h, h2)


def test_padded_rows_streams_and_zero_rows(N):
    rows, cols = 33, 512
    x, y, w = rand(rows, cols, 1, ld=520), rand(rows, cols, 2, ld=1024), rand(1, cols, 3)[0]
    x[7] = 0
    y[7] = 0
    r, h = (torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        N.residual_norm_nvfp4(x, y, r, h, w, w_post=w)
    s.synchronize()
    want_r, mag_r, want_h, mag_h = plain(x, y, w, w)
    close(r, want_r, mag_r, 2.0 ** -17)
    close(h, want_h, mag_h, 2.0 ** -17)
    assert (h[7] == 0).all()
    before = N.nvfp4_launch_count()
    N.residual_norm_nvfp4(x[:0], y[:0], r[:0], h[:0], w)
    assert N.nvfp4_launch_count() == before


def test_large_and_small_rows(N):
    """Rows whose squares are far from one another in size, within fp32."""
    cols = 1536
    for scale in (1e15, 1e-12):
        x, y, w = rand(4, cols, 1, scale), rand(4, cols, 2, scale), rand(1, cols, 3)[0]
        r, h = (torch.empty(4, cols, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        N.residual_norm_nvfp4(x, y, r, h, w)
        want_r, mag_r, want_h, mag_h = plain(x, y, w)
        close(r, want_r, mag_r, 2.0 ** -19)
        close(h, want_h, mag_h, 2.0 ** -17)


def test_bad_tensor_scale_is_reported(N):
    rows, cols = 5, 128
    x, w = rand(rows, cols, 1), rand(1, cols, 3)[0]
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        g = torch.tensor([bad], device="cuda")
        codes = torch.full((rows, cols // 2), 0xAA, dtype=torch.uint8, device="cuda")
        scales = torch.full((N.nvfp4_scales_bytes(rows, cols, N.SCALES_MMA),), 0xAA, dtype=torch.uint8, device="cuda")
        N.residual_norm_nvfp4(x, None, None, None, w, g_out=g, codes=codes, scales=scales)
        assert N.nvfp4_get_device_status() == 1
        assert (codes == 0).all() and (scales == 0).all()
