"""Paged and contiguous test caches, and the operators' plain forms in 64 bits."""
import math

import numpy as np
import torch

from oracle import nvfp4_oracle as O

D = 128
GK, GV = 0.013, 0.021
# Bytes that no quantizer writes: E4M3 NaN in both signs, and a mix of codes.
JUNK_SCALES = (0x7F, 0xFF)

E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])
E1M2 = np.array([0, .5, 1, 1.5, 2, 2.5, 3, 3.5, -4, -3.5, -3, -2.5, -2, -1.5, -1, -.5])


def e4m3(b):
    b = np.asarray(b, np.int64)
    e, m = b >> 3, b & 7
    return np.where(e == 0, m / 512.0, (1 + m / 8.0) * 2.0 ** (e - 7.0))


def values(codes, scales, kv_format):
    """64-bit e2m1 (or e1m2) * e4m3 of code rows [..., 64] and scale rows [..., 8] (numpy)."""
    grid = E1M2 if kv_format else E2M1
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 128)
    return grid[nib] * np.repeat(e4m3(scales), 16, axis=-1)


class Case:
    """A cache with seeded rows for `lens` tokens of each sequence; everything else in it is junk."""

    def __init__(self, N, lens, hkv, page=0, kv_format=0, seed=0, capacity=None, spare_pages=3, scale_range=(0x28, 0x48)):
        rng = np.random.default_rng(seed)
        B, top = len(lens), max(max(lens), 1)
        self.lens, self.hkv, self.kv_format, self.N = list(lens), hkv, kv_format, N
        if page:
            per = -(-(capacity or top) // page)
            rows = B * per + spare_pages
            self.table = rng.permutation(rows)[:B * per].reshape(B, per).astype(np.int32)
            size = page
        else:
            size = capacity or top
            per, rows = 1, B
            self.table = np.arange(B, dtype=np.int32).reshape(B, 1)
        self.size, self.rows, self.per, self.page = size, rows, per, page
        self.cache = N.KVCache(rows, hkv, size, GK, GV, kv_format=kv_format)
        self.data = {}
        for name in ("k", "v"):
            codes = rng.integers(0, 256, (rows, hkv, size, 64), dtype=np.uint8)
            if kv_format:  # the nibble -8 is never written
                codes = np.where((codes & 15) == 8, codes ^ 8, codes)
                codes = np.where((codes >> 4) == 8, codes ^ 0x80, codes).astype(np.uint8)
            scales = rng.choice(np.array(JUNK_SCALES, np.uint8), (rows, hkv, size, 8))
            for b, n in enumerate(lens):
                for i in range(per):
                    m = min(size, n - i * size)
                    if m > 0:
                        scales[self.table[b, i], :, :m] = rng.integers(*scale_range, (hkv, m, 8), dtype=np.uint8)
            self.data[name] = (codes, scales)
            getattr(self.cache, name + "_codes").copy_(torch.from_numpy(codes))
            getattr(self.cache, name + "_scales").copy_(torch.from_numpy(scales))
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.cache.seq_lens = self.lens_dev
        self.set_table(self.table)

    def set_table(self, table):
        self.table = table
        self.pages = None
        if self.page:
            self.table_dev = torch.from_numpy(np.ascontiguousarray(table)).cuda()
            self.pages = self.N.KVPages(self.table_dev, self.lens_dev)

    @property
    def context(self):
        return self.size * self.per

    def rows_of(self, name, b):
        """(64-bit values [hkv, len, 128] of sequence b without g, present [len])."""
        codes, scales = self.data[name]
        n = min(self.lens[b], self.context)
        out, here = np.zeros((self.hkv, n, 128)), np.zeros(n, bool)
        for i in range(-(-n // self.size)):
            page, m = self.table[b, i], min(self.size, n - i * self.size)
            if 0 <= page < self.rows:
                out[:, i * self.size:i * self.size + m] = values(codes[page, :, :m], scales[page, :, :m], self.kv_format)
                here[i * self.size:i * self.size + m] = True
        return out, here


def attention64(case, q, news, scale, cap=0.0, window=0, slopes=None, prefix=None, doc_start=None):
    """(out, sum of weight * |v|, rows that see nothing), 64 bits, [tokens, heads, 128]; q bf16 on the GPU."""
    hq = q.shape[1]
    group = hq // case.hkv
    q = q.double().cpu().numpy()
    out, mass = np.zeros((q.shape[0], hq, 128)), np.zeros((q.shape[0], hq, 128))
    empty = np.ones(q.shape[0], bool)
    first = 0
    for b, n in enumerate(news):
        length = min(case.lens[b], case.context)
        (k, here), (v, _) = case.rows_of("k", b), case.rows_of("v", b)
        t = np.arange(length)
        for j in range(n):
            p, i = length - n + j, first + j
            see = here & ((t <= p) | (t < (prefix[b] if prefix is not None else 0)))
            if p < 0:
                see &= False
            if window:
                see &= t > p - window
            if doc_start is not None:
                see &= t >= doc_start[i]
            if not see.any():
                continue
            empty[i] = False
            for h in range(hq):
                s = scale * float(np.float32(GK)) * (k[h // group][see] @ q[i, h])
                if cap:
                    s = cap * np.tanh(s / cap)
                if slopes is not None:
                    s = s - float(slopes[h]) * np.abs(p - t[see])
                w = np.exp(s - s.max())
                w /= w.sum()
                vv = v[h // group][see] * float(np.float32(GV))
                out[i, h], mass[i, h] = w @ vv, w @ np.abs(vv)
        first += n
    return out, mass, empty


def half_ulp(y):
    e = np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -126)))
    return 2.0 ** (e - 8)


def bf16(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).float().numpy()
