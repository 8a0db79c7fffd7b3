"""4-bit paged caches for the tests: e2m1 and its scales by the definition in 64 bits, and batches made of them."""
from __future__ import annotations

import numpy as np
import torch

from paged_util import Paged

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise4(x):
    """Rows x [..., D] as (codes [..., D], scale bytes [..., D / 32])."""
    x = np.asarray(x, np.float64)
    y = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(np.where(np.isfinite(y), y, 0.0)).max(-1)
    with np.errstate(divide="ignore"):
        k = np.where(top > 0, np.ceil(np.log2(top / 6.0)), 0.0)
    for _ in range(2):  # the logarithm may be one off
        k = np.where((top > 0) & (top <= 6.0 * 2.0 ** (k - 1)), k - 1, k)
        k = np.where(top > 6.0 * 2.0 ** k, k + 1, k)
    k = np.where(top > 0, np.clip(k, -126, 125), 0)
    z = np.where(np.isfinite(y), y, 0.0) / 2.0 ** k[..., None]
    gap = np.abs(np.abs(z)[..., None] - MAGNITUDES)  # the nearest; of two the one whose code is even
    near = gap.min(-1, keepdims=True)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.argmax((gap == near)[..., order], -1)]
    code = code + 8 * np.signbit(z)
    bad = ~np.isfinite(y).all(-1)  # an element that is not finite makes its block NaN
    code = np.where(bad[..., None], 0, code).astype(np.uint8)
    return code.reshape(x.shape), np.where(bad, 255, k + 127).astype(np.uint8)


def values4(code, byte):
    """The numbers that codes [..., D] with scale bytes [..., D / 32] stand for."""
    v = np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return v * np.repeat(scale, 32, -1)


def pack(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def unpack(b):
    return np.stack((b & 15, b >> 4), -1).reshape(*b.shape[:-1], -1)


class Paged4(Paged):
    """Paged with a 4-bit cache: pages [P, H_kv, page, D / 2], scales [P, H_kv, page, D / 32].

    Memory that is nobody's holds zeros, or with `junk` any codes with scales of 255.
    """

    def __init__(self, n, lens, H_q, H_kv, D, page, dtype="bf16", cache=None, junk=False, seed=0, **kw):
        super().__init__(n, lens, H_q, H_kv, D, page, dtype, None, seed=seed, junk=np.nan, **kw)
        self.cache = "e2m1"
        rng = np.random.default_rng(seed + 1)
        for name in "kv":
            x = self.vals[name]  # token-major
            dead = np.isnan(x).any((2, 3))
            code, byte = quantise4(np.where(np.isnan(x), 0.0, x))
            if junk:
                code[dead] = rng.integers(0, 16, code[dead].shape)
                byte[dead] = 255
            self.set(name, code, byte)

    def set(self, name, code, byte):
        self.vals[name] = values4(code, byte)
        self.raw[name] = np.ascontiguousarray(pack(code).transpose(0, 2, 1, 3))
        self.scales[name] = np.ascontiguousarray(byte.transpose(0, 2, 1, 3))

    def pages(self, name):
        return torch.from_numpy(self.raw[name]).cuda()

    def scale(self, name):
        return torch.from_numpy(self.scales[name]).cuda()

    def spoil(self, name, s, t, head=slice(None), block=slice(None)):
        """Makes blocks of 32 elements of a row NaN, here and on the device."""
        page, row = int(self.table[s, t // self.page]), t % self.page
        self.raw[name].reshape(*self.raw[name].shape[:3], -1, 16)[page, head, row, block] = 0
        self.scales[name][page, head, row, block] = 255
        self.vals[name].reshape(*self.vals[name].shape[:3], -1, 32)[page, row, head, block] = np.nan
        if hasattr(self, "dev"):
            self.dev[name + "_pages"].copy_(self.pages(name))
            self.dev_scales[name + "_scales"].copy_(self.scale(name))
