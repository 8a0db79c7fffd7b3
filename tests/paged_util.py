"""Paged caches for the tests: made on the host with their float64 contents, and the operators in 64 bits."""
from __future__ import annotations

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # of a rounding, relative to the value


def bf16_round(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def quantise(x):
    """Rows x [..., D] (float32) as (e4m3 bytes, scale bytes [...]), by the definition in 64 bits."""
    x = np.asarray(x, np.float64)
    fin = np.isfinite(x)
    top = np.max(np.where(fin, np.abs(x), 0.0), axis=-1)
    with np.errstate(divide="ignore"):
        k = np.ceil(np.log2(top / 448.0))
    k = np.where(top > 0, k, 0.0)
    for _ in range(2):  # the logarithm may be one off
        k = np.where((top > 0) & (top <= 448.0 * 2.0 ** (k - 1)), k - 1, k)
        k = np.where(top > 448.0 * 2.0 ** k, k + 1, k)
    k = np.where(top > 0, np.clip(k, -126, 119), 0)
    y = np.clip(np.where(fin, x, 0.0) / 2.0 ** k[..., None], -448.0, 448.0)
    mag = np.abs(y)
    e = np.floor(np.log2(np.maximum(mag, 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    units = np.rint(mag / step)  # to nearest even; 16 units are the next binade's 8
    e, units = np.where(units == 16, e + 1, e), np.where(units == 16, 8, units)
    bits = np.where(units < 8, units, (e + 7) * 8 + units - 8)  # below 8 units: subnormal, e = -6
    bits = np.where(fin, bits, 0x7F).astype(np.uint8)
    sign = np.signbit(x)
    return (bits | (sign.astype(np.uint8) << 7)), (k + 127).astype(np.uint8)


def e4m3_values(bits):
    b = bits.astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b & 128, -v, v)


class Paged:
    """A random paged cache of a batch and its new tokens' queries.

    n, lens: new tokens and keys of every sequence.  absent: {(sequence, page column)} without a page.
    Pages no sequence has, and rows behind a sequence's end, hold `junk`.
    """

    def __init__(self, n, lens, H_q, H_kv, D, page, dtype="bf16", cache=None, seed=0, absent=(), extra=3, pad=0,
                 cols=None, junk=0.0):
        rng = np.random.default_rng(seed)
        self.n, self.lens, self.H_q, self.H_kv, self.D, self.page = list(n), list(lens), H_q, H_kv, D, page
        self.dtype, self.cache, self.absent = dtype, cache or dtype, set(absent)
        S, used = len(self.n), [-(-t // page) for t in self.lens]
        self.cols = cols or max(max(used), 1)
        P = sum(used) + extra
        order = rng.permutation(P)
        self.table = np.full((S, self.cols), -1, np.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = order[at:at + u]
            at += u
        self.free = order[at:]
        for s, c in self.absent:
            self.table[s, c] = (-1, 10 ** 6, P)[c % 3]
        self.cu = np.concatenate([[0], np.cumsum(self.n)]).astype(np.int32)
        self.T = int(self.cu[-1]) + pad
        self.q = rng.standard_normal((self.T, H_q, D)).astype(np.float32) * 1.5
        self.q[self.cu[-1]:] = np.nan
        if dtype == "bf16":
            self.q = bf16_round(self.q)
        self.vals, self.raw, self.scales = {}, {}, {}
        live = np.zeros((P, page), bool)
        for s in range(S):
            for t in range(self.lens[s]):
                p = self.table[s, t // page]
                if 0 <= p < P:
                    live[p, t % page] = True
        for name, sigma in (("k", 1.0), ("v", 0.5)):
            x = rng.standard_normal((P, page, H_kv, D)).astype(np.float32) * sigma
            if dtype == "bf16":
                x = bf16_round(x)
            x[~live] = junk
            if self.cache == "e4m3":
                bits, byte = quantise(x)
                if junk != 0:  # nor have the scales of those rows a meaning
                    byte[~live] = 255
                self.raw[name], self.scales[name] = bits, np.ascontiguousarray(byte.transpose(0, 2, 1))
                self.vals[name] = e4m3_values(bits) * 2.0 ** (byte.astype(np.float64) - 127)[..., None]
            else:
                self.vals[name] = x.astype(np.float64)

    # ---- device ----
    def pages(self, name):
        if self.cache == "e4m3":
            return torch.from_numpy(self.raw[name]).view(torch.float8_e4m3fn).cuda()
        return torch.from_numpy(self.vals[name].astype(np.float32)).to(DTYPES[self.dtype]).cuda()

    def scale(self, name):
        return torch.from_numpy(self.scales[name]).cuda() if self.cache == "e4m3" else None

    def i32(self, x):
        return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()

    def rows(self, x):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(DTYPES[self.dtype]).cuda()

    def put(self):
        """Device arguments of paged_attn, kept."""
        self.dev = dict(q=self.rows(self.q), k_pages=self.pages("k"), v_pages=self.pages("v"),
                        block_table=self.i32(self.table), cu_tokens=self.i32(self.cu), seq_lens=self.i32(self.lens))
        self.dev_scales = dict(k_scales=self.scale("k"), v_scales=self.scale("v"))
        return self

    def attn(self, **kw):
        from paper_2607_02963_amd import pdec
        if not hasattr(self, "dev"):
            self.put()
        return pdec.paged_attn(**self.dev, **self.dev_scales, **kw)

    # ---- 64 bits ----
    def keys(self, name, s):
        """[len, H_kv, D] and which of them are present."""
        t = np.arange(self.lens[s])
        p = self.table[s, t // self.page] if len(t) else t
        ok = (p >= 0) & (p < self.vals[name].shape[0])
        return self.vals[name][np.where(ok, p, 0), t % self.page], ok

    def reference(self, causal=True, scale=None):
        """out, lse, and what bounds their errors: size[row, head, d] = sum p |v|, spread[row, head] = the largest
        scale * sum_d |q_d k_d| over the keys seen."""
        scale = self.D ** -0.5 if scale is None else scale
        T = int(self.cu[-1])
        out, size = np.zeros((T, self.H_q, self.D)), np.zeros((T, self.H_q, self.D))
        lse, spread = np.full((T, self.H_q), -np.inf), np.zeros((T, self.H_q))
        G = self.H_q // self.H_kv
        for s, n in enumerate(self.n):
            if n == 0 or self.lens[s] == 0:
                continue
            (k, ok), (v, _) = self.keys("k", s), self.keys("v", s)
            L = self.lens[s]
            seen = ok[None] & ((np.arange(L)[None] <= L - n + np.arange(n)[:, None]) if causal else np.ones((n, L), bool))
            a = int(self.cu[s])
            qs = self.q[a:a + n].astype(np.float64)
            for h in range(self.H_q):
                kk, vv = k[:, h // G], v[:, h // G]
                with np.errstate(invalid="ignore", over="ignore"):
                    z = np.where(seen, qs[:, h] @ kk.T * scale, -np.inf)
                    w = np.where(seen, np.abs(qs[:, h]) @ np.abs(kk).T * scale, 0.0)
                some = seen.any(1)
                m = np.where(some, z.max(1), 0.0)
                p = np.exp(z - m[:, None])
                l = p.sum(1)
                lse[a:a + n, h] = np.where(some, m + np.log(np.where(some, l, 1.0)), -np.inf)
                p = p / np.where(some, l, 1.0)[:, None]
                used = np.where(seen.any(0)[:, None], vv, 0.0)  # a value no query sees counts for none
                if np.isfinite(used).all():
                    out[a:a + n, h], size[a:a + n, h] = p @ used, p @ np.abs(used)
                else:
                    for i in range(n):  # only the keys that the query sees
                        j = np.nonzero(seen[i])[0]
                        with np.errstate(invalid="ignore"):
                            out[a + i, h], size[a + i, h] = p[i, j] @ vv[j], p[i, j] @ np.abs(vv[j])
                spread[a:a + n, h] = w.max(1)
        return out, lse, size, spread


def bounds(dtype, D, out, lse, size, spread):
    """How far out and lse may be off, element by element.

    A score is a float32 sum of D exact or once-rounded products (the scale, log2 e and the subtraction round
    the exponent three times more): off by delta = 2^-24 ((D + 4) spread + 4 (|lse| + spread)) nats at most, so
    every p by that share, and lse by it.  Sums over the keys, exp2 and log2 add 2^-17 (2^7 half steps: partial
    sums are formed in a tree of a few hundred at most).  bf16: each p is rounded once (2^-8 of it), and out.
    """
    fin = np.where(np.isfinite(lse), lse, 0.0)
    delta = 2.0 ** -24 * ((D + 4) * spread + 4 * (np.abs(fin) + spread)) + 2.0 ** -17
    rel = 2 * delta[..., None] + (HALF_STEP["bf16"] if dtype == "bf16" else 0.0)
    tol_out = size * rel * (1 + 2.0 ** -6) + HALF_STEP[dtype] * np.abs(out) * (1 + 2.0 ** -6) + 1e-37
    return tol_out, delta + 2.0 ** -23 * np.abs(fin)


def compare(dtype, got_out, got_lse, ref, what=""):
    out, lse, size, spread = ref
    T, D = out.shape[0], out.shape[-1]
    o = got_out[:T].float().cpu().numpy().astype(np.float64)
    dead = np.isneginf(lse)
    assert np.all(o[dead] == 0), f"{what}: rows that see nothing are not 0"
    tol_o, tol_l = bounds(dtype, D, out, lse, size, spread)
    fin = np.isfinite(out)
    assert np.array_equal(np.isfinite(o), fin), f"{what}: finite where the definition is not, or the reverse"
    err = np.abs(o - out)
    bad = fin & (err > tol_o)
    assert not bad.any(), f"{what}: out off by {np.max(np.where(bad, err, 0)):.3e} at {np.argwhere(bad)[0]}, " \
                          f"{bad.sum()} of {bad.size}, allowed there {tol_o[tuple(np.argwhere(bad)[0])]:.3e}"
    if got_lse is not None:
        l = got_lse[:T].cpu().numpy().astype(np.float64)
        assert np.all(np.isneginf(l[dead])), f"{what}: lse of rows that see nothing"
        fin = np.isfinite(lse)
        with np.errstate(invalid="ignore"):
            err = np.abs(l - lse)
        bad = fin & ~(err <= tol_l)
        assert not bad.any(), f"{what}: lse off by {np.max(np.where(bad, err, 0)):.3e} at {np.argwhere(bad)[0]}"
