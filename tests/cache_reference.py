"""The 8-bit paged cache, rotary positions and attention over the cache from their definitions, on the CPU: plain loops over
sequences and heads, binary32 only where the definition names it, 64 bits elsewhere.  Shares nothing with the library."""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128
QMAX = {"int8": np.float32(127), "e4m3": np.float32(448)}


def code_values(codes: torch.Tensor, fmt: str) -> np.ndarray:
    """bytes -> the numbers that they stand for, float64"""
    t = codes.contiguous().view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn)
    return t.to(torch.float32).numpy().astype(np.float64)


def round_code(y: np.ndarray, fmt: str) -> np.ndarray:
    """float32 quotients -> the nearest code value, ties to even"""
    if fmt == "int8":
        return np.rint(y).astype(np.float64)
    _, e = np.frexp(np.abs(y).astype(np.float64))
    step = np.ldexp(1.0, np.maximum(e - 4, -9))          # 4 significant bits, subnormals in steps of 2^-9
    return np.rint(y.astype(np.float64) / step) * step


def code_page(x: np.ndarray, scale: np.float32, fmt: str) -> np.ndarray:
    if scale == 0:
        return np.zeros(x.shape)
    return round_code(np.divide(x.astype(np.float32), scale, dtype=np.float32), fmt)


class Cache:
    """Code values k [pages][H][bs][D], v [pages][H][bs][D] (both token-major here) and float32 scales."""

    def __init__(self, c, fmt):
        self.fmt, self.bs = fmt, c.k_codes.shape[2]
        self.k = code_values(c.k_codes.cpu(), fmt)
        self.v = code_values(c.v_codes.cpu().transpose(-1, -2), fmt)
        self.ks, self.vs = c.k_scales.cpu().numpy().copy(), c.v_scales.cpu().numpy().copy()
        self.table, self.lens = c.block_table.cpu().numpy(), c.lens.cpu().numpy()
        self.B, self.H = self.table.shape[0], self.k.shape[1]

    def append(self, k, v, counts):
        cap = self.table.shape[1] * self.bs
        for x, codes, scales in ((k, self.k, self.ks), (v, self.v, self.vs)):
            x = x.float().cpu().numpy()
            for b in range(self.B):
                n, end = int(self.lens[b]), min(int(self.lens[b]) + int(counts[b]), cap)
                for page in range(n // self.bs, -(-end // self.bs)):
                    t0 = page * self.bs
                    s0, s1 = max(n - t0, 0), min(end - t0, self.bs)
                    if s0 >= s1:
                        continue
                    p = self.table[b, page]
                    for h in range(self.H):
                        new = x[b, t0 + s0 - n:t0 + s1 - n, h]
                        fresh = np.float32(np.abs(new).max()) / QMAX[self.fmt]
                        old = scales[p, h]
                        scale = max(old, fresh) if s0 else fresh
                        if s0 and scale != old:
                            codes[p, h, :s0] = code_page((codes[p, h, :s0].astype(np.float32) * old), scale, self.fmt)
                        codes[p, h, s0:s1] = code_page(new, scale, self.fmt)
                        scales[p, h] = scale

    def values(self, b, h, n, exact=True):
        """keys and values [n][D] of a sequence's head: float64 products, or the float32 products that eviction and reading use"""
        out = []
        for codes, scales in ((self.k, self.ks), (self.v, self.vs)):
            pages = self.table[b, :-(-n // self.bs)] if n else self.table[b, :0]
            x, s = codes[pages, h], scales[pages, h][:, None, None]
            x = x * s.astype(np.float64) if exact else x.astype(np.float32) * s
            out.append(x.reshape(-1, D)[:n])
        return out


def attend(cache, q, q_lens, causal, scale, max_len=None):
    """out [B][W][Hq][D], drawn [B][H][T], and what a tolerance needs: sum p |v| like out, and the largest sum |q k| scale per sequence."""
    B, W, Hq, _ = q.shape
    G, T = Hq // cache.H, int(max(cache.lens.max(), 1))
    q = q.double().cpu().numpy()
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    drawn, vmax, size = np.zeros((B, cache.H, T)), np.zeros(B), np.zeros(B)
    for b in range(B):
        n = int(cache.lens[b]) if max_len is None else min(int(cache.lens[b]), max_len)
        m = W if q_lens is None else min(max(int(q_lens[b]), 0), W)
        if n <= 0 or m == 0:
            continue
        for h in range(cache.H):
            k, v = cache.values(b, h, n)
            vmax[b] = max(vmax[b], np.abs(v).max())
            for w in range(m):
                see = n - m + w + 1 if causal else n
                if see <= 0:
                    continue
                z = q[b, w, h * G:(h + 1) * G] @ k[:see].T * scale
                size[b] = max(size[b], (np.abs(q[b, w, h * G:(h + 1) * G]) @ np.abs(k[:see]).T).max() * abs(scale))
                p = np.exp(z - z.max(axis=1, keepdims=True))
                p /= p.sum(axis=1, keepdims=True)
                out[b, w, h * G:(h + 1) * G] = p @ v[:see]
                mag[b, w, h * G:(h + 1) * G] = p @ np.abs(v[:see])
                drawn[b, h, :see] += p.sum(axis=0)
    return out, drawn, mag, vmax, size


def out_tolerance(out, mag, vmax, size, lens):
    """Half a bf16 step of the result; half a half-precision step (2^-11) of every probability; 2^-25 of the largest value for those that are
    subnormal halves, per token; the probabilities' own error: logits of 128 products and the scaling, each rounded in fp32 (at
    most 140 roundings of 2^-24 on a sum of magnitude `size`, twice, as the row's sum has it too), and 2^-20 for exponential and sums."""
    delta = (2 * 140 * 2.0 ** -24 * size + 2.0 ** -20)[:, None, None, None]
    return 2.0 ** -8 * np.abs(out) + (2.0 ** -11 + delta) * mag * 1.01 + (np.asarray(lens) * 2.0 ** -25 * vmax)[:, None, None, None] + 1e-30


def drawn_tolerance(drawn, acc_in, size):
    delta = (2 * 140 * 2.0 ** -24 * size + 2.0 ** -18)[:, None, None]   # sums over up to 2^5 rows beyond what a row has
    return delta * drawn + 2.0 ** -23 * np.abs(acc_in) + 1e-30


def evict(cache, acc, budget, sink, recent, max_len=None):
    """keep [B][H][budget], new lengths, and per (b, h) the float32 keys and values that move."""
    keep = -np.ones((cache.B, cache.H, budget), dtype=np.int64)
    lens, moved = [], {}
    for b in range(cache.B):
        n = int(cache.lens[b]) if max_len is None else min(int(cache.lens[b]), max_len)
        m = min(n, budget)
        lens.append(m)
        for h in range(cache.H):
            a = acc[b, h, :n].astype(np.float64).copy()
            a[:sink] = math.inf
            if recent:
                a[max(0, n - recent):] = math.inf
            kept = np.sort(np.argsort(-a, kind="stable")[:m])
            keep[b, h, :m] = kept
            moved[b, h] = [x[kept] for x in cache.values(b, h, n, exact=False)]
    return keep, np.array(lens), moved


def pages_of(x, fmt, bs):
    """float32 rows [m][D] coded page by page on each page's own scale: (code values [m][D], scales)"""
    codes, scales = [], []
    for i in range(0, len(x), bs):
        s = np.float32(np.abs(x[i:i + bs]).max()) / QMAX[fmt]
        codes.append(code_page(x[i:i + bs], s, fmt))
        scales.append(s)
    return (np.concatenate(codes) if codes else np.zeros((0, D))), np.array(scales, dtype=np.float32)


def rotary(x, pos, freq, layout, inverse, mscale):
    """x [L][T][H][D] float64, pos [L][T][H]; every pair as a complex number"""
    rd = 2 * len(freq)
    a, b = (np.arange(rd // 2), np.arange(rd // 2, rd)) if layout == "half" else (np.arange(0, rd, 2), np.arange(1, rd, 2))
    t = pos[..., None].astype(np.float64) * np.asarray(freq)
    z = (x[..., a] + 1j * x[..., b]) * mscale * np.exp((-1j if inverse else 1j) * t)
    y = np.array(x, dtype=np.float64)
    y[..., a], y[..., b] = z.real, z.imag
    return y
