"""Seeded caches, queries and weights for the tests of the 8-bit paged cache.  Everything that no call may look at holds poison."""
from __future__ import annotations

import torch

D = 128


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rows(shape, seed, outliers=True):
    """bf16 [..][H][128] normal values, four channels of every head 8 times as large"""
    g = gen(seed)
    x = torch.randn(shape, generator=g)
    if outliers:
        mult = torch.ones(shape[-2], D)
        mult.scatter_(-1, torch.rand(shape[-2], D, generator=g).argsort(-1)[:, :4], 8.0)
        x = x * mult
    return x.to(torch.bfloat16)


def empty_cache(kvp, lens, max_blocks, H, bs, fmt, seed, device, spare=3):
    """A cache whose pages hold 0xFF bytes (NaN as e4m3) and NaN scales, pages dealt in random order, table rows wider than needed."""
    B = len(lens)
    nb = B * max_blocks + spare
    table = torch.full((B, max_blocks + 2), -7, dtype=torch.int32)
    table[:, :max_blocks] = torch.randperm(nb, generator=gen(seed))[:B * max_blocks].view(B, max_blocks).to(torch.int32)
    c = kvp.alloc_cache(nb, H, D, bs, table.to(device)[:, :max_blocks], torch.tensor(lens, dtype=torch.int32, device=device), fmt)
    for t in (c.k_codes, c.v_codes):
        t.fill_(255)
    for t in (c.k_scales, c.v_scales):
        t.fill_(float("nan"))
    return c


def filled_cache(kvp, lens, max_blocks, H, bs, fmt, seed, device, spread=0.0):
    """... and the tokens of every sequence written by the reference's own page coding; `spread` > 0 gives pages of very different
    scales."""
    import numpy as np
    import cache_reference as ref
    c = empty_cache(kvp, lens, max_blocks, H, bs, fmt, seed, "cpu")
    for b, n in enumerate(lens):
        if n <= 0:
            continue
        k, v = rows((n, H, D), seed * 31 + b).float(), rows((n, H, D), seed * 37 + b + 5, False).float()
        if spread:
            f = torch.exp(spread * torch.randn(-(-n // bs), H, 1, generator=gen(seed + b))).repeat_interleave(bs, 0)[:n]
            k, v = (k * f).to(torch.bfloat16).float(), (v * f.flip(0)).to(torch.bfloat16).float()
        for x, codes, scales, turn in ((k, c.k_codes, c.k_scales, False), (v, c.v_codes, c.v_scales, True)):
            for h in range(H):
                y, s = ref.pages_of(x[:, h].numpy(), fmt, bs)
                y = torch.from_numpy(np.ascontiguousarray(y))
                y = (y.to(torch.int8).view(torch.uint8) if fmt == "int8" else y.float().to(torch.float8_e4m3fn).view(torch.uint8))
                for i in range(len(s)):
                    p = int(c.block_table[b, i])
                    part = y[i * bs:(i + 1) * bs]
                    if turn:
                        codes[p, h, :, :len(part)] = part.T
                    else:
                        codes[p, h, :len(part)] = part
                    scales[p, h] = float(s[i])
    wide = torch.full((len(lens), max_blocks + 2), -7, dtype=torch.int32)
    wide[:, :max_blocks] = c.block_table
    return kvp.KVCache(c.k_codes.to(device), c.v_codes.to(device), c.k_scales.to(device), c.v_scales.to(device),
                       wide.to(device)[:, :max_blocks], c.lens.to(device), fmt)


def copy_of(kvp, c):
    return kvp.KVCache(c.k_codes.clone(), c.v_codes.clone(), c.k_scales.clone(), c.v_scales.clone(), c.block_table, c.lens, c.fmt)
