"""Eviction where scales are subnormal: a page's own scale, amax / qmax, is then a whole number of units of 2^-149, off by up to a third, and
quotients pass the largest code.  They become the largest code."""
import math

import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
UNIT = 2.0 ** -149


@pytest.mark.parametrize("fmt,units,most", [("e4m3", 146, 4.5), ("e4m3", 3, 320.0), ("int8", 3, 63), ("int8", 1, 127), ("int8", 700, 127), ("int8", 1, 40),
                                            ("e4m3", 1 << 40, 448.0)])
@pytest.mark.parametrize("bs", [16, 64])
def test_codes_on_subnormal_scales(fmt, units, most, bs):
    import paper_2512_14946_amd as kvp
    lens, H, budget = [100, 37], 2, 50
    c = inputs.filled_cache(kvp, lens, -(-100 // bs), H, bs, fmt, 7, "cpu")
    for codes in (c.k_codes, c.v_codes):                     # codes no larger than `most`, some of them it
        x = torch.from_numpy(ref.code_values(codes, fmt)).nan_to_num(0).clamp(-most, most)
        codes.copy_(x.to(torch.int8).view(torch.uint8) if fmt == "int8" else x.float().to(torch.float8_e4m3fn).view(torch.uint8))
    for s in (c.k_scales, c.v_scales):
        s.fill_(units * UNIT)
    c = kvp.KVCache(*[t.to(DEV) for t in (c.k_codes, c.v_codes, c.k_scales, c.v_scales, c.block_table, c.lens)], fmt)
    acc = torch.rand(2, H, c.block_table.shape[1] * bs, generator=inputs.gen(8)).to(DEV)
    d = inputs.empty_cache(kvp, [0, 0], -(-budget // bs), H, bs, fmt, 9, DEV)
    kvp.kvp_cache_evict(c, acc, budget, d, sink=1, recent=5, lens_out=d.lens)
    _, new, moved = ref.evict(ref.Cache(c, fmt), acc.cpu().numpy(), budget, 1, 5)
    got, beyond = ref.Cache(d, fmt), 0
    for (b, h), planes in moved.items():
        for x, codes, scales in zip(planes, (got.k, got.v), (got.ks, got.vs)):
            for i in range(0, int(new[b]), bs):
                page, part = got.table[b, i // bs], x[i:min(i + bs, int(new[b]))]
                s = np.float32(np.abs(part).max()) / ref.QMAX[fmt]
                assert scales[page, h].view(np.uint32) == s.view(np.uint32)
                if s == 0:
                    assert np.all(codes[page, h, :len(part)] == 0)
                    continue
                y = np.divide(part, s, dtype=np.float32)
                beyond += int((np.abs(y) > ref.QMAX[fmt]).sum())
                want = ref.round_code(np.clip(y, -ref.QMAX[fmt], ref.QMAX[fmt]), fmt)
                assert np.array_equal(codes[page, h, :len(part)], want)
    assert beyond > 0 if units in (146, 3, 1) and (fmt, units, most) not in (("int8", 1, 127), ("int8", 1, 40)) else True
    q = inputs.rows((2, 1, 4, 128), 1, False).to(DEV)
    out = kvp.kvp_cache_attend(q, d, scale=1.0 / math.sqrt(128))
    assert bool(out.isfinite().all())
