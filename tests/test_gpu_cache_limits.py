"""Calls near what the sizes allow, run whole: batches of more than 2^16 cells of 256 query rows."""
import math

import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_more_than_65536_tiles_of_256_rows():
    import paper_2512_14946_amd as kvp
    B, H, W, T = 8194, 8, 130, 128
    few = inputs.filled_cache(kvp, [T, 77], 8, H, 16, "int8", 3, DEV)
    rows = torch.arange(B, device=DEV) % 2
    c = kvp.KVCache(few.k_codes, few.v_codes, few.k_scales, few.v_scales, few.block_table[rows].contiguous(), few.lens[rows].contiguous(), "int8")
    q = inputs.rows((2, W, H, 128), 4, False).to(DEV)
    qs = q[rows].contiguous()
    want, drawn, mag, vmax, size = ref.attend(ref.Cache(few, "int8"), q.float().cpu(), None, True, 1 / math.sqrt(128))
    tol = ref.out_tolerance(want, mag, vmax, size, [T, 77])
    acc = torch.zeros(B, H, T, device=DEV)
    for weights in (None, acc):
        got = kvp.kvp_cache_attend(qs, c, acc_out=weights)
        assert np.all(np.abs(got[:2].double().cpu().numpy() - want) <= tol)
        assert torch.equal(got.view(B // 2, 2, W, H, 128), got[None, :2].expand(B // 2, 2, W, H, 128))
    e = np.abs(acc[:2].double().cpu().numpy() - drawn)
    assert np.all(e <= ref.drawn_tolerance(drawn, 0.0, size))
    assert torch.equal(acc.view(B // 2, 2, H, T), acc[None, :2].expand(B // 2, 2, H, T))
