"""Weights of up to 16 query rows: a wave keeps the logits of a few tiles in LDS, 4096 / (64 rows) of them, and hands them from lane to lane on their
way to memory.  Token counts around full and partly full batches of tiles, rows that divide them and rows that do not, one chunk and many."""
import math

import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("W,G", [(1, 1), (3, 1), (1, 7), (1, 8), (3, 5), (4, 4)])
@pytest.mark.parametrize("B", [2, 300])
def test_batches_of_kept_tiles(fmt, W, G, B):
    # two sequences' pages shared by all: with 300 one block has all tokens, whose waves take a quarter each
    import paper_2512_14946_amd as kvp
    batch = 4096 // (64 * W * G)                             # tiles that a wave keeps
    n = min(4 * 64 * (2 * batch + 1) + 65, 9000)
    print("[case] kept", fmt, W, G, B, n, flush=True)
    few = inputs.filled_cache(kvp, [n, min(4 * 64 * batch, 8000) - 63], -(-n // 64), 1, 64, fmt, W + G, DEV)
    rows = torch.arange(B, device=DEV) % 2
    c = kvp.KVCache(few.k_codes, few.v_codes, few.k_scales, few.v_scales, few.block_table[rows].contiguous(), few.lens[rows].contiguous(), fmt)
    q = inputs.rows((2, W, G, 128), 5, False).to(DEV)
    acc_in = torch.rand(2, 1, n, generator=inputs.gen(6)).to(DEV)
    acc = torch.zeros(B, 1, n, device=DEV)
    ws = torch.empty(kvp.kvp_cache_attend_workspace_bytes(B, 1, G, W, n, True), dtype=torch.uint8, device=DEV)
    want, drawn, mag, vmax, size = ref.attend(ref.Cache(few, fmt), q.float().cpu(), None, True, 1 / math.sqrt(128))
    for poison in (0xFF, 0):
        ws.fill_(poison)
        got = kvp.kvp_cache_attend(q[rows].contiguous(), c, max_len=n, acc_in=acc_in[rows].contiguous(), acc_out=acc, ws=ws)
        lens = few.lens.tolist()
        tol = ref.out_tolerance(want, mag, vmax, size, lens)
        assert np.all(np.abs(got[:2].double().cpu().numpy() - want) <= tol)
        for b, m in enumerate(lens):
            a0 = acc_in[b:b + 1, :, :m].double().cpu().numpy()
            e = np.abs(acc[b:b + 1, :, :m].double().cpu().numpy() - a0 - drawn[b:b + 1, :, :m])
            assert np.all(e <= ref.drawn_tolerance(drawn[b:b + 1, :, :m], a0, size[b:b + 1]))
            assert torch.equal(acc[b::2], acc[b:b + 1].expand_as(acc[b::2]))
            assert bool((acc[b, :, m:] == 0).all())
