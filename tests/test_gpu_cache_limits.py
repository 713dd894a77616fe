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


def test_rotary_of_more_than_2_to_the_24_tokens():
    # 142 GB turned in place: blocks take two tokens of 33 heads each, as one apiece would be more than a grid holds
    import paper_2512_14946_amd as kvp
    T, H = (1 << 24) + 5, 33
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < T * H * 256 + (8 << 30):
        pytest.skip("not enough free memory on this card")
    x = torch.zeros(1, T, H, 128, dtype=torch.bfloat16, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    freq = kvp.kvp_rotary_frequencies(128)[0].to(DEV)
    spans = [(0, 9), (T // 2 - 4, T // 2 + 3), ((1 << 24) - 3, T)]
    want = []
    for i, (a, b) in enumerate(spans):
        part = inputs.rows((1, b - a, H, 128), 20 + i).to(DEV)
        x[:, a:b] = part
        want.append(kvp.kvp_rotary(part, pos[a:b], freq))
    kvp.kvp_rotary(x, pos, freq, out=x)
    for (a, b), y in zip(spans, want):
        assert torch.equal(x[:, a:b], y)
    assert not bool(x[:, 9:40].any())
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("H", [33, 64, 200])
def test_rotary_of_many_heads(H):
    # 200 heads: more rows than a block has in flight
    import paper_2512_14946_amd as kvp
    x, freq = inputs.rows((2, 5, H, 128), H).to(DEV), kvp.kvp_rotary_frequencies(128)[0]
    pos = torch.tensor([3, 0, -7, 40000, 12], dtype=torch.int32)
    want = ref.rotary(x.double().cpu().numpy(), np.broadcast_to(pos.numpy()[None, :, None], (2, 5, H)), freq.numpy(), "half", False, 1.0)
    got = kvp.kvp_rotary(x, pos.to(DEV), freq.to(DEV)).double().cpu().numpy()
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * np.abs(x.double().cpu().numpy()).max(axis=-1, keepdims=True) + 1e-38   # as in test_gpu_rotary.py
    assert np.all(np.abs(got - want) <= tol)
