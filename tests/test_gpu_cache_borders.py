"""The 8-bit paged cache where rules change and sizes pass 32 bits: row counts on both sides of the tile rules, chunks on both sides of one,
pools and batches beyond 4 GiB, results that the binding allocates on another stream, weights that are no numbers."""
import math

import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref
from test_gpu_cache_attend import _check
from test_gpu_cache_evict import _acc, _run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("W,G", [(15, 1), (16, 1), (17, 1), (4, 8), (33, 1), (11, 3), (32, 8), (257, 1), (43, 12)])
def test_row_counts_around_the_tile_rules(fmt, W, G):
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [W + 70, W - 1, 1, 0], 10, 1, 64, fmt, W, DEV)
    _check(kvp, c, W, G, G)
    _check(kvp, c, W, G, G + 1, causal=False, q_lens=[W, 1, W - 1, 2])


@pytest.mark.parametrize("W,G", [(1, 4), (5, 4), (40, 2)])
@pytest.mark.parametrize("n", [255, 256, 257, 511, 513])
def test_one_chunk_and_two(W, G, n):
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [n, n - 64], 9, 1, 64, "int8", n, DEV)
    _check(kvp, c, W, G, n)
    _check(kvp, c, W, G, n, max_len=n)


def test_pools_and_batches_beyond_32_bits():
    import paper_2512_14946_amd as kvp
    H, bs, B, W = 8, 128, 2, 3
    small = inputs.filled_cache(kvp, [300, 129], 3, H, bs, "int8", 5, DEV)
    far = 40000                                              # pages of 128 KiB
    big = kvp.alloc_cache(far + small.k_codes.shape[0], H, 128, bs, (small.block_table + far).contiguous(), small.lens, "int8")
    for a, b in ((big.k_codes, small.k_codes), (big.v_codes, small.v_codes), (big.k_scales, small.k_scales), (big.v_scales, small.v_scales)):
        a[far:].copy_(b)
    room = torch.empty((1 << 31) + 2 * W * H * 4 * 128, dtype=torch.bfloat16, device=DEV)
    view = lambda heads, at: room[at:].as_strided((B, W, heads, 128), (1 << 31, heads * 128, 128, 1))
    q = inputs.rows((B, W, H * 4, 128), 6, False).to(DEV)
    far_q = view(H * 4, 0)
    far_q.copy_(q)
    acc = [torch.zeros(B, H, 3 * bs, device=DEV) for _ in range(2)]
    want = kvp.kvp_cache_attend(q, small, acc_out=acc[0])
    assert torch.equal(kvp.kvp_cache_attend(far_q, big, acc_out=acc[1]), want) and torch.equal(*acc)
    far_out = view(H * 4, W * H * 4 * 128)
    kvp.kvp_cache_attend(q, big, far_out)
    assert torch.equal(far_out, want)
    # appending and restoring
    k, v = (inputs.rows((B, W, H, 128), 7 + i).to(DEV) for i in range(2))
    far_k = view(H, 0)
    far_k.copy_(k)
    for c, key in ((small, k), (big, far_k)):
        kvp.kvp_cache_append(c, key, v)
    for a, b in ((big.k_codes, small.k_codes), (big.v_codes, small.v_codes)):
        assert torch.equal(a[far:], b)
    rows = [[torch.zeros(B, 300, H, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)] for _ in range(2)]
    for c, r in zip((small, big), rows):
        kvp.kvp_cache_read(c, *r)
    assert all(torch.equal(a, b) for a, b in zip(*rows)) and bool((rows[0][0][0, 299] != 0).any())
    # rotary positions there
    pos, freq = torch.arange(W, dtype=torch.int32, device=DEV), kvp.kvp_rotary_frequencies(128)[0].to(DEV)
    assert torch.equal(kvp.kvp_rotary(far_k, pos, freq), kvp.kvp_rotary(k, pos, freq))
    # and eviction from the far pool into its beginning
    near = [kvp.KVCache(p.k_codes, p.v_codes, p.k_scales, p.v_scales, (torch.arange(B * 2, dtype=torch.int32, device=DEV) + o).view(B, 2),
                        torch.zeros(B, dtype=torch.int32, device=DEV), "int8") for p, o in ((big, 0), (kvp.alloc_cache(4, H, 128, bs, small.block_table,
                                                                                                             small.lens, "int8"), 0))]
    keep = [torch.empty(B, H, 140, dtype=torch.int32, device=DEV) for _ in range(2)]
    for c, d, idx in ((big, near[0], keep[0]), (small, near[1], keep[1])):
        kvp.kvp_cache_evict(c, acc[0], 140, d, sink=2, recent=9, keep_idx=idx, lens_out=d.lens)
    assert torch.equal(*keep) and near[0].lens.tolist() == [140, 129]
    for b, m in enumerate(near[0].lens.tolist()):
        for i in range(2):
            part = min(m - i * bs, bs)
            x, y = near[0].block_table[b, i].long(), near[1].block_table[b, i].long()
            assert torch.equal(near[0].k_codes[x, :, :part], near[1].k_codes[y, :, :part])
            assert torch.equal(near[0].v_codes[x, :, :, :part], near[1].v_codes[y, :, :, :part])
            assert torch.equal(near[0].v_scales[x], near[1].v_scales[y])


def test_results_allocated_on_another_stream():
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [300, 40], 5, 2, 64, "e4m3", 3, DEV)
    q = inputs.rows((2, 6, 8, 128), 4, False).to(DEV)
    ql = torch.tensor([2, 6], dtype=torch.int32, device=DEV)
    want = kvp.kvp_cache_attend(q, c, q_lens=ql)
    assert bool((want[0, 2:] == 0).all()) and bool((want[0, :2] != 0).any())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        torch.cuda._sleep(2_000_000)                         # the current stream is behind: nothing of the call may wait there
        got = kvp.kvp_cache_attend(q, c, q_lens=ql, stream=stream)
        s.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_weights_that_are_not_finite():
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [200, 130], 13, 2, 16, "int8", 2, DEV)
    acc = _acc(2, 2, 208, 1)
    acc[0, 0, 10:80] = math.inf                              # below the protected last tokens, above every finite weight
    acc[1, 1, 30:60] = -math.inf
    acc[0, 1, 150:] = 0.0
    d, idx = _run(kvp, c, acc.clamp(max=3.0e38), 60, 3, 20)
    e = inputs.empty_cache(kvp, [0, 0], 4, 2, 16, "int8", 3, DEV)
    odd = torch.where(acc == math.inf, torch.tensor(math.nan, device=DEV), acc)
    for weights in (acc, odd):
        again = torch.empty_like(idx)
        kvp.kvp_cache_evict(c, weights, 60, e, sink=3, recent=20, keep_idx=again)
        assert torch.equal(again, idx)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("B,W,G,n", [(24, 5, 4, 16500), (12, 8, 8, 16500), (40, 3, 11, 7000), (3, 16, 8, 1500)])
def test_tiles_of_32_rows(fmt, B, W, G, n):
    # work enough for tiles of 32 rows, most sequences short; two whole ones against the definition, through the cache of the batch
    import paper_2512_14946_amd as kvp
    few = inputs.filled_cache(kvp, [n, 77], -(-n // 64), 1, 64, fmt, W, DEV)
    rows = torch.arange(B, device=DEV) % 2
    c = kvp.KVCache(few.k_codes, few.v_codes, few.k_scales, few.v_scales, few.block_table[rows].contiguous(), few.lens[rows].contiguous(), fmt)
    q = inputs.rows((2, W, G, 128), 3, False).to(DEV)
    acc = torch.zeros(B, 1, n, device=DEV)
    many = kvp.kvp_cache_attend(q[rows].contiguous(), c, max_len=n, acc_out=acc)
    model = ref.Cache(few, fmt)
    want, drawn, mag, vmax, size = ref.attend(model, q.float().cpu(), None, True, 1 / math.sqrt(128))
    tol = ref.out_tolerance(want, mag, vmax, size, model.lens)
    err = np.abs(many[:2].double().cpu().numpy() - want)
    assert np.all(err <= tol), (err / tol).max()
    assert torch.equal(many[2:4], many[:2]) if B > 3 else torch.equal(many[2], many[0])
    a = acc.double().cpu().numpy()
    for b in range(2):
        m = int(model.lens[b])
        t = ref.drawn_tolerance(drawn[b:b + 1, :, :m], np.zeros((1, 1, m)), size[b:b + 1])[0]
        e = np.abs(a[b, :, :m] - drawn[b, :, :m])
        assert np.all(e <= t), (e / t).max()
        assert np.all(a[b, :, m:] == 0.0) and np.array_equal(a[b], a[b + 2 if b + 2 < B else b])
