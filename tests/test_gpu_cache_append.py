"""kvp_cache_append and kvp_cache_read against the definition: codes and scales exactly, page by page, with everything else untouched."""
import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _same_codes(cache, model):
    """values of all codes (a zero's sign is free; unused bytes are poison on both sides) and bits of all scales"""
    got = ref.Cache(cache, model.fmt)
    for what in ("ks", "vs", "k", "v"):
        a, b = getattr(got, what), getattr(model, what)
        differ = (a.view(np.uint32) != b.view(np.uint32)) if what in ("ks", "vs") else ((a != b) & ~(np.isnan(a) & np.isnan(b)))
        at = np.argwhere(differ)
        same = len(at) == 0
        assert same, (what, len(at), at[:4].tolist(), a[differ][:4], b[differ][:4])


CASES = [   # lens before, counts, W, max_blocks
    ([0], [1], 1, 2), ([0, 5, 15, 16, 17, 31], [1, 1, 1, 1, 1, 0], 1, 4), ([3, 0, 64, 100], [70, 7, 0, 33], 70, 12),
    ([200, 130, 250], [60, 130, 3], 130, 17), ([1, 127, 128, 129], None, 256, 30)]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_codes_and_scales(fmt, bs, case):
    import paper_2512_14946_amd as kvp
    lens, counts, W, blocks = CASES[case]
    H, B = (3, len(lens)) if case else (1, 1)
    blocks = max(1, blocks * 16 // bs)                     # some sequences reach the end of their pages: what is behind is dropped
    lens = [min(n, blocks * bs) for n in lens]
    print("[case] append", fmt, bs, case, flush=True)
    c = inputs.filled_cache(kvp, lens, blocks, H, bs, fmt, 11 + case, DEV)
    model = ref.Cache(c, fmt)
    k, v = inputs.rows((B, W, H, 128), 1, True), inputs.rows((B, W, H, 128), 2, False)
    k[-1] *= 4.0                                           # pages whose scale grows
    v[0] *= 0.25                                           # and one that keeps it
    if counts is not None:
        for b, n in enumerate(counts):                     # padding rows are not read
            k[b, n:], v[b, n:] = float("nan"), float("inf")
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV)
    kvp.kvp_cache_append(c, k.to(DEV), v.to(DEV), cnt)
    model.append(k, v, [W] * B if counts is None else counts)
    _same_codes(c, model)
    assert c.lens.tolist() == lens


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_token_by_token_and_recoding(fmt):
    """One token at a time, magnitudes growing and falling: every growth recodes the page's older tokens."""
    import paper_2512_14946_amd as kvp
    B, H, bs, n = 2, 2, 16, 37
    c = inputs.empty_cache(kvp, [0, 3], 4, H, bs, fmt, 1, DEV)
    c.k_codes.zero_(), c.v_codes.zero_(), c.k_scales.fill_(0.5), c.v_scales.fill_(2.0)
    model = ref.Cache(c, fmt)
    for t in range(n):
        k = inputs.rows((B, 1, H, 128), 100 + t) * (1.5 ** (t % 7))
        v = inputs.rows((B, 1, H, 128), 200 + t) * (0.7 ** (t % 5))
        kvp.kvp_cache_append(c, k.to(DEV), v.to(DEV))
        model.append(k, v, [1, 1])
        c.lens.add_(1)
        model.lens = model.lens + 1
    _same_codes(c, model)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_extreme_magnitudes_and_zero_pages(fmt):
    import paper_2512_14946_amd as kvp
    B, H, bs = 6, 1, 16
    c = inputs.empty_cache(kvp, [0] * B, 2, H, bs, fmt, 2, DEV)
    model = ref.Cache(c, fmt)
    x = inputs.rows((B, 32, H, 128), 3)
    for b, s in enumerate((0.0, 1e-38, 1e-30, 1e30, 3e36, 1.0)):
        x[b] *= s
    x[5, :16] = 0.0
    x[5, 16:, :, 1:] = 0.0                                 # a page with one channel, ties of every kind
    x[1, 0, 0, 0] = 2.0 ** -133
    kvp.kvp_cache_append(c, x.to(DEV), x.to(DEV))
    model.append(x, x, [32] * B)
    _same_codes(c, model)
    out = torch.zeros(B, 32, H, 128, dtype=torch.bfloat16, device=DEV)
    c.lens.fill_(32)
    kvp.kvp_cache_read(c, out)
    assert bool(out.isfinite().all()) and bool((out[0] == 0).all())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_every_quotient_is_the_divisions(fmt):
    """Half a million values per scale: the codes are those of the IEEE quotient, ties included."""
    import paper_2512_14946_amd as kvp
    B, T = 4, 4096
    c = inputs.empty_cache(kvp, [0] * B, T // 16, 1, 16, fmt, 3, DEV)
    model = ref.Cache(c, fmt)
    x = torch.randint(-32768, 32767, (B, T, 1, 128), generator=inputs.gen(4)).to(torch.int16).view(torch.bfloat16)
    x = torch.where(x.isfinite(), x, torch.zeros((), dtype=torch.bfloat16))
    small = x.float().abs() < 2.0 ** 100
    x[1:] = torch.where(small[1:], x[1:], torch.ones((), dtype=torch.bfloat16))
    x[2] = torch.randint(-255, 256, x[2].shape, generator=inputs.gen(5)).to(torch.bfloat16)             # many exact ties
    x[3] = torch.randint(-127, 128, x[3].shape, generator=inputs.gen(6)).to(torch.bfloat16) * 0.5
    kvp.kvp_cache_append(c, x.to(DEV), x.to(DEV))
    model.append(x, x, [T] * B)
    _same_codes(c, model)


@pytest.mark.parametrize("bs", [16, 128])
def test_strided_rows_and_a_table_wider_than_its_sequences(bs):
    import paper_2512_14946_amd as kvp
    B, W, H = 3, 50, 4
    c = inputs.filled_cache(kvp, [10, 0, 77], 160 // bs + 1, H, bs, "int8", 5, DEV)
    model = ref.Cache(c, "int8")
    buf = inputs.rows((W, B, 2 * H, 128), 6).to(DEV)       # token-major batch, keys and values of a fused projection
    k, v = buf.transpose(0, 1)[:, :, :H], buf.transpose(0, 1)[:, :, H:]
    counts = torch.tensor([50, 49, 1], dtype=torch.int32, device=DEV)
    kvp.kvp_cache_append(c, k, v, counts)
    model.append(k, v, [50, 49, 1])
    _same_codes(c, model)


@pytest.mark.parametrize("bs", [16, 64])
def test_lengths_counts_and_pages_out_of_range_are_clamped(bs):
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [5, 5, 5, 5], 2, 2, bs, "int8", 7, DEV)
    model = ref.Cache(c, "int8")
    c.lens.copy_(torch.tensor([-4, 1 << 30, 5, 5]))
    counts = torch.tensor([9, 9, -3, 1 << 30], dtype=torch.int32, device=DEV)
    x = inputs.rows((4, 20, 2, 128), 8)
    model.lens = np.array([0, 2 * bs, 5, 5])
    kvp.kvp_cache_append(c, x.to(DEV), x.to(DEV), counts)
    model.append(x, x, [9, 9, 0, 20])
    _same_codes(c, model)
    table = torch.tensor([[-9, 1 << 30]], dtype=torch.int32, device=DEV)      # first and last page of the pool
    d = kvp.KVCache(c.k_codes, c.v_codes, c.k_scales, c.v_scales, table, torch.zeros(1, dtype=torch.int32, device=DEV), "int8")
    x = inputs.rows((1, 2 * bs, 2, 128), 9)
    kvp.kvp_cache_append(d, x.to(DEV), x.to(DEV))
    y, s = ref.pages_of(x[0, :, 1].float().numpy(), "int8", bs)
    got = ref.code_values(c.k_codes[[0, -1], 1].cpu(), "int8").reshape(-1, 128)
    assert np.array_equal(got, y) and c.k_scales[[0, -1], 1].tolist() == [float(i) for i in s]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("bs", [16, 32, 64, 128])
def test_read(fmt, bs):
    import paper_2512_14946_amd as kvp
    H, R, lens = 3, 75, [0, 1, bs, 200, 131, 256]
    c = inputs.filled_cache(kvp, lens, -(-256 // bs), H, bs, fmt, 9, DEV)
    first = [0, 0, bs - 1, 130, 131, -5]
    model = ref.Cache(c, fmt)
    for firsts in (None, first):
        out = torch.full((2, len(lens), R, H, 136), 3.0, dtype=torch.bfloat16, device=DEV)
        k, v = out[0, ..., :128], out[1, ..., :128]
        kvp.kvp_cache_read(c, k, v, None if firsts is None else torch.tensor(firsts, dtype=torch.int32, device=DEV))
        want = torch.full((2, len(lens), R, H, 136), 3.0, dtype=torch.bfloat16)
        for b, n in enumerate(lens):
            f = 0 if firsts is None else max(firsts[b], 0)
            for h in range(H):
                for i, x in enumerate(model.values(b, h, n, exact=False)):
                    x = torch.from_numpy(x[f:f + R]).to(torch.bfloat16)
                    want[i, b, :len(x), h, :128] = x
        assert torch.equal(out.cpu(), want)
    only = torch.zeros(len(lens), R, H, 128, dtype=torch.bfloat16, device=DEV)
    kvp.kvp_cache_read(c, None, only)
    assert torch.equal(only[3], kvp.kvp_cache_read(c, torch.zeros_like(only), torch.zeros_like(only))[1][3])
