"""kvp_cache_attend against softmax in 64 bits over the cache's own values: formats, page sizes, head groups, lengths from none to
thousands, ragged batches, masks that leave rows empty, poison wherever no call may look, and the weights that tokens draw."""
import math

import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(kvp, c, W, G, seed, q_lens=None, causal=True, scale=None, max_len=0, weights=True, sharp=1.0, note=""):
    B, H = c.block_table.shape[0], c.k_codes.shape[1]
    print("[case] attend", c.fmt, c.bs, c.lens.tolist(), dict(W=W, G=G, q_lens=q_lens, causal=causal, max_len=max_len), note, flush=True)
    q = inputs.rows((B, W, H * G, 128), seed, False) * sharp
    if q_lens is not None:
        for b, n in enumerate(q_lens):
            q[b, max(n, 0):] = float("nan")                 # rows that are no queries
    model = ref.Cache(c, c.fmt)
    cap = c.block_table.shape[1] * c.bs
    bound = min(max_len, cap) if max_len else cap
    f = 1 / math.sqrt(128) if scale is None else scale
    model.lens = np.clip(model.lens, 0, bound)
    want, drawn, mag, vmax, size = ref.attend(model, q, q_lens, causal, f)
    out = torch.full(q.shape, 5.0, dtype=torch.bfloat16, device=DEV)
    ql = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device=DEV)
    acc = acc_out = None
    if weights:
        acc = torch.rand(B, H, bound + 3, generator=inputs.gen(seed)).to(DEV)
        acc_out = torch.full_like(acc, -1.0)
    kvp.kvp_cache_attend(q.to(DEV), c, out, q_lens=ql, causal=causal, scale=scale, max_len=max_len, acc_in=acc, acc_out=acc_out)
    got = out.double().cpu().numpy()
    tol = ref.out_tolerance(want, mag, vmax, size, model.lens)
    for b in range(B):
        m = W if q_lens is None else min(max(q_lens[b], 0), W)
        err = np.abs(got[b, :m] - want[b, :m])
        assert np.all(err <= tol[b, :m]), (b, err.max(), tol[b, :m].flat[err.argmax()])
        assert np.all(got[b, m:] == 5.0)                    # padding rows are left alone
    if not weights:
        return out, None
    a_in, a = acc.double().cpu().numpy(), acc_out.double().cpu().numpy()
    for b in range(B):
        n = int(model.lens[b])
        t = ref.drawn_tolerance(drawn[b:b + 1, :, :n], a_in[b:b + 1, :, :n], size[b:b + 1])[0]
        err = np.abs(a[b, :, :n] - a_in[b, :, :n] - drawn[b, :, :n])
        assert np.all(err <= t), (b, (err / t).max())
        assert np.all(a[b, :, n:] == -1.0)
    # the same without an input sum, and in place: the same sums
    zero = torch.full_like(acc, -1.0)
    kvp.kvp_cache_attend(q.to(DEV), c, torch.empty_like(out).copy_(out), q_lens=ql, causal=causal, scale=scale, max_len=max_len, acc_out=zero)
    kvp.kvp_cache_attend(q.to(DEV), c, torch.empty_like(out).copy_(out), q_lens=ql, causal=causal, scale=scale, max_len=max_len, acc_in=acc, acc_out=acc)
    for b in range(B):
        n = int(model.lens[b])
        assert torch.equal(acc[b, :, :n], acc_out[b, :, :n])
        assert torch.equal(torch.from_numpy(a_in[b, :, :n]).float().to(DEV) + zero[b, :, :n], acc_out[b, :, :n])
    return out, acc_out


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("G", [1, 3, 4, 7, 8, 16, 17])
def test_decode(fmt, bs, G):
    import paper_2512_14946_amd as kvp
    lens = [1, 0, 2, 15, 16, 17, 63, 64, 65, 129, 300, 511]
    c = inputs.filled_cache(kvp, lens, 512 // bs, 2, bs, fmt, G + bs, DEV)
    _check(kvp, c, 1, G, G)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("W,G", [(2, 4), (3, 5), (5, 16), (40, 1), (33, 7), (130, 4)])
@pytest.mark.parametrize("causal", [True, False])
def test_many_query_tokens(fmt, W, G, causal):
    import paper_2512_14946_amd as kvp
    lens = [W, W + 1, 0, W // 2, 200, 257]                 # shorter than the queries: the first rows see nothing
    c = inputs.filled_cache(kvp, lens, 18, 2, 16, fmt, W + G, DEV)
    _check(kvp, c, W, G, W, causal=causal)
    q_lens = [0, 1, W, W // 2, W + 9, max(W - 1, 0)]       # a padded batch; more than W counts as W
    _check(kvp, c, W, G, W + 1, q_lens=[min(x, W) for x in q_lens], causal=causal)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("G,W,H,n", [(4, 1, 1, 20000), (8, 1, 8, 4500), (7, 3, 1, 9001), (4, 70, 2, 3001)])
def test_long_sequences_are_split_and_joined(fmt, G, W, H, n):
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [n, 100], -(-n // 64), H, 64, fmt, 3, DEV)
    a, wa = _check(kvp, c, W, G, 5)
    b, wb = _check(kvp, c, W, G, 5)                        # the same bits on another call
    assert torch.equal(a, b) and torch.equal(wa, wb)
    _check(kvp, c, W, G, 6, max_len=n + 1000)
    _check(kvp, c, W, G, 6, max_len=n - 77)                # longer sequences count as max_len tokens


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("W", [1, 24])
def test_sharp_and_flat_distributions_and_scales(fmt, W):
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [700, 333], 44, 2, 16, fmt, 8, DEV, spread=2.0)       # page scales e^2 apart and more
    _check(kvp, c, W, 4, 1, note="spread")
    _check(kvp, c, W, 4, 2, sharp=30.0, note="sharp")      # one token takes all
    _check(kvp, c, W, 4, 3, scale=0.0, note="uniform")
    _check(kvp, c, W, 4, 4, scale=-0.05, note="negative scale")
    _check(kvp, c, W, 4, 5, sharp=2.0 ** -120, note="tiny")
    _check(kvp, c, W, 4, 6, sharp=2.0 ** 100, scale=2.0 ** -104, note="huge")
    # logits that grow along the sequence move the reference again and again
    for b in range(2):
        for i in range(44):
            c.k_scales[c.block_table[b, i].long()] *= 1.2 ** i if b else 1.2 ** (44 - i)
    _check(kvp, c, W, 4, 7, scale=0.002, note="growing")


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_zero_pages(fmt):
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [150, 64], 10, 2, 16, fmt, 9, DEV)
    for i in (0, 1, 2, 3, 7):                              # the first tile's values are all zero
        p = c.block_table[0, i].long()
        c.v_codes[p] = 0
        c.v_scales[p] = 0.0
    p = c.block_table[1, 2].long()
    c.k_codes[p] = 0
    c.k_scales[p] = 0.0
    _check(kvp, c, 1, 4, 1)
    _check(kvp, c, 9, 4, 2)


def test_strided_queries_outputs_and_shared_pages():
    import paper_2512_14946_amd as kvp
    B, W, H, G, bs = 3, 2, 2, 4, 32
    c = inputs.filled_cache(kvp, [70, 70, 70], 3, H, bs, "int8", 4, DEV)
    table = c.block_table.clone()
    table[1, :2] = table[0, :2]                            # a shared prefix of full pages
    c.block_table = table
    buf = inputs.rows((W, B, H * G + 3, 128), 5, False).to(DEV)
    q = buf.transpose(0, 1)[:, :, 3:]
    out = torch.full((B, H * G, W + 1, 136), 9.0, dtype=torch.bfloat16, device=DEV)
    view = out.transpose(1, 2)[:, :W, :, :128]
    kvp.kvp_cache_attend(q, c, view)
    want = kvp.kvp_cache_attend(q.contiguous(), c)
    assert torch.equal(view, want)
    assert bool((out[:, :, W] == 9.0).all()) and bool((out[..., 128:] == 9.0).all())
    one = kvp.KVCache(c.k_codes, c.v_codes, c.k_scales, c.v_scales, table[1:2], c.lens[1:2], "int8")
    assert torch.equal(kvp.kvp_cache_attend(q[1:2], one), want[1:2])     # a sequence alone gives what it gives in a batch
    acc = torch.zeros(B, H, 200, device=DEV)[..., :100]
    kvp.kvp_cache_attend(q, c, view, acc_out=acc)
    assert abs(float(acc.sum()) - B * H * G * W) < 1e-3


def test_lengths_and_pages_out_of_range_are_clamped():
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [48, 48, 48], 3, 2, 16, "int8", 6, DEV)
    c.lens.copy_(torch.tensor([1 << 30, -5, 48]))
    out, _ = _check(kvp, c, 2, 4, 1)
    assert bool((out[1] == 0).all())
    bad = c.block_table.clone()
    bad[2, 1] = 1 << 30
    bad[2, 2] = -1
    d = kvp.KVCache(c.k_codes, c.v_codes, torch.nan_to_num(c.k_scales, 1.0), torch.nan_to_num(c.v_scales, 1.0), bad, c.lens, "int8")
    good = bad.clone()
    good[2, 1], good[2, 2] = c.k_codes.shape[0] - 1, 0
    e = kvp.KVCache(c.k_codes, c.v_codes, d.k_scales, d.v_scales, good, c.lens, "int8")
    q = inputs.rows((3, 1, 8, 128), 2, False).to(DEV)
    assert torch.equal(kvp.kvp_cache_attend(q, d), kvp.kvp_cache_attend(q, e))


def test_two_streams_with_workspaces_of_their_own():
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [3000, 2500], 188, 2, 16, "e4m3", 7, DEV)
    qs = [inputs.rows((2, 1, 8, 128), 10 + i, False).to(DEV) for i in range(2)]
    want = [kvp.kvp_cache_attend(q, c) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [torch.zeros_like(q) for q in qs]
    for _ in range(5):
        for s, q, o in zip(streams, qs, got):
            kvp.kvp_cache_attend(q, c, o, stream=s)        # a workspace of the call's own
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


def test_binding_refuses_mixed_arguments():
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [20], 2, 2, 16, "int8", 8, DEV)
    q = inputs.rows((1, 1, 4, 128), 1, False).to(DEV)
    with pytest.raises(ValueError):
        kvp.kvp_cache_attend(q.cpu(), c)
    with pytest.raises(ValueError):
        kvp.kvp_cache_attend(q, c, acc_in=torch.zeros(1, 2, 32, device=DEV))
    with pytest.raises(ValueError):
        kvp.kvp_cache_attend(q, c, acc_out=torch.zeros(1, 2, 31, device=DEV))
    with pytest.raises(ValueError):
        kvp.kvp_cache_attend(q, c, q_lens=torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        kvp.kvp_cache_attend(q.float(), c)
    with pytest.raises(kvp.KVPError):
        kvp.kvp_cache_attend(q[:, :, :3], c)
    with pytest.raises(kvp.KVPError):
        kvp.kvp_cache_attend(q, c, ws=torch.zeros(1, dtype=torch.uint8, device=DEV), acc_out=torch.zeros(1, 2, 32, device=DEV))
