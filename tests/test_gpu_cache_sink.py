"""kvp_cache_attend where most of a row's weight lies on a token of no value (the first token of a real prompt draws most of it and has next
to no value: a code of 0 on its page's scale), so that the result is made of the many probabilities far below the largest; and values at the
ends of the range."""
import math

import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _bytes(x, fmt):
    return x.to(torch.int8).view(torch.uint8) if fmt == "int8" else x.to(torch.float8_e4m3fn).view(torch.uint8)


def _sink_cache(kvp, T, bs, fmt, seed):
    """One sequence and head: token 0 has the largest key code in every channel and the value 0, the others small keys and positive values."""
    g, most, pages = inputs.gen(seed), int(ref.QMAX[fmt]), -(-T // bs)
    k = torch.randint(-3, 4, (pages, 1, bs, 128), generator=g).float()
    v = torch.randint(1, 128, (pages, 1, 128, bs), generator=g).float() * (most / 127)
    k[0, 0, 0], v[0, 0, :, 0] = most, 0
    scales = [torch.full((pages, 1), 0.01 * 127 / most, device=DEV) for _ in range(2)]
    table = torch.randperm(pages, generator=g)
    codes = []
    for x in (k, v):
        y = torch.empty(x.shape, dtype=torch.uint8)
        y[table] = _bytes(x, fmt)
        codes.append(y.to(DEV))
    return kvp.KVCache(*codes, *scales, table.to(torch.int32).view(1, -1).to(DEV), torch.tensor([T], dtype=torch.int32, device=DEV), fmt)


def _sink_queries(W, G, T, seed):
    """Rows whose weight on the sink is 0.9 to 0.995: a logit of ln(weight / (1 - weight) * others) by way of 128 equal products."""
    g = inputs.gen(seed)
    part = 0.9 + 0.095 * torch.rand(1, W, G, 1, generator=g)
    logit = torch.log(part / (1 - part) * (T - 1))
    return (logit * math.sqrt(128) / (128 * 1.27) * (1 + 0.1 * torch.randn(1, W, G, 128, generator=g))).to(torch.bfloat16)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("T,bs", [(300, 16), (16384, 32), (131072, 128)])
@pytest.mark.parametrize("W,G", [(1, 4), (2, 10), (26, 5)])
@pytest.mark.parametrize("B", [1, 256])
def test_weight_on_a_token_of_no_value(fmt, T, bs, W, G, B):
    # B sequences over the same pages: 256 leave a block all tokens, one splits them, and the largest logit reaches only its own chunk
    import paper_2512_14946_amd as kvp
    print("[case] sink", fmt, T, bs, W, G, B, flush=True)
    c, q = _sink_cache(kvp, T, bs, fmt, T + W), _sink_queries(W, G, T, W).to(DEV)
    want, drawn, mag, vmax, size = ref.attend(ref.Cache(c, fmt), q.float().cpu(), None, True, 1 / math.sqrt(128))
    assert 0.5 < float(drawn[0, 0, 0]) / (W * G) < 0.999
    # half a bf16 step; 2^-11 of every product; 2^-35 of the largest probability times the largest value for each token; the probabilities'
    # own error as in ref.out_tolerance
    delta = 2 * 140 * 2.0 ** -24 * size[0] + 2.0 ** -20
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + delta) * mag * 1.01 + T * 2.0 ** -35 * vmax[0]
    many = kvp.KVCache(c.k_codes, c.v_codes, c.k_scales, c.v_scales, c.block_table.repeat(B, 1), c.lens.repeat(B), fmt)
    qs = q.repeat(B, 1, 1, 1)
    acc = torch.zeros(B, 1, T, device=DEV)
    for weights in (None, acc):
        got = kvp.kvp_cache_attend(qs, many, max_len=T, acc_out=weights)
        err = np.abs(got[:1].double().cpu().numpy() - want)
        assert np.all(err <= tol), (err / tol).max()
        assert torch.equal(got, got[:1].expand_as(got))
    e = np.abs(acc[:1].double().cpu().numpy() - drawn)
    assert np.all(e <= ref.drawn_tolerance(drawn, 0.0, size))
    assert torch.equal(acc, acc[:1].expand_as(acc))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("power", [117, 60, -80])
@pytest.mark.parametrize("W,G", [(1, 4), (2, 10), (26, 5)])
def test_values_at_the_ends_of_the_range(fmt, power, W, G):
    # sums of probabilities reach 2^15.5 times the tokens: sums of their products with values may not be formed on the values' own scale
    import paper_2512_14946_amd as kvp
    c = inputs.filled_cache(kvp, [3000, 200], 188, 2, 16, fmt, W, DEV, spread=0.5)
    c.v_scales.mul_(2.0 ** power)
    q = inputs.rows((2, W, 2 * G, 128), 9, False).to(DEV)
    print("[case] range", fmt, power, W, G, flush=True)
    want, _, mag, vmax, size = ref.attend(ref.Cache(c, fmt), q.float().cpu(), None, True, 1 / math.sqrt(128))
    assert np.all(np.isfinite(want.astype(np.float32)))
    # the logarithm of a scale of 2^-128 .. 2^128 is off by 2^-18 at most, that of the reference scale too
    tol = ref.out_tolerance(want, mag, vmax, size, [3000, 200]) + 2 * 2.0 ** -18 * mag
    err = np.abs(kvp.kvp_cache_attend(q, c).double().cpu().numpy() - want)
    assert np.all(err <= tol), (err / tol).max()
