"""kvp_cache_attend where values cancel: every token of a key comes twice, with a value and its negative, and the logits of the two differ a little, so that
the result is the difference of nearly equal probabilities and shows their rounding."""
import math

import numpy as np
import pytest
import torch

import cache_inputs as inputs
import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("W,G,bits", [(1, 1, 22), (1, 4, 22), (1, 16, 22), (4, 4, 22), (1, 20, 11), (5, 8, 11), (20, 7, 11)])
@pytest.mark.parametrize("pairs", [1, 3, 100])
@pytest.mark.parametrize("weights", [False, True])
def test_differences_of_probabilities(fmt, W, G, bits, pairs, weights):
    import paper_2512_14946_amd as kvp
    n, H = 2 * pairs, 2
    v = inputs.rows((1, pairs, H, 128), pairs, False).repeat_interleave(2, 1)
    v[:, 1::2] *= -1
    k = inputs.rows((1, n, H, 128), 3, False)
    c = inputs.empty_cache(kvp, [0], -(-n // 16), H, 16, fmt, 4, DEV)
    kvp.kvp_cache_append(c, k.to(DEV), v.to(DEV))
    c.lens.fill_(n)
    q = (inputs.rows((1, W, H * G, 128), 5, False).float() * 0.01).to(torch.bfloat16).to(DEV)   # logits of some hundredths
    print("[case] cancel", fmt, W, G, pairs, weights, flush=True)
    want, _, mag, vmax, size = ref.attend(ref.Cache(c, fmt), q.float().cpu(), None, False, 1 / math.sqrt(128))
    acc = torch.zeros(1, H, c.block_table.shape[1] * 16, device=DEV) if weights else None
    got = kvp.kvp_cache_attend(q, c, causal=False, acc_out=acc).double().cpu().numpy()
    # as ref.out_tolerance, with the bits that the header states
    delta = 2 * 140 * 2.0 ** -24 * size[0] + 2.0 ** -20
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -bits + delta) * mag * 1.01 + n * 2.0 ** -35 * vmax[0]
    err = np.abs(got - want)
    assert np.all(err <= tol), (err / tol).max()
