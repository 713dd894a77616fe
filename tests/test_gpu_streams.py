"""Calls on a stream that is not the current one, while the current stream still writes into memory that torch's allocator counts as free:
results and temporaries of the call may not lie there."""
import pytest
import torch

import cache_inputs as inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _operations(kvp):
    """name -> (call with a stream, bytes of what it allocates)"""
    c = inputs.filled_cache(kvp, [300, 40], 5, 2, 64, "e4m3", 3, DEV)
    q = inputs.rows((2, 6, 8, 128), 4, False).to(DEV)
    ql = torch.tensor([2, 6], dtype=torch.int32, device=DEV)
    acc = torch.rand(2, 2, 320, generator=inputs.gen(5)).to(DEV)
    pos, freq = torch.arange(6, dtype=torch.int32, device=DEV), kvp.kvp_rotary_frequencies(128)[0].to(DEV)
    k = inputs.rows((2, 700, 2, 128), 6).to(DEV)
    scores = torch.rand(5, 20000, generator=inputs.gen(7)).to(DEV)
    d = inputs.empty_cache(kvp, [0, 0], 1, 2, 64, "e4m3", 8, DEV)
    drawn = torch.zeros(2, 2, 320, device=DEV)

    def evict(stream):
        idx = torch.zeros(2, 2, 50, dtype=torch.int32, device=DEV)
        torch.cuda.current_stream().synchronize()
        kvp.kvp_cache_evict(c, acc, 50, d, keep_idx=idx, stream=stream)
        return idx

    def weights(stream):
        kvp.kvp_cache_attend(q, c, acc_out=drawn, stream=stream)
        return drawn
    need = kvp.kvp_cache_attend_workspace_bytes(2, 2, 8, 6, 320, True)
    return {"attend": (lambda s: kvp.kvp_cache_attend(q, c, q_lens=ql, stream=s), q.numel() * 2),
            "attend, weights": (weights, need),
            "evict": (evict, kvp.kvp_cache_evict_workspace_bytes(2, 2, 320, 50)),
            "rotary": (lambda s: kvp.kvp_rotary(q, pos, freq, stream=s), q.numel() * 2),
            "score": (lambda s: kvp.kvp_score_tokens(q, k, stream=s), 2 * 2 * 700 * 4),
            "select": (lambda s: kvp.kvp_select_topk(scores, 300, stream=s), kvp.kvp_select_workspace_bytes(5, 20000, 300))}


@pytest.mark.parametrize("name", ["attend", "attend, weights", "evict", "rotary", "score", "select"])
def test_memory_that_the_current_stream_still_writes_is_left_alone(name):
    import paper_2512_14946_amd as kvp
    call, nbytes = _operations(kvp)[name]
    want = call(None).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        torch.cuda.empty_cache()
        used = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (nbytes, nbytes, 2 * nbytes, 4096)]
        torch.cuda._sleep(20_000_000)                        # 10 ms: the call below is over before the current stream comes to the fills
        for t in used:
            t.fill_(0xFF)
        del used, t                                          # free for the allocator, not yet written
        got = call(stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
