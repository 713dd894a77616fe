"""Which stream the binding allocates, clears and launches on (no GPU: the calls of torch and of the library are recorded)."""
import pytest
import torch

from paper_2512_14946_amd import kvp as binding


def test_a_stream_handle_belongs_to_the_tensors_device(monkeypatch):
    made = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: made.append((handle, device)) or "stream")
    assert binding._torch_stream(77, torch.device("cuda", 1)) == "stream"
    assert made == [(77, torch.device("cuda", 1))]                 # not the current device's


class _Recorder:
    """torch and the library replaced where a call would need a GPU; `where` is the stream of every allocation and fill."""

    def __init__(self, monkeypatch):
        self.now, self.where = None, []
        rec = self

        class On:
            def __init__(self, stream):
                self.stream = stream

            def __enter__(self):
                self.before, rec.now = rec.now, self.stream

            def __exit__(self, *exc):
                rec.now = self.before

        def spy(owner, name):
            real = getattr(owner, name)

            def call(*a, **k):
                rec.where.append((name, rec.now))
                return real(*a, **k)
            monkeypatch.setattr(owner, name, call)

        class Library:
            def __getattr__(self, name):
                return lambda *a: 64 if name.endswith("_bytes") else 0

        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
        monkeypatch.setattr(torch.cuda, "stream", On)
        monkeypatch.setattr(binding, "_lib", Library())
        monkeypatch.setattr(binding, "_need_cuda", lambda *ts: None)
        monkeypatch.setattr(binding, "_one_device", lambda *ts: None)
        monkeypatch.setattr(binding, "_stream", lambda stream, like=None: stream)
        monkeypatch.setattr(binding, "_launch", lambda like, stream, what, fn, *a: fn(*a, stream))
        for owner, name in ((torch, "empty"), (torch, "empty_like"), (torch, "zeros"), (torch.Tensor, "zero_")):
            spy(owner, name)


def _calls():
    x = torch.ones(2, 6, 4, 128, dtype=torch.bfloat16)
    s = torch.ones(3, 40)
    n = torch.ones(2, dtype=torch.int32)
    c = binding.KVCache(*[torch.ones(4, 2, *p, dtype=torch.uint8) for p in ((16, 128), (128, 16))], torch.ones(4, 2), torch.ones(4, 2),
                        torch.ones(2, 2, dtype=torch.int32), n)
    d = binding.KVCache(c.k_codes, c.v_codes, c.k_scales, c.v_scales, torch.zeros_like(c.block_table), n)
    acc, pos, freq = torch.ones(2, 2, 32), torch.ones(6, dtype=torch.int32), torch.ones(64, dtype=torch.float64)
    return {"score_tokens": (lambda st: binding.kvp_score_tokens(x, x, stream=st), 2),
            "score_keys": (lambda st: binding.kvp_score_keys(x, 0, stream=st), 2),
            "select_topk": (lambda st: binding.kvp_select_topk(s, 5, stream=st), 2),
            "smooth_scores": (lambda st: binding.kvp_smooth_scores(s, 4, 3, stream=st), 1),
            "eval_configs": (lambda st: binding.kvp_eval_configs(x, x, x, [(4, 64, 3)], stream=st, want_partial=True), 3),
            "cache_attend": (lambda st: binding.kvp_cache_attend(x, c, stream=st), 2),
            "cache_attend, rows left out": (lambda st: binding.kvp_cache_attend(x, c, q_lens=n, stream=st), 3),
            "cache_evict": (lambda st: binding.kvp_cache_evict(c, acc, 9, d, stream=st), 1),
            "rotary": (lambda st: binding.kvp_rotary(x, pos, freq, stream=st), 1)}


@pytest.mark.parametrize("name", sorted(_calls()))
def test_what_a_call_allocates_belongs_to_its_stream(monkeypatch, name):
    call, n = _calls()[name]
    rec = _Recorder(monkeypatch)
    for stream in (77, None):
        rec.where.clear()
        call(stream)
        assert len(rec.where) == n and all(at == stream for _, at in rec.where), rec.where
    assert rec.now is None
