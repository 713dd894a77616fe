"""Which stream the binding allocates, clears and launches on (no GPU: the calls of torch and of the library are recorded)."""
import torch

from paper_2512_14946_amd import kvp as binding


def test_a_stream_handle_belongs_to_the_tensors_device(monkeypatch):
    made = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: made.append((handle, device)) or "stream")
    assert binding._torch_stream(77, torch.device("cuda", 1)) == "stream"
    assert made == [(77, torch.device("cuda", 1))]                 # not the current device's
