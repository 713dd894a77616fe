"""The struct that the binding keeps for a KVCache (no GPU: only pointers, shapes, strides and types are read)."""
import pytest
import torch

from paper_2512_14946_amd import kvp as binding


def test_cache_struct_follows_tensors_changed_in_place(monkeypatch):
    monkeypatch.setattr(binding, "_one_device", lambda *ts: None)
    lens = torch.zeros(4, dtype=torch.int32)[:2]
    c = binding.alloc_cache(8, 2, 128, 16, torch.zeros(2, 4, dtype=torch.int32), lens)
    a = binding._cache(c)
    assert binding._cache(c) is a
    lens.as_strided_((2,), (2,))                                   # same object, pointer and shape
    with pytest.raises(ValueError, match="lens"):
        binding._cache(c)
    lens.as_strided_((2,), (1,))
    assert binding._cache(c).lens == a.lens
    c.k_scales.data = c.k_scales.view(torch.int32)
    with pytest.raises(ValueError, match="scales"):
        binding._cache(c)


def test_the_distance_of_a_single_row_does_not_matter():
    a, b = torch.zeros(1, 1, 100), torch.zeros(1, 3, 200)[:, 1:2]
    assert binding._weight_rows(a, 1, 1, 90, "acc_in")[1] == binding._weight_rows(b, 1, 1, 90, "acc_out")[1] == 90
    assert binding._weight_rows(torch.zeros(2, 1, 100), 2, 1, 90, "acc")[1] == 100
    assert binding._weight_rows(torch.zeros(1, 2, 100)[..., 5:], 1, 2, 90, "acc")[1] == 100
