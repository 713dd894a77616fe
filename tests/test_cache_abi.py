"""Refusals of the 8-bit paged cache and of rotary positions: host arithmetic on structs whose pointers are never followed."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2512_14946_amd as kvp
from paper_2512_14946_amd import kvp as binding

lib = binding._lib
NULL, ALIGN, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4, -5


def cache(**kw):
    f = dict(k_codes=4096, v_codes=8192, k_scales=12288, v_scales=16384, block_table=20480, lens=24576, B=3, num_blocks=64, bs=16, H=2, D=128,
             max_blocks=8, table_stride=8, format=0)
    f.update(kw)
    return binding._Cache(**f)


def view(**kw):
    f = dict(ptr=1 << 20, L=3, T=4, H=2, D=128)
    f.update(kw)
    f.setdefault("stride_h", 128)
    f.setdefault("stride_t", f["H"] * 128)
    f.setdefault("stride_l", f["T"] * f["H"] * 128)
    return binding._View(**f)


def ref(x):
    return ctypes.byref(x) if x is not None else None


BAD_CACHES = [(dict(k_codes=None), NULL), (dict(v_scales=None), NULL), (dict(block_table=None), NULL), (dict(lens=None), NULL),
              (dict(D=64), UNSUPPORTED), (dict(bs=8), UNSUPPORTED), (dict(bs=48), UNSUPPORTED), (dict(bs=256), UNSUPPORTED),
              (dict(format=2), UNSUPPORTED), (dict(B=0), SHAPE), (dict(H=0), SHAPE), (dict(num_blocks=0), SHAPE), (dict(max_blocks=0), SHAPE),
              (dict(table_stride=7), SHAPE), (dict(num_blocks=1 << 30), SHAPE), (dict(max_blocks=1 << 27, table_stride=1 << 27), SHAPE),
              (dict(k_codes=4100), ALIGN), (dict(v_scales=16386), ALIGN), (dict(lens=24577), ALIGN)]


@pytest.mark.parametrize("bad,code", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(bad, code):
    c, k = cache(**bad), view()
    assert lib.kvp_cache_append(ref(c), ref(k), ref(k), None, None) == code
    assert lib.kvp_cache_read(ref(c), None, ref(k), ref(k), None) == code
    assert lib.kvp_cache_attend(ref(view()), ref(c), None, 1, 0.1, ref(view()), None, None, 0, 0, 1 << 22, 1 << 30, None) == code
    assert lib.kvp_cache_evict(ref(c), 4096, 128, 8, 0, 0, ref(cache(block_table=1 << 21)), None, None, 0, None, 0, 1 << 22, 1 << 30, None) == code
    if "lens" not in bad:   # the destination's lengths are not read
        assert lib.kvp_cache_evict(ref(cache()), 4096, 128, 8, 0, 0, ref(cache(**{"block_table": 1 << 21, **bad})), None, None, 0, None, 0, 1 << 22,
                                   1 << 30, None) == code


def test_append_and_read_refuse():
    c, k = cache(), view()
    assert lib.kvp_cache_append(None, ref(k), ref(k), None, None) == NULL
    assert lib.kvp_cache_append(ref(c), None, ref(k), None, None) == NULL
    assert lib.kvp_cache_append(ref(c), ref(k), ref(view(T=5)), None, None) == SHAPE
    assert lib.kvp_cache_append(ref(c), ref(k), ref(view(H=1)), None, None) == SHAPE
    assert lib.kvp_cache_append(ref(c), ref(view(L=2)), ref(k), None, None) == SHAPE
    assert lib.kvp_cache_append(ref(c), ref(k), ref(view(D=64)), None, None) == UNSUPPORTED
    assert lib.kvp_cache_append(ref(c), ref(k), ref(view(stride_t=260)), None, None) == ALIGN
    assert lib.kvp_cache_append(ref(c), ref(k), ref(k), 2, None) == ALIGN
    assert lib.kvp_cache_read(ref(c), None, None, None, None) == NULL
    assert lib.kvp_cache_read(ref(c), None, ref(k), ref(view(T=9)), None) == SHAPE
    assert lib.kvp_cache_read(ref(c), None, None, ref(view(H=4)), None) == SHAPE
    assert lib.kvp_cache_read(ref(c), 3, ref(k), None, None) == ALIGN


def attend(q=None, out=None, c=None, acc_in=None, acc_out=None, stride=128, max_len=0, scale=0.1, ws=1 << 22, ws_bytes=1 << 30, q_lens=None):
    q = q or view(H=8)
    return lib.kvp_cache_attend(ref(q), ref(c or cache()), q_lens, 1, scale, ref(out or q), acc_in, acc_out, stride, max_len, ws, ws_bytes, None)


def test_attend_refuses():
    assert attend(q=view(H=3)) == SHAPE
    assert attend(q=view(H=8, L=2)) == SHAPE
    assert attend(out=view(H=8, T=3)) == SHAPE
    assert attend(out=view(H=4)) == SHAPE
    assert attend(q=view(H=8, ptr=None)) == NULL
    assert attend(q=view(H=8, T=1 << 22)) == SHAPE
    assert attend(scale=math.inf) == SHAPE and attend(scale=math.nan) == SHAPE
    assert attend(max_len=-1) == SHAPE
    assert attend(acc_in=4096) == NULL
    assert attend(acc_out=4096, stride=127) == SHAPE
    assert attend(acc_out=4096, stride=99, max_len=100) == SHAPE
    assert attend(acc_out=4098) == ALIGN and attend(q_lens=2) == ALIGN
    need = kvp.kvp_cache_attend_workspace_bytes(3, 2, 8, 4, 128, True)
    assert need > 0
    assert attend(acc_out=4096, ws_bytes=need - 1) == WORKSPACE
    assert attend(acc_out=4096, ws=None) == WORKSPACE
    assert attend(acc_out=4096, ws=(1 << 22) + 8) == WORKSPACE


def evict(src=None, dst=None, acc=4096, stride=128, budget=32, sink=0, recent=0, keep=None, acc_out=None, out_stride=0, lens_out=None, max_len=0,
          ws=1 << 22, ws_bytes=1 << 30):
    return lib.kvp_cache_evict(ref(src or cache()), acc, stride, budget, sink, recent, ref(dst or cache(block_table=1 << 21)), keep, acc_out,
                               out_stride, lens_out, max_len, ws, ws_bytes, None)


def test_evict_refuses():
    assert evict(acc=None) == NULL
    assert evict(budget=0) == SHAPE and evict(budget=-1) == SHAPE
    assert evict(sink=20, recent=13) == SHAPE and evict(sink=-1) == SHAPE and evict(recent=-1) == SHAPE
    assert evict(sink=(1 << 63) - 1, recent=(1 << 63) - 1) == SHAPE
    assert evict(budget=129) == SHAPE                                                  # more than the destination holds
    assert evict(stride=127) == SHAPE and evict(max_len=-1) == SHAPE
    assert evict(acc_out=4096, out_stride=31) == SHAPE
    assert evict(acc=4097) == ALIGN and evict(keep=4098) == ALIGN and evict(acc_out=2, out_stride=32) == ALIGN and evict(lens_out=2) == ALIGN
    assert evict(lens_out=24576) == SHAPE                                              # the source's own lengths
    assert evict(dst=cache()) == SHAPE                                                 # the source's own pages
    for field, value in (("B", 2), ("H", 1), ("format", 1)):
        assert evict(dst=cache(block_table=1 << 21, **{field: value})) == SHAPE
    assert evict(dst=cache(block_table=1 << 21, bs=32)) == SHAPE
    need = kvp.kvp_cache_evict_workspace_bytes(3, 2, 128, 32)
    assert evict(ws_bytes=need - 1) == WORKSPACE and evict(ws=None) == WORKSPACE


def test_one_sizing_call_knows_the_cache_operations():
    assert kvp.kvp_workspace_bytes(kvp.KVP_WS_CACHE_ATTEND, L=3, Hkv=8, Hq=32, W=1, T=4096, method=1) == \
        kvp.kvp_cache_attend_workspace_bytes(3, 8, 32, 1, 4096, True) > kvp.kvp_cache_attend_workspace_bytes(3, 8, 32, 1, 4096, False)
    assert kvp.kvp_workspace_bytes(kvp.KVP_WS_CACHE_EVICT, L=3, Hkv=8, T=20000, k=77) == kvp.kvp_cache_evict_workspace_bytes(3, 8, 20000, 77) > 0
    assert kvp.kvp_cache_attend_workspace_bytes(3, 8, 33, 1, 4096, True) == 0 and kvp.kvp_cache_evict_workspace_bytes(0, 8, 4096, 7) == 0


def rotary(x=None, out=None, pos=4096, strides=(0, 1, 0), freq=8192, rd=128, layout=0):
    x = x or view()
    return lib.kvp_rotary(ref(x), ref(out or x), pos, *strides, freq, rd, layout, 0, 1.0, None)


def test_rotary_refuses():
    assert rotary(pos=None) == NULL and rotary(freq=None) == NULL and rotary(x=view(ptr=None)) == NULL
    assert rotary(rd=0) == UNSUPPORTED and rotary(rd=3) == UNSUPPORTED and rotary(rd=130) == UNSUPPORTED and rotary(layout=2) == UNSUPPORTED
    assert rotary(out=view(T=5)) == SHAPE and rotary(out=view(H=1)) == SHAPE and rotary(strides=(0, -1, 0)) == SHAPE
    assert rotary(out=view(stride_t=512)) == SHAPE                                     # the same memory with other strides
    assert rotary(pos=2) == ALIGN and rotary(freq=8196) == ALIGN
    assert rotary(x=view(L=70000)) == SHAPE


def test_binding_checks_shapes_and_types():
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    c = kvp.alloc_cache(8, 2, 128, 16, table, lens)
    x = torch.zeros(2, 1, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="cuda"):
        kvp.kvp_cache_append(c, x, x)
    with pytest.raises(ValueError, match="cuda"):
        kvp.kvp_rotary(x, torch.zeros(1, dtype=torch.int32), torch.ones(64, dtype=torch.float64))
    for broken in (dict(fmt="fp8"), dict(lens=lens.long()), dict(lens=torch.zeros(3, dtype=torch.int32)), dict(block_table=table.t()),
                   dict(v_codes=c.k_codes), dict(k_scales=c.k_scales[:, :1]), dict(k_codes=c.k_codes.float())):
        with pytest.raises(ValueError):
            binding._cache(kvp.KVCache(**{**{f: getattr(c, f) for f in ("k_codes", "v_codes", "k_scales", "v_scales", "block_table", "lens", "fmt")},
                                          **broken}))
    with pytest.raises(ValueError):
        kvp.kvp_rotary_frequencies(64, scaling="other")


def test_marshalled_cache_follows_replaced_tensors(monkeypatch):
    monkeypatch.setattr(binding, "_one_device", lambda *ts: None)
    c = kvp.alloc_cache(8, 2, 128, 16, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    a = binding._cache(c)
    assert binding._cache(c) is a
    c.lens = torch.zeros(2, dtype=torch.int32)
    b = binding._cache(c)
    assert b is not a and b.lens == c.lens.data_ptr()
    c.block_table = torch.zeros(2, 6, dtype=torch.int32)[:, :3]
    d = binding._cache(c)
    assert (d.max_blocks, d.table_stride) == (3, 6)
    c.fmt = "e4m3"
    assert binding._cache(c).format == 1


@pytest.mark.parametrize("rd", [2, 64, 128])
@pytest.mark.parametrize("scaling", ["plain", "linear", "ntk", "yarn", "banded"])
def test_rotary_frequencies(rd, scaling):
    base, factor, original, low, high = 500000.0, 8.0, 8192.0, 1.0, 4.0
    if scaling == "ntk" and rd == 2:
        with pytest.raises(kvp.KVPError):
            kvp.kvp_rotary_frequencies(rd, base, scaling, factor)
        return
    f, m = kvp.kvp_rotary_frequencies(rd, base, scaling, factor, original, low, high)
    plain = np.array([base ** (-2 * i / rd) for i in range(rd // 2)])
    turns = original * plain / (2 * math.pi)
    if scaling == "plain":
        want = plain
    elif scaling == "linear":
        want = plain / factor
    elif scaling == "ntk":
        want = np.array([(base * factor ** (rd / (rd - 2))) ** (-2 * i / rd) for i in range(rd // 2)])
        assert abs(want[-1] * factor / plain[-1] - 1) < 1e-12 and want[0] == 1.0       # slowest pair as linear, fastest as it was
    elif scaling == "banded":
        u = np.clip((turns - low) / (high - low), 0, 1)
        want = (1 - u) * plain / factor + u * plain
    else:
        at = lambda r: rd * math.log(original / (r * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rd - 1)
        u = np.array([min(max((i - a) / (b - a), 0), 1) for i in range(rd // 2)])
        want = u * plain / factor + (1 - u) * plain
    assert np.allclose(f.numpy(), want, rtol=1e-13, atol=0)
    assert m == pytest.approx(0.1 * math.log(factor) + 1 if scaling == "yarn" else 1.0, rel=1e-7)


def test_rotary_frequencies_refuse():
    for kw in (dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=256), dict(rotary_dim=64, base=1.0), dict(rotary_dim=64, base=math.inf),
               dict(rotary_dim=64, scaling="linear", factor=0.5), dict(rotary_dim=64, scaling="yarn", factor=2.0),
               dict(rotary_dim=64, scaling="banded", factor=2.0, original=4096.0, low=4.0, high=4.0)):
        with pytest.raises(kvp.KVPError):
            kvp.kvp_rotary_frequencies(**kw)


def test_results_that_would_overwrite_what_is_read_are_refused():
    need = kvp.kvp_cache_attend_workspace_bytes(3, 2, 8, 4, 128, True)
    assert attend(ws_bytes=need, acc_out=4096) == SHAPE                                # queries and results in one place
    assert evict(acc_out=4096, out_stride=128) == SHAPE                                # weights in and out


def test_launches_beyond_what_a_grid_takes_are_refused():
    big = dict(num_blocks=1 << 20, max_blocks=1 << 20, table_stride=1 << 20, bs=16, B=16)
    c = cache(**big)                                                                   # 2^25 pages of a head
    k = view(L=16, T=1 << 24)
    assert lib.kvp_cache_append(ref(c), ref(k), ref(k), None, None) == SHAPE
    assert lib.kvp_cache_read(ref(c), None, ref(k), None, None) == SHAPE
    assert evict(src=c, dst=cache(block_table=1 << 21, **big), budget=1 << 24, stride=1 << 24, ws_bytes=1 << 62) == SHAPE
    wide = cache(B=1 << 22, num_blocks=1, max_blocks=1, table_stride=1)
    assert attend(q=view(L=1 << 22, H=8), out=view(L=1 << 22, H=8, ptr=1 << 30), c=wide, ws_bytes=1 << 62) == SHAPE
    assert rotary(x=view(T=1 << 27, H=8), rd=8) == SHAPE


def test_a_workspace_serves_every_smaller_bound():
    g = torch.Generator().manual_seed(1)
    for B, H, G, W in [(1, 1, 1, 1), (1, 8, 4, 1), (3, 2, 7, 3), (2, 1, 1, 100), (1, 2, 4, 600), (64, 8, 8, 1), (33, 8, 4, 1), (5, 8, 8, 5), (2, 8, 4, 1100), (43, 1, 3, 15), (1, 8, 20, 1),
                       (7, 8, 12, 8), (2, 8, 16, 7)]:
        for weights in (False, True):
            before = 0
            for T in sorted(torch.randint(1, 70000, (400,), generator=g).tolist() + [255, 256, 257, 512, 513, 768, 1024, 1025]):
                need = kvp.kvp_cache_attend_workspace_bytes(B, H, H * G, W, T, weights)
                assert need >= before, (B, H, G, W, T)
                before = need


def test_sizes_that_no_call_accepts_are_none():
    big = 1 << 32
    assert kvp.kvp_cache_attend_workspace_bytes(big, big, big, 1, 4096, True) == 0     # a product that wraps to nothing
    assert kvp.kvp_cache_attend_workspace_bytes(1, 1, 1, 1, 1 << 62, True) == 0
    assert kvp.kvp_cache_attend_workspace_bytes(1, 1, 1 << 40, 1 << 40, 64, False) == 0
    assert kvp.kvp_cache_evict_workspace_bytes(big, big, 64, 8) == 0 and kvp.kvp_cache_evict_workspace_bytes(1, 1, 1 << 62, 8) == 0
    assert kvp.kvp_workspace_bytes(kvp.KVP_WS_CACHE_ATTEND, L=big, Hkv=big, Hq=big, W=1, T=64, method=0) == 0
    assert kvp.kvp_workspace_bytes(kvp.KVP_WS_CACHE_EVICT, L=big, Hkv=big, T=64, k=8) == 0


def test_copies_of_a_used_cache_refer_to_their_own_tensors(monkeypatch):
    import copy
    import pickle
    monkeypatch.setattr(binding, "_one_device", lambda *ts: None)
    c = kvp.alloc_cache(8, 2, 128, 16, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    a = binding._cache(c)
    for d in (copy.deepcopy(c), pickle.loads(pickle.dumps(c))):
        b = binding._cache(d)
        assert b.k_codes == d.k_codes.data_ptr() != a.k_codes and b.lens == d.lens.data_ptr() != a.lens
    assert binding._cache(c) is a
