"""kvp_rotary against the formula in 64 bits (complex products): layouts, parts of the head, positions per token, sequence and kept token,
far and negative positions, strides, in place; its backward and its inverse."""
import numpy as np
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _x(L, T, H, seed):
    return torch.randn(L, T, H, 128, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _positions(kind, L, T, H, seed, far):
    g = torch.Generator().manual_seed(seed)
    shape = {"token": (T,), "sequence": (L, T), "head": (L, H, T)}[kind]
    return torch.randint(-far, far, shape, generator=g).to(torch.int32)


def _full(pos, kind, L, T, H):
    p = pos.numpy()
    return np.broadcast_to({"token": lambda: p[None, :, None], "sequence": lambda: p[:, :, None], "head": lambda: p.transpose(0, 2, 1)}[kind](), (L, T, H))


def _close(got, want, x, mscale):
    # half a bf16 step of the result; of the inputs 2^-20: sine and cosine off by 4 units of 2^-24, an angle of up to
    # half a turn rounded to fp32 (2^-25 turns, 2 pi of it in radians), three roundings of the rotation
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * mscale * np.abs(x).max(axis=-1, keepdims=True) + 1e-38
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rd", [128, 64, 96, 32, 16, 34, 2])
@pytest.mark.parametrize("kind", ["token", "sequence", "head"])
def test_matches_the_formula(layout, rd, kind):
    import paper_2512_14946_amd as kvp
    for L, T, H, far, inverse in ((1, 1, 1, 5, False), (3, 67, 5, 200000, True), (2, 130, 8, 2 ** 31 - 1, False)):
        print("[case] rotary", layout, rd, kind, L, T, H, flush=True)
        x, pos = _x(L, T, H, rd + T), _positions(kind, L, T, H, rd, far)
        freq, _ = kvp.kvp_rotary_frequencies(rd, 10000.0)
        m = 1.25
        want = ref.rotary(x.double().numpy(), _full(pos, kind, L, T, H), freq.numpy(), layout, inverse, m)
        # an angle in double: position * frequency / 2 pi has 53 bits, of which a far position's turns take 31
        assert far <= 2 ** 31
        y = kvp.kvp_rotary(x.to(DEV), pos.to(DEV), freq.to(DEV), layout=layout, inverse=inverse, mscale=m)
        _close(y, want, x.double().numpy(), m)
        assert torch.equal(y[..., rd:].cpu(), x[..., rd:])
        z = x.to(DEV)
        kvp.kvp_rotary(z, pos.to(DEV), freq.to(DEV), out=z, layout=layout, inverse=inverse, mscale=m)   # in place
        assert torch.equal(y.view(torch.int16), z.view(torch.int16))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rd", [128, 40])
def test_strided_views_and_what_lies_between(layout, rd):
    import paper_2512_14946_amd as kvp
    L, T, H = 2, 41, 3
    # heads of a fused projection: every second token of a wider buffer
    buf = _x(L, 2 * T, H + 4, 3).to(DEV)
    x = buf[:, ::2, 2:2 + H]
    pos = _positions("token", L, T, H, 1, 4000)
    freq, _ = kvp.kvp_rotary_frequencies(rd)
    want = ref.rotary(x.double().cpu().numpy(), _full(pos, "token", L, T, H), freq.numpy(), layout, False, 1.0)
    out = torch.full((T, L, H, 136), 7.0, dtype=torch.bfloat16, device=DEV)
    view = out.transpose(0, 1)[..., :128]
    kvp.kvp_rotary(x, pos.to(DEV), freq.to(DEV), out=view, layout=layout)
    _close(view, want, x.double().cpu().numpy(), 1.0)
    assert bool((out[..., 128:] == 7.0).all())
    before = buf.clone()
    kvp.kvp_rotary(x, pos.to(DEV), freq.to(DEV), out=x, layout=layout)
    assert torch.equal(x, view)
    before[:, ::2, 2:2 + H] = x
    assert torch.equal(buf, before)
    # one sequence's rows for all layers: a broadcast source, and positions with a stride of their own
    wide = torch.stack((pos, pos + 9), dim=1).to(DEV)
    y = kvp.kvp_rotary(before[:1, ::2, 2:2 + H].expand(4, T, H, 128), wide[:, 0], freq.to(DEV), layout=layout)
    for l in range(4):
        assert torch.equal(y[l], kvp.kvp_rotary(before[:1, ::2, 2:2 + H], pos.to(DEV), freq.to(DEV), layout=layout)[0])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_backward_is_the_inverse_turn(layout):
    """The call is linear in x: its gradient is the inverse turn of the gradient, against the formula's matrix and against differences."""
    import paper_2512_14946_amd as kvp
    L, T, H, rd, m = 1, 9, 2, 64, 1.5
    x, g, pos = _x(L, T, H, 5), _x(L, T, H, 6), _positions("token", L, T, H, 7, 1000)
    freq, _ = kvp.kvp_rotary_frequencies(rd)
    dx = kvp.kvp_rotary(g.to(DEV), pos.to(DEV), freq.to(DEV), layout=layout, inverse=True, mscale=m)
    f = lambda v: ref.rotary(v, _full(pos, "token", L, T, H), freq.numpy(), layout, False, m)  # noqa: E731
    leaf = torch.zeros(L, T, H, 128, dtype=torch.float64, requires_grad=True)
    a, b = (leaf[..., :rd // 2], leaf[..., rd // 2:rd]) if layout == "half" else (leaf[..., 0:rd:2], leaf[..., 1:rd:2])
    angle = pos[None, :, None, None].double() * freq
    ya, yb = m * (a * angle.cos() - b * angle.sin()), m * (b * angle.cos() + a * angle.sin())
    y = torch.cat((ya, yb), -1) if layout == "half" else torch.stack((ya, yb), -1).flatten(-2)
    (torch.cat((y, leaf[..., rd:]), -1) * g.double()).sum().backward()
    _close(dx, leaf.grad.numpy(), g.double().numpy(), m)
    r = np.random.default_rng(1)
    for _ in range(20):                                       # directional differences of <g, f(x)>
        e = r.standard_normal((L, T, H, 128))
        diff = ((f(x.double().numpy() + e) - f(x.double().numpy() - e)) / 2 * g.double().numpy()).sum()
        got = (dx.double().cpu().numpy() * e).sum()
        assert abs(diff - got) <= 2.0 ** -8 * np.abs(leaf.grad.numpy() * e).sum()
    back = kvp.kvp_rotary(kvp.kvp_rotary(x.to(DEV), pos.to(DEV), freq.to(DEV), layout=layout, mscale=m), pos.to(DEV), freq.to(DEV), layout=layout,
                          inverse=True, mscale=1 / m)
    # (channels behind rd are copied both ways) two roundings of a pair: half a step of each of the two channels it mixes, twice
    assert np.all(np.abs(back.double().cpu().numpy() - x.double().numpy()) <= 4 * 2.0 ** -8 * np.abs(x.double().numpy()).max())


def test_kept_tokens_move_to_their_new_places():
    """Keys rotated at their old positions and moved by the difference equal keys rotated at the new ones."""
    import paper_2512_14946_amd as kvp
    L, T, k, H = 2, 500, 60, 4
    x = _x(L, T, H, 9).to(DEV)
    freq, _ = kvp.kvp_rotary_frequencies(128, 500000.0, "banded", 8.0, 8192.0, 1.0, 4.0)
    f = freq.to(DEV)
    keep = torch.stack([torch.randperm(T, generator=torch.Generator().manual_seed(i))[:k].sort().values for i in range(L * H)]).view(L, H, k).to(torch.int32)
    old = kvp.kvp_rotary(x, torch.arange(T, dtype=torch.int32, device=DEV), f)
    pick = lambda t: t.transpose(1, 2).gather(2, keep.long().to(DEV)[..., None].expand(L, H, k, 128)).transpose(1, 2).contiguous()  # noqa: E731
    moved = kvp.kvp_rotary(pick(old), (torch.arange(k, dtype=torch.int32) - keep).to(DEV), f)
    want = ref.rotary(pick(x).double().cpu().numpy(), np.broadcast_to(np.arange(k)[None, :, None], (L, k, H)), freq.numpy(), "half", False, 1.0)
    # one bf16 rounding more than a single turn: half a step of the larger channel of each pair
    assert np.all(np.abs(moved.double().cpu().numpy() - want) <= 3 * 2.0 ** -8 * np.abs(want).max())
