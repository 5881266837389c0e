"""Rotary positions with several axes (conduit_rotary) against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2609_05821_amd import api
from tests import mx_oracle as M
from tests.gpu_helpers import DEV

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rope_of(half, axes, pairing=api.PAIR_HALVES, interleaved=False, base=1e4):
    inv = (base ** (-np.arange(half) / half)).astype(np.float32)
    axis = np.arange(half) % axes if interleaved else np.arange(half) * axes // half
    return api.Rope(inv, axis, n_axes=axes, pairing=pairing)


def expect(x, rope, pos, inverse=False):
    return M.turned(x.cpu(), rope.inv_freq, rope.axis, pos.cpu(), rope.desc.pairing == api.PAIR_ADJACENT, inverse)


def check(got, want, x, dtype):
    """One rounding to fp32 and one to the dtype (half a step each); the 64-bit turn
    itself within 1e-12 of the pair's magnitude (the largest entry of the head)."""
    half_step = torch.finfo(dtype).eps / 2
    big = x.cpu().double().abs().amax(-1, keepdim=True)
    tol = want.abs() * (half_step + 2.0 ** -23) + 1e-12 * big + 1e-38
    err = (got.cpu().double() - want).abs()
    assert (err <= tol).all(), f"worst {(err / tol).max():.3g} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,heads,d,rot,axes,pairing", [
    (1, 1, 8, 8, 1, 0), (1, 28, 128, 128, 3, 0), (7, 4, 64, 64, 3, 1), (1029, 3, 80, 80, 2, 0),
    (33, 5, 72, 72, 2, 0), (33, 5, 72, 72, 2, 1), (130, 2, 128, 64, 4, 0), (130, 2, 128, 34, 2, 0),
    (130, 2, 128, 34, 2, 1), (9, 3, 256, 256, 3, 0), (2050, 7, 96, 48, 1, 0), (5, 2, 64, 2, 1, 0),
    (5, 2, 24, 14, 1, 0), (8200, 1, 16, 16, 2, 1)])
def test_rotary(dtype, n, heads, d, rot, axes, pairing):
    g = torch.Generator().manual_seed(n * 7 + d)
    x = torch.randn(n, heads, d, generator=g).to(DT[dtype]).to(DEV)
    pos = torch.randint(-50, 70000, (axes, n), generator=g, dtype=torch.int32).to(DEV)
    for interleaved in (False, True):
        rope = rope_of(rot // 2, axes, pairing, interleaved)
        for inverse in (False, True):
            out = torch.full_like(x, 7.0)
            api.conduit_rotary(x, rope, pos, out, inverse=inverse)
            check(out, expect(x, rope, pos, inverse), x, DT[dtype])
            assert torch.equal(out[..., rot:], x[..., rot:])


@pytest.mark.parametrize("value", [2 ** 31 - 1, -2 ** 31, 2 ** 20 + 1, 10 ** 7])
def test_far_positions(value):
    """Angles of far positions: the product of a 31-bit position and a 24-bit
    frequency is rounded once (2^-53 relative), so the angle is off by at most
    2^31 * 2^-53 and the result by that times the pair's magnitude."""
    x = torch.randn(3, 2, 64, generator=torch.Generator().manual_seed(1)).to(DEV)
    rope = rope_of(32, 1, base=7.0)
    pos = torch.tensor([value, value // 3, 0], dtype=torch.int32, device=DEV)
    out = torch.empty_like(x)
    api.conduit_rotary(x, rope, pos, out)
    want = expect(x, rope, pos[None])
    tol = want.abs() * 2.0 ** -23 + x.cpu().double().abs().amax(-1, keepdim=True) * 2 * 2.0 ** -22 + 1e-12
    assert ((out.cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,pairing", [(128, 128, 0), (80, 80, 0), (72, 72, 0), (96, 96, 1), (128, 32, 0)])
def test_in_place_and_strided(dtype, d, rot, pairing):
    n, heads = 517, 3
    x = torch.randn(n, heads, d, generator=torch.Generator().manual_seed(d)).to(DT[dtype]).to(DEV)
    pos = torch.arange(2 * n, dtype=torch.int32, device=DEV).view(2, n)
    rope = rope_of(rot // 2, 2, pairing)
    want = torch.empty_like(x)
    api.conduit_rotary(x, rope, pos, want)
    wide = torch.full((n, heads + 2, d), 3.0, dtype=x.dtype, device=DEV)
    wide[:, 1:-1] = x
    api.conduit_rotary(wide[:, 1:-1], rope, pos, wide[:, 1:-1])           # in place, heads of a wider row
    assert torch.equal(wide[:, 1:-1], want)
    assert (wide[:, 0] == 3).all() and (wide[:, -1] == 3).all()
    big = torch.zeros(2, 3 * n, dtype=torch.int32, device=DEV)             # positions inside a longer table
    big[:, n:2 * n] = pos
    out = torch.empty_like(x)
    api.conduit_rotary(x, rope, big[:, n:2 * n], out)
    assert torch.equal(out, want)


def test_gradient():
    """The inverse turn of the output's gradient is the input's: against autograd of the
    formula in 64 bits and against differences (the turn is linear: exact up to
    fp32 roundings of the two calls)."""
    n, heads, d = 5, 2, 80
    g = torch.Generator().manual_seed(3)
    x, go = torch.randn(n, heads, d, generator=g), torch.randn(n, heads, d, generator=g)
    pos = torch.randint(0, 5000, (2, n), generator=g, dtype=torch.int32)
    rope = rope_of(40, 2)
    got = torch.empty(n, heads, d, device=DEV)
    api.conduit_rotary(go.to(DEV), rope, pos.to(DEV), got, inverse=True)
    leaf = x.double().requires_grad_()
    (M.turned(leaf, rope.inv_freq, rope.axis, pos) * go.double()).sum().backward()
    check(got, leaf.grad, go.to(DEV), torch.float32)
    # differences of sum(go * turn(x)) along unit steps of h = 1
    for i, h, e in ((0, 0, 0), (2, 1, 41), (4, 0, 79)):
        up, down = x.clone(), x.clone()
        up[i, h, e] += 1.0
        down[i, h, e] -= 1.0
        vals = []
        for z in (up, down):
            out = torch.empty(n, heads, d, device=DEV)
            api.conduit_rotary(z.to(DEV), rope, pos.to(DEV), out)
            vals.append((out.cpu().double()[i, h] * go.double()[i, h]).sum())
        # 80 outputs of magnitude <= 6 rounded to fp32 in each call, weighted by |go| <= 5
        assert abs((vals[0] - vals[1]) / 2 - got.cpu().double()[i, h, e]) <= 80 * 6 * 5 * 2.0 ** -24


def test_no_rows_and_other_stream():
    x = torch.randn(40, 4, 64, device=DEV)
    rope = rope_of(32, 1)
    pos = torch.arange(40, dtype=torch.int32, device=DEV)
    out = torch.full_like(x, 5.0)
    api.conduit_rotary(x[:0], rope, pos[:0], out[:0])
    assert (out == 5).all()
    want = torch.empty_like(x)
    api.conduit_rotary(x, rope, pos, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        api.conduit_rotary(x, rope, pos, out)
    s.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    torch.cuda.synchronize()
    api.conduit_rotary(x, rope, pos, out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


def test_rows_past_32_bits():
    """Rows spread over more than 2^32 elements."""
    n, stride = 520, 1 << 23                       # 2^32.02 elements of 2 bytes
    buf = torch.empty(n * stride, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((n, 2, 64), (stride, 64, 1))
    small = torch.randn(n, 2, 64, device=DEV).to(torch.bfloat16)
    x.copy_(small)
    rope = rope_of(32, 1)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    want = torch.empty_like(small)
    api.conduit_rotary(small, rope, pos, want)
    api.conduit_rotary(x, rope, pos, x)
    assert torch.equal(x.contiguous(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,heads", [(67, 1), (66, 2), (65, 3), (2700, 36)])
@pytest.mark.parametrize("d,rot,pairing", [(16, 16, 0), (32, 32, 0), (48, 48, 0), (48, 16, 0), (64, 64, 0), (128, 64, 0),
                                           (128, 128, 1), (176, 176, 0), (256, 256, 0), (256, 20, 0)])
def test_heads_over_lanes(dtype, n, heads, d, rot, pairing):
    """Few heads a row and many, over all ways that a head is shared out over lanes."""
    x = torch.randn(n, heads, d, generator=torch.Generator().manual_seed(d + rot)).to(DT[dtype]).to(DEV)
    pos = torch.randint(0, 9000, (2, n), generator=torch.Generator().manual_seed(n), dtype=torch.int32).to(DEV)
    rope = rope_of(rot // 2, 2, pairing)
    out = torch.full_like(x, 7.0)
    api.conduit_rotary(x, rope, pos, out)
    check(out, expect(x, rope, pos), x, DT[dtype])
    assert torch.equal(out[..., rot:], x[..., rot:])
    api.conduit_rotary(x, rope, pos, x)
    assert torch.equal(x, out)
