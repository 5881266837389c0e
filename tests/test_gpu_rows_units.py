"""Turns, appends and loads large enough that a wave takes two units of heads: equal, bit for
bit, to the same rows in calls of a few hundred, which the other tests hold to 64 bits."""
import pytest
import torch

from paper_2609_05821_amd import api
from tests.gpu_helpers import DEV
from tests.test_gpu_rotary import DT

pytestmark = pytest.mark.gpu

D, HQ, HKV, N, CTX, PIECE = 128, 16, 16, 4200, 4224, 300
# how a head is shared out: both dims of a pair in a lane, 8 dims a lane with the pairs side by
# side or with partners of their own, partners one by one
ROPES = {"whole": (128, api.PAIR_HALVES), "adjacent": (96, api.PAIR_ADJACENT), "part": (64, api.PAIR_HALVES),
         "single": (72, api.PAIR_HALVES)}


def rope(kind):
    rot, pairing = ROPES[kind]
    half = rot // 2
    return api.Rope([10000.0 ** (-i / half) for i in range(half)], [i % 3 for i in range(half)], pairing=pairing)


def data(dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, HQ + 2 * HKV, D, generator=g).to(DT[dtype]).to(DEV)
    pos = torch.randperm(CTX, generator=g)[:N].to(torch.int32).to(DEV)
    return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:], pos, \
        torch.randint(-99, 9999, (3, N), generator=g, dtype=torch.int32).to(DEV)


def pieces():
    return [slice(i, min(i + PIECE, N)) for i in range(0, N, PIECE)]


def pools():
    return [torch.zeros(CTX // 64, HKV, 64, b, dtype=torch.uint8, device=DEV) for b in (D // 2, D // 2, D // 32, D // 32)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["whole", "adjacent", "part", "single"])
def test_turn(dtype, kind):
    q, _, _, _, rp = data(dtype)
    whole, parts = (torch.zeros(N, HQ, D, dtype=q.dtype, device=DEV) for _ in range(2))
    api.conduit_rotary(q, rope(kind), rp, whole)
    for s in pieces():
        api.conduit_rotary(q[s], rope(kind), rp[:, s].contiguous(), parts[s])
    assert torch.equal(whole, parts) and not torch.equal(whole, q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["whole", "adjacent", "part"])
@pytest.mark.parametrize("bits", [4, 16])
def test_append(dtype, kind, bits):
    q, k, v, pos, rp = data(dtype, 1)
    out = []
    for call in ([slice(0, N)], pieces()):
        c = pools() if bits == 4 else [torch.zeros(CTX, HKV, D, dtype=q.dtype, device=DEV) for _ in range(2)]
        rows = [torch.zeros(N, HQ, D, dtype=q.dtype, device=DEV) for _ in range(3 if bits == 4 else 1)]
        for s in call:
            kw = dict(rope=rope(kind), rope_pos=rp[:, s].contiguous(), q=q[s], q_out=rows[0][s])
            if bits == 4:
                api.conduit_append_mx(api.mx_desc(*c, HQ), pos[s], k[s], v[s], k_out=rows[1][s], v_out=rows[2][s], **kw)
            else:
                api.conduit_append_kv(api.kv_desc(*c, HQ), pos[s], k[s], v[s], **kw)
        out.append(c + rows)
    assert all(torch.equal(a, b) and a.any() for a, b in zip(*out))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["whole", "adjacent", "part"])
def test_load(dtype, kind):
    _, k, v, pos, rp = data(dtype, 2)
    p = pools()
    mx = api.mx_desc(*p, HQ)
    api.conduit_append_mx(mx, pos, k, v)
    to = pos.flip(0).contiguous()
    out = []
    for call in ([slice(0, N)], pieces()):
        c = [torch.zeros(CTX, HKV, D, dtype=k.dtype, device=DEV) for _ in range(2)]
        for s in call:
            api.conduit_load_mx(mx, pos[s], api.kv_desc(*c, HQ), to[s], rope=rope(kind), rope_pos=rp[:, s].contiguous())
        out.append(c)
    assert all(torch.equal(a, b) and a.any() for a, b in zip(*out))
