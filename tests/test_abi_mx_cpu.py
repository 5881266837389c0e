"""Refusals of the rotary, append, load and 4-bit attention calls, without a GPU (every
check runs on the host before anything is launched), and self-checks of the
64-bit definitions that the GPU tests use."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from paper_2609_05821_amd import api
from tests import mx_oracle as M

pytestmark = pytest.mark.skipif(not os.path.exists(api.LIB_PATH),
                                reason="libconduit.so not built (run __graft_entry__.build())")

FAKE = 0x100000  # a 256-byte aligned non-NULL address; never dereferenced here
INV, UNS, WS = api.ERR_INVALID_ARG, api.ERR_UNSUPPORTED, api.ERR_WORKSPACE


def rope(half=64, axes=1, pairing=0, freq=0.5, axis=None, **over):
    r = api.Rope([freq] * half, axis if axis is not None else [0] * half, n_axes=axes, pairing=pairing)
    for k, v in over.items():
        setattr(r.desc, k, v)
    return r


def kv(**over):
    d = dict(k=FAKE, v=FAKE, k_stride=512, v_stride=512, n_ctx=1344, n_q_heads=28, n_kv_heads=4, head_dim=128,
             dtype=api.BF16)
    d.update(over)
    return api.KV(**d)


def rows(**over):
    d = dict(n=3, dtype=api.BF16, k=FAKE, v=FAKE, k_stride=512, v_stride=512, q=FAKE, q_out=FAKE, q_stride=3584,
             q_out_stride=3584)
    d.update(over)
    return api.Rows(**d)


def mx(**over):
    d = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, code_stride=4 * 64 * 64, scale_stride=4 * 64 * 4, n_pages=32,
             page_size=64, n_seqs=1, table_stride=16, n_ctx=1000, block_table=FAKE, n_q_heads=28, n_kv_heads=4,
             head_dim=128)
    d.update(over)
    return api.KVMX(**d)


def err():
    return api.lib().conduit_last_error().decode()


def rotary(x=FAKE, xs=3584, n=5, heads=28, d=128, dtype=api.BF16, r=None, pos=FAKE, ps=5, inverse=0, out=FAKE * 2,
           os_=3584, no_rope=False):
    r = r or rope()
    return api.lib().conduit_rotary(x, xs, n, heads, d, dtype, None if no_rope else ctypes.byref(r.desc), pos, ps,
                                    inverse, out, os_, None)


@pytest.mark.parametrize("case,status", [
    (dict(x=0), INV), (dict(x=FAKE + 8), INV), (dict(out=0), INV), (dict(out=FAKE + 4), INV), (dict(xs=3583), INV),
    (dict(xs=3588), INV), (dict(os_=3500), INV), (dict(xs=1 << 24), UNS), (dict(n=-1), INV), (dict(heads=0), INV),
    (dict(d=4), UNS), (dict(d=100), UNS), (dict(d=264), UNS), (dict(dtype=2), INV), (dict(inverse=2), INV),
    (dict(no_rope=True), INV), (dict(pos=0), INV), (dict(pos=FAKE + 2), INV), (dict(out=FAKE, os_=3592), INV),
    (dict(r=rope(rot_dim=130)), INV), (dict(r=rope(rot_dim=63)), INV), (dict(r=rope(rot_dim=0)), INV),
    (dict(r=rope(n_axes=0)), INV), (dict(r=rope(n_axes=5)), INV), (dict(r=rope(pairing=2)), INV),
    (dict(r=rope(axes=2), ps=4), INV), (dict(r=rope(freq=float("nan"))), INV), (dict(r=rope(freq=float("inf"))), INV),
    (dict(r=rope(freq=1025.0)), INV), (dict(n=(1 << 31) - 1, heads=1, xs=128, os_=128, ps=1 << 31), UNS),
    (dict(n=76700000, ps=1 << 31), UNS), (dict(r=rope(axes=2, axis=[2] * 64)), INV),
    (dict(r=rope(axes=2, axis=[-1] * 64)), INV), (dict(r=rope(inv_freq=None)), INV)])
def test_rotary_rejects(case, status):
    assert rotary(**case) == status
    assert err() != ""


def append(k=None, r=None, pos=FAKE, ro=None, rp=FAKE, ps=3):
    k, r = k or kv(), r or rows()
    return api.lib().conduit_append_kv(ctypes.byref(k), ctypes.byref(r), pos,
                                       None if ro is None else ctypes.byref(ro.desc), rp, ps, None)


ROW_CASES = [
    (dict(k=0), INV), (dict(v=FAKE + 8), INV), (dict(k_stride=508), INV), (dict(v_stride=516), INV),
    (dict(k_stride=1 << 24), UNS), (dict(n=-3), INV), (dict(q_out=0), INV), (dict(q=0), INV), (dict(q=FAKE + 2), INV),
    (dict(n=(1 << 31) - 1), UNS), (dict(n=67200000), UNS), (dict(q_stride=3580), INV), (dict(q_out_stride=3585), INV), (dict(q_out_stride=3592), INV)]


@pytest.mark.parametrize("case,status", ROW_CASES + [(dict(dtype=api.F32), INV)])
def test_append_kv_rejects_rows(case, status):
    assert append(r=rows(**case)) == status
    assert err() != ""


@pytest.mark.parametrize("case,status", [
    (dict(k=kv(head_dim=96, k_stride=384, v_stride=384)), UNS), (dict(k=kv(n_ctx=0)), INV), (dict(pos=0), INV),
    (dict(pos=FAKE + 1), INV), (dict(ro=rope(4)), UNS), (dict(ro=rope(65)), INV), (dict(ro=rope(), rp=0), INV),
    (dict(ro=rope(axes=3), ps=2), INV)])
def test_append_kv_rejects(case, status):
    assert append(**case) == status
    assert err() != ""


MX_CASES = [
    (dict(k=0), INV), (dict(v=0), INV), (dict(k_scale=0), INV), (dict(v_scale=FAKE + 8), INV), (dict(n_pages=0), INV),
    (dict(page_size=32), UNS), (dict(page_size=96), INV), (dict(page_size=0), INV), (dict(page_size=1 << 21), UNS),
    (dict(n_seqs=0), INV), (dict(table_stride=0), INV), (dict(n_ctx=0), INV), (dict(n_ctx=1025), INV),
    (dict(code_stride=16383), INV), (dict(code_stride=16392), INV), (dict(scale_stride=1008), INV),
    (dict(scale_stride=1032), INV), (dict(block_table=FAKE + 2), INV), (dict(n_q_heads=30), INV),
    (dict(n_kv_heads=0), INV), (dict(head_dim=96), UNS), (dict(block_table=None, table_stride=33), INV),
    (dict(code_stride=1 << 59), INV), (dict(n_kv_heads=257, n_q_heads=257), UNS),
    (dict(page_size=1 << 20, table_stride=2048, n_ctx=(1 << 30) + 1, code_stride=1 << 28, scale_stride=1 << 24), UNS)]


def calls(m, n=3):
    L = api.lib()
    r, k = rows(n=n), kv()
    return {
        "append": L.conduit_append_mx(ctypes.byref(m), ctypes.byref(r), FAKE, None, None, 0, None, None, None),
        "load": L.conduit_load_mx(ctypes.byref(m), FAKE, n, ctypes.byref(k), FAKE, None, None, 0, None),
        "attn": L.conduit_attn_mx(ctypes.byref(m), FAKE, api.BF16, FAKE, n, 0.1, FAKE, None, FAKE, 1 << 30, None)}


@pytest.mark.parametrize("case,status", MX_CASES)
def test_cache_descriptor_rejected_by_every_call(case, status):
    assert set(calls(mx(**case)).values()) == {status}
    assert err() != ""


def test_rows_that_do_not_fit_the_sequences():
    assert set(calls(mx(n_seqs=2), n=3).values()) == {INV}
    assert set(calls(mx(), n=-1).values()) == {INV}


@pytest.mark.parametrize("case,status", ROW_CASES + [(dict(dtype=5), INV)])
def test_append_mx_rejects_rows(case, status):
    m, r = mx(), rows(**case)
    assert api.lib().conduit_append_mx(ctypes.byref(m), ctypes.byref(r), FAKE, None, None, 0, None, None, None) == status


def test_append_mx_and_load_reject():
    L, m, r, k, ro = api.lib(), mx(), rows(), kv(), rope()
    b = ctypes.byref
    assert L.conduit_append_mx(b(m), b(r), 0, None, None, 0, None, None, None) == INV
    assert L.conduit_append_mx(b(m), b(r), FAKE, b(ro.desc), None, 3, None, None, None) == INV
    assert L.conduit_append_mx(b(m), b(r), FAKE, None, None, 0, FAKE + 8, None, None) == INV
    assert L.conduit_append_mx(b(m), b(r), FAKE, None, None, 0, None, FAKE + 4, None) == INV
    assert L.conduit_append_mx(b(m), b(r), FAKE, b(rope(20).desc), FAKE, 3, None, None, None) == UNS
    assert L.conduit_load_mx(b(m), 0, 3, b(k), FAKE, None, None, 0, None) == INV
    assert L.conduit_load_mx(b(m), FAKE, 3, b(k), FAKE + 1, None, None, 0, None) == INV
    assert L.conduit_load_mx(b(m), FAKE, 3, b(k), FAKE, b(ro.desc), None, 3, None) == INV
    assert L.conduit_load_mx(b(m), FAKE, 1 << 29, b(k), FAKE, None, None, 0, None) == UNS
    other = kv(n_kv_heads=2)
    assert L.conduit_load_mx(b(m), FAKE, 3, b(other), FAKE, None, None, 0, None) == INV
    other = kv(head_dim=64)
    assert L.conduit_load_mx(b(m), FAKE, 3, b(other), FAKE, None, None, 0, None) == INV


def attn(m=None, q=FAKE, dtype=api.BF16, pos=FAKE, n=3, scale=0.1, o=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30):
    m = m or mx()
    return api.lib().conduit_attn_mx(ctypes.byref(m), q, dtype, pos, n, scale, o, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("case,status", [
    (dict(q=0), INV), (dict(q=FAKE + 8), INV), (dict(dtype=3), INV), (dict(pos=0), INV), (dict(pos=FAKE + 2), INV),
    (dict(scale=0.0), INV), (dict(scale=-1.0), INV), (dict(scale=math.inf), INV), (dict(scale=math.nan), INV),
    (dict(o=0), INV), (dict(o=FAKE + 4), INV), (dict(lse=FAKE + 2), INV), (dict(n=600000), UNS),
    (dict(m=mx(n_ctx=65536, table_stride=1024), ws_bytes=64), WS),
    (dict(m=mx(n_ctx=65536, table_stride=1024), ws=FAKE + 16), INV), (dict(m=mx(n_ctx=65536, table_stride=1024), ws=0), INV)])
def test_attn_rejects(case, status):
    assert attn(**case) == status
    assert err() != ""


def test_workspace_query():
    L = api.lib()
    q = lambda m, n, dt=api.BF16: L.conduit_attn_mx_workspace_bytes(ctypes.byref(m), n, dt)
    assert q(mx(n_ctx=65536, table_stride=1024), 3) > 0
    assert q(mx(n_ctx=100), 3) == 0                               # one workgroup per block: nothing to merge
    assert q(mx(), 0) == 0 and q(mx(n_seqs=2), 3) == 0 and q(mx(head_dim=96), 3) == 0
    assert L.conduit_attn_mx_workspace_bytes(None, 3, api.BF16) == 0


def test_no_rows_succeed_without_a_device():
    L, m, k, b = api.lib(), mx(), kv(), ctypes.byref
    none = rows(n=0, k=0, v=0, q=0, q_out=0)
    assert rotary(n=0, x=0, out=0) == api.OK
    assert L.conduit_append_kv(b(k), b(none), None, None, None, 0, None) == api.OK
    assert L.conduit_append_mx(b(m), b(none), None, None, None, 0, None, None, None) == api.OK
    assert L.conduit_load_mx(b(m), None, 0, b(k), None, None, None, 0, None) == api.OK
    assert attn(n=0, q=0, pos=0, o=0, ws=0, ws_bytes=0) == api.OK


def refused(fn, *a, **kw):
    with pytest.raises(api.ConduitError) as e:
        fn(*a, **kw)
    assert e.value.status in (INV, UNS)


def test_binding_rejects_tensors():
    x = torch.zeros(4, 2, 64)
    r = api.Rope([0.1] * 32)
    p = torch.zeros(4, dtype=torch.int32)
    refused(api.conduit_rotary, x, r, p, torch.zeros(4, 2, 64))                  # not on the GPU
    refused(api.conduit_rotary, x, r, p.long(), x)
    refused(api.conduit_rotary, x, r, p[:3], x)
    refused(api.conduit_rotary, x, r, None, x)
    refused(api.conduit_rotary, x.transpose(1, 2), r, p, x.transpose(1, 2))
    refused(api.conduit_rotary, x.half(), r, p, x.half())
    refused(api.conduit_rotary, x, r, p, x[:3])
    refused(api.Rope, [0.1] * 4, [0] * 3)
    refused(api.Rope, [[0.1] * 4])
    pools = [torch.zeros(4, 2, 64, b, dtype=torch.uint8) for b in (32, 32, 2, 2)]
    m = api.mx_desc(*pools, 4)
    assert m.n_ctx == 256 and m.table_stride == 4 and m.head_dim == 64
    refused(api.mx_desc, pools[0], pools[1][:3], pools[2], pools[3], 4)
    refused(api.mx_desc, pools[0], pools[1], pools[2], pools[3][..., :1], 4)
    refused(api.mx_desc, pools[0].to(torch.int32), *pools[1:], 4)
    refused(api.mx_desc, pools[0].transpose(1, 2), *pools[1:], 4)
    refused(api.mx_desc, *pools, 4, 128, torch.zeros(2, 2))
    refused(api.mx_desc, *pools, 4, 128, torch.zeros(4, dtype=torch.int32))
    refused(api.conduit_append_mx, m, p, x, x[:3])
    refused(api.conduit_append_mx, m, p, x, x.to(torch.bfloat16))
    refused(api.conduit_append_mx, m, p, x, x, q=torch.zeros(4, 4, 64))
    refused(api.conduit_append_mx, m, p, x, x, q=torch.zeros(4, 3, 64), q_out=torch.zeros(4, 3, 64))
    refused(api.conduit_append_mx, m, p[:2], x, x)
    refused(api.conduit_append_mx, m, p, x, x, k_out=torch.zeros(4, 2, 32))
    refused(api.conduit_append_mx, m, p, x, x, rope=r)
    refused(api.conduit_append_mx, m, p, torch.zeros(4, 1, 64), torch.zeros(4, 1, 64))
    q = torch.zeros(4, 4, 64)
    refused(api.conduit_attn_mx, m, q, p, torch.zeros(4, 4, 64))
    refused(api.conduit_attn_mx, m, q[:, :2], p, q[:, :2])
    refused(api.conduit_attn_mx, m, q, p, q.to(torch.bfloat16))
    refused(api.conduit_attn_mx, m, q, p.to(torch.int64), q)
    refused(api.conduit_attn_mx, m, q, p, q, lse_out=torch.zeros(4, 5))
    refused(api.conduit_load_mx, m, p, kv(), p[:2])


# ---------------------------------------------------------------------------
# The 64-bit definitions themselves
# ---------------------------------------------------------------------------

def test_turn_is_a_rotation():
    x = torch.randn(6, 2, 16, generator=torch.Generator().manual_seed(0), dtype=torch.float64)
    pos = torch.randint(-99, 99, (2, 6), generator=torch.Generator().manual_seed(1))
    for adj in (False, True):
        y = M.turned(x, [1.0, 0.3, 0.1, 0.01], [0, 1, 0, 1], pos, adj)
        assert torch.equal(y[..., 8:], x[..., 8:])
        assert torch.allclose(y.pow(2).sum(-1), x.pow(2).sum(-1))
        assert torch.allclose(M.turned(y, [1.0, 0.3, 0.1, 0.01], [0, 1, 0, 1], pos, adj, inverse=True), x)
    y = M.turned(torch.tensor([[[1.0, 0.0]]]), [math.pi / 2], None, torch.tensor([[1]]))
    assert torch.allclose(y, torch.tensor([[[0.0, 1.0]]], dtype=torch.float64), atol=1e-7)


def test_packing_by_hand():
    x = torch.zeros(1, 1, 32)
    x[0, 0, :9] = torch.tensor([6.0, -6.0, 0.25, 0.75, 2.5, -3.5, 5.0, 5.1, -0.2])
    c, s = M.pack(x)
    assert s.item() == 127
    assert torch.equal(M.held(c, s)[0, 0, :9], torch.tensor([6.0, -6.0, 0.0, 1.0, 2.0, -4.0, 4.0, 6.0, -0.0],
                                                            dtype=torch.float64))
    x[0, 0, 0] = 6.001                                        # the next scale: nothing saturates
    c, s = M.pack(x)
    assert s.item() == 128 and M.held(c, s)[0, 0, 0] == 6.0
    c, s = M.pack(torch.zeros(1, 1, 32))
    assert s.item() == 2 and not c.any()
    kc, ks, vc, vs = M.pack_rows(torch.full((1, 1, 64), np.inf), torch.ones(1, 1, 64))
    assert (ks == 255).all() and (vs == 2).all() and not kc.any() and not vc.any()


def test_packing_is_within_half_a_step():
    x = torch.randn(50, 2, 64, generator=torch.Generator().manual_seed(2)) * 3
    c, s = M.pack(x)
    h = M.held(c, s)
    top = x.double().abs().unflatten(-1, (-1, 32)).amax(-1).repeat_interleave(32, -1)
    # a block's largest value lies in (3, 6] units: half a step is at most 1 unit, a third of it
    assert ((h - x.double()).abs() <= top / 3).all()
    # held values pack to themselves (a block whose largest became 3 units takes the next smaller scale,
    # in which all of its values have codes too)
    c2, s2 = M.pack(h)
    assert torch.equal(M.held(c2, s2), h) and (s2 <= s).all()


def test_attention_by_hand():
    k = torch.tensor([[[0.0]], [[math.log(3.0)]]], dtype=torch.float64)
    v = torch.tensor([[[2.0]], [[6.0]]], dtype=torch.float64)
    o, lse, _, _ = M.attention(torch.ones(3, 2, 1), k, v, torch.tensor([0, 1, -1]), scale=1.0)
    assert torch.allclose(o[:, 0, 0], torch.tensor([2.0, 5.0, 0.0], dtype=torch.float64))
    assert torch.allclose(lse[:2, 1], torch.tensor([0.0, math.log(4.0)], dtype=torch.float64))
    assert lse[2, 0] == -math.inf


@pytest.mark.parametrize("n", [1, 5])
def test_positions_that_the_axes_share_are_refused(n):
    """An expanded tensor holds one row for all axes; the call would read n per axis."""
    x = torch.zeros(n, 2, 64)
    with pytest.raises(api.ConduitError, match="rope_pos"):
        api.conduit_rotary(x, api.Rope([0.5] * 32, [0, 1] * 16), torch.zeros(1, n, dtype=torch.int32).expand(2, n), x)


def test_launch_sizes_end_below_32_bits():
    """2^32 threads do not fit a launch: refused before, not by it."""
    n = 1 << 23
    assert rotary(n=n, heads=32, xs=4096, os_=4096, ps=n) == UNS          # 2^28 heads of 128 dims
    assert rotary(n=n + 1, heads=256, d=8, xs=2048, os_=2048, ps=n + 1, r=rope(half=4)) == UNS
    big = mx(n_seqs=1 << 20, n_q_heads=16, n_kv_heads=16, code_stride=16 * 64 * 64, scale_stride=16 * 64 * 4)
    L = api.lib()
    assert L.conduit_attn_mx_workspace_bytes(ctypes.byref(big), 1 << 20, api.BF16) == 0
    assert L.conduit_attn_mx(ctypes.byref(big), FAKE, api.BF16, FAKE, 1 << 20, 0.1, FAKE, None, None, 0, None) == UNS
    # many blocks of 32 pairs: a workgroup per block, no merge of more than 2^24 pairs
    wide = mx(n_seqs=2047, n_q_heads=240 * 33, n_kv_heads=240, head_dim=64, n_ctx=1024 * 1024, table_stride=16384)
    assert L.conduit_attn_mx_workspace_bytes(ctypes.byref(wide), 2047, api.F32) == 0
