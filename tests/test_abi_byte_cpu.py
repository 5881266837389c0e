"""Refusals of the 8-bit cache's calls, without a GPU (every check runs on the host before
anything is launched), how an attention call is cut up, and self-checks of the 64-bit
definitions that the GPU tests use."""
import ctypes
import math
import os
import weakref

import pytest
import torch

from paper_2609_05821_amd import api
from tests import byte_oracle as B
from tests.test_abi_mx_cpu import FAKE, INV, ROW_CASES, UNS, WS, err, kv, refused, rope, rows
from tests.test_cache_devices_cpu import on_gpu

pytestmark = pytest.mark.skipif(not os.path.exists(api.LIB_PATH),
                                reason="libconduit.so not built (run __graft_entry__.build())")


def cache(**over):
    d = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, code_stride=4 * 64 * 128, scale_stride=4 * 64 // 16,
             n_pages=32, page_size=64, n_seqs=1, table_stride=16, n_ctx=1000, block_table=FAKE, n_q_heads=28,
             n_kv_heads=4, head_dim=128)
    d.update(over)
    return api.KVByte(**d)


CACHE_CASES = [
    (dict(k=0), INV), (dict(v=0), INV), (dict(k=FAKE + 8), INV), (dict(k_scale=0), INV), (dict(v_scale=FAKE + 2), INV),
    (dict(n_pages=0), INV), (dict(page_size=32), UNS), (dict(page_size=96), INV), (dict(page_size=0), INV),
    (dict(page_size=1 << 21), UNS), (dict(n_seqs=0), INV), (dict(table_stride=0), INV), (dict(n_ctx=0), INV),
    (dict(n_ctx=1025), INV), (dict(code_stride=32767), INV), (dict(code_stride=32776), INV),
    (dict(scale_stride=12), INV), (dict(scale_stride=18), INV), (dict(block_table=FAKE + 2), INV),
    (dict(n_q_heads=30), INV), (dict(n_kv_heads=0), INV), (dict(head_dim=96), UNS), (dict(head_dim=256), UNS),
    (dict(block_table=None, table_stride=33), INV), (dict(code_stride=1 << 59), INV),
    (dict(n_kv_heads=257, n_q_heads=257), UNS),
    (dict(page_size=1 << 20, table_stride=2048, n_ctx=(1 << 30) + 1, code_stride=1 << 29, scale_stride=1 << 18), UNS)]


def append(c=None, r=None, pos=FAKE, held=None, ro=None, rp=None, ps=0, ko=None, vo=None):
    c, r = c or cache(), r or rows()
    return api.lib().conduit_append_byte(ctypes.byref(c), ctypes.byref(r), pos, held, ro and ctypes.byref(ro.desc), rp,
                                         ps, ko, vo, None)


def load(c=None, src=FAKE, n=3, k=None, dst=FAKE, ro=None, rp=None, ps=0):
    c, k = c or cache(), k or kv()
    return api.lib().conduit_load_byte(ctypes.byref(c), src, n, ctypes.byref(k), dst, ro and ctypes.byref(ro.desc), rp,
                                       ps, None)


def attn(c=None, q=FAKE, dtype=api.BF16, pos=FAKE, n=3, scale=0.1, o=FAKE, lse=None, ws=FAKE, ws_bytes=1 << 30):
    c = c or cache()
    return api.lib().conduit_attn_byte(ctypes.byref(c), q, dtype, pos, n, scale, o, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("case,status", CACHE_CASES)
def test_cache_descriptor_rejected_by_every_call(case, status):
    for call in (append, load, attn):
        assert call(cache(**case)) == status
        assert err() != ""


def test_null_descriptors():
    L, c, r, k, b = api.lib(), cache(), rows(), kv(), ctypes.byref
    assert L.conduit_append_byte(None, b(r), FAKE, None, None, None, 0, None, None, None) == INV
    assert L.conduit_append_byte(b(c), None, FAKE, None, None, None, 0, None, None, None) == INV
    assert L.conduit_load_byte(None, FAKE, 3, b(k), FAKE, None, None, 0, None) == INV
    assert L.conduit_load_byte(b(c), FAKE, 3, None, FAKE, None, None, 0, None) == INV
    assert L.conduit_attn_byte(None, FAKE, api.BF16, FAKE, 3, 0.1, FAKE, None, FAKE, 1 << 30, None) == INV
    assert L.conduit_attn_byte_workspace_bytes(None, 3, api.BF16) == 0


def test_rows_that_do_not_fit_the_sequences():
    two = cache(n_seqs=2)
    assert append(two) == load(two) == attn(two) == INV
    assert append(r=rows(n=-1)) == load(n=-1) == attn(n=-1) == INV


@pytest.mark.parametrize("case,status", ROW_CASES + [(dict(dtype=5), INV)])
def test_append_rejects_rows(case, status):
    assert append(r=rows(**case)) == status
    assert err() != ""


@pytest.mark.parametrize("case,status", [
    (dict(pos=0), INV), (dict(pos=FAKE + 2), INV), (dict(held=FAKE + 2), INV), (dict(ro=rope(), ps=3), INV),
    (dict(ro=rope(), rp=FAKE + 2, ps=3), INV), (dict(ro=rope(axes=3), rp=FAKE, ps=2), INV),
    (dict(ro=rope(20), rp=FAKE, ps=3), UNS), (dict(ro=rope(65), rp=FAKE, ps=3), INV), (dict(ko=FAKE + 8), INV),
    (dict(vo=FAKE + 4), INV)])
def test_append_rejects(case, status):
    assert append(**case) == status
    assert err() != ""


@pytest.mark.parametrize("case,status", [
    (dict(src=0), INV), (dict(src=FAKE + 1), INV), (dict(dst=0), INV), (dict(dst=FAKE + 1), INV),
    (dict(ro=rope(), ps=3), INV), (dict(n=1 << 29), UNS), (dict(k=kv(n_kv_heads=2)), INV),
    (dict(k=kv(head_dim=64)), INV), (dict(k=kv(n_ctx=0)), INV)])
def test_load_rejects(case, status):
    assert load(**case) == status
    assert err() != ""


LONG = dict(n_ctx=65536, table_stride=1024)


@pytest.mark.parametrize("case,status", [
    (dict(q=0), INV), (dict(q=FAKE + 8), INV), (dict(dtype=3), INV), (dict(pos=0), INV), (dict(pos=FAKE + 2), INV),
    (dict(scale=0.0), INV), (dict(scale=-1.0), INV), (dict(scale=math.inf), INV), (dict(scale=math.nan), INV),
    (dict(scale=1e-40), INV), (dict(scale=3e38), INV), (dict(o=0), INV), (dict(o=FAKE + 4), INV),
    (dict(lse=FAKE + 2), INV),
    (dict(n=600000), UNS), (dict(c=cache(**LONG), ws_bytes=64), WS), (dict(c=cache(**LONG), ws=FAKE + 16), INV),
    (dict(c=cache(**LONG), ws=0), INV)])
def test_attn_rejects(case, status):
    assert attn(**case) == status
    assert err() != ""


def test_no_rows_succeed_without_a_device():
    none = rows(n=0, k=0, v=0, q=0, q_out=0)
    assert append(r=none, pos=None) == api.OK
    assert load(src=None, n=0, dst=None) == api.OK
    assert attn(n=0, q=0, pos=0, o=0, ws=0, ws_bytes=0) == api.OK


def workspace(n_seqs, r, group, d, dtype=api.BF16, ctx=2048, hkv=1):
    c = cache(code_stride=hkv * 64 * d, scale_stride=hkv * 4, n_pages=1 << 20, n_seqs=n_seqs,
              table_stride=-(-ctx // 64), n_ctx=ctx, n_q_heads=group * hkv, n_kv_heads=hkv, head_dim=d)
    return int(api.lib().conduit_attn_byte_workspace_bytes(ctypes.byref(c), n_seqs * r, dtype))


def test_workspace_query():
    assert workspace(1, 3, 7, 128, ctx=65536) > 0
    assert workspace(1, 3, 7, 128, ctx=100) == 0              # one workgroup per block: nothing to merge
    assert workspace(1, 0, 7, 128) == 0 and workspace(1, 3, 7, 96) == 0
    c = cache(n_seqs=2)
    assert api.lib().conduit_attn_byte_workspace_bytes(ctypes.byref(c), 3, api.BF16) == 0


def parts(workers, pairs, blocks, d):
    """Bytes of the list of blocks, of 65 places, and of two parts of a workgroup's pairs."""
    up = lambda x: -(-x // 256) * 256
    return up(4 * (blocks + 1)) + up(4 * 65) + up(2 * workers * pairs * 8) + up(2 * workers * pairs * d * 4)


@pytest.mark.parametrize("d,few", [(128, 64), (64, 128)])
def test_pairs_of_a_block(d, few):
    """Blocks of 16 and of 32 pairs, and of 256 beyond `few` pairs once blocks of 32 would have 2^18 keys in all."""
    waves = {128: (2, 2), 64: (4, 3)}[d]                      # workgroups of a CU with 16 and with 32 pairs
    assert workspace(1, 16, 1, d, ctx=1 << 18) == parts(256 * waves[0], 16, 1, d)
    assert workspace(1, 17, 1, d, ctx=1 << 18) == parts(256 * waves[1], 32, 1, d)
    assert workspace(1, few, 1, d, ctx=1 << 20) == parts(256 * waves[1], 32, few // 32, d)
    assert workspace(1, few + 1, 1, d, ctx=1 << 18) == parts(256, 256, 1, d)
    assert workspace(1, 512, 1, d, ctx=16384) == parts(128, 256, 2, d)        # two steps of 128 keys each at least
    assert workspace(1, 512, 1, d, ctx=16320) == parts(256 * waves[1], 32, 16, d)
    fine = parts(512, 16, 32, d) if d == 128 else parts(512, 32, 16, d)
    assert workspace(1, 512, 1, d, ctx=16384, dtype=api.F32) == fine


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("blocks", [1, 64, 65, 4096, 4097])
def test_lists_fit_a_workgroup(blocks, d):
    """256 pairs a block: four tiles of 64 keys and values of bf16, sums, and the list of blocks."""
    used = 4 * 64 * (2 * d + 24) * 2 + 64 + 4 * (blocks + 1)
    assert blocks > 4096 or used <= 160 * 1024
    assert (workspace(blocks, 300, 1, d, ctx=8192) > 0) == (2 * blocks <= 4096)
    assert (workspace(blocks, 256, 1, d, ctx=16384) > 0) == (blocks <= 4096)
    assert (workspace(blocks, 1, 8, d, ctx=8192) > 0) == (blocks <= 4096)


def test_launch_sizes_end_below_32_bits():
    big = cache(n_seqs=1 << 20, n_q_heads=16, n_kv_heads=16, code_stride=16 * 64 * 128, scale_stride=16 * 4)
    assert api.lib().conduit_attn_byte_workspace_bytes(ctypes.byref(big), 1 << 20, api.BF16) == 0
    assert attn(big, n=1 << 20, ws=None, ws_bytes=0) == UNS


# ---------------------------------------------------------------------------
# The Python entry points
# ---------------------------------------------------------------------------

def pools(make=torch.zeros, d=128, page=64):
    return [make(2, 2, page, d, dtype=torch.uint8) for _ in range(2)] + \
        [make(2, 2, page // 16, dtype=torch.uint8) for _ in range(2)]


def test_descriptor():
    p = pools()
    c = api.byte_desc(*p, 4)
    assert (c.n_ctx, c.table_stride, c.page_size, c.head_dim, c.n_kv_heads, c.n_q_heads) == (128, 2, 64, 128, 2, 4)
    assert (c.code_stride, c.scale_stride) == (2 * 64 * 128, 2 * 4)
    c = api.byte_desc(*(x.view(torch.float8_e4m3fn) for x in p[:2]), *p[2:], 4, n_seqs=2)
    assert (c.n_ctx, c.table_stride, c.n_seqs) == (64, 1, 2)
    wide = [torch.zeros(2, 3, *x.shape[1:], dtype=torch.uint8)[:, 1] for x in p]      # a layer of a larger pool
    c = api.byte_desc(*wide, 4, 100)
    assert (c.code_stride, c.scale_stride, c.n_ctx) == (3 * 2 * 64 * 128, 3 * 2 * 4, 100)
    refused(api.byte_desc, p[0], p[1][:1], p[2], p[3], 4)
    refused(api.byte_desc, p[0], p[1], p[2], p[3][..., :1], 4)
    refused(api.byte_desc, p[0].to(torch.int32), *p[1:], 4)
    refused(api.byte_desc, p[0], p[1], p[2].to(torch.int8), p[3], 4)
    refused(api.byte_desc, p[0].transpose(1, 2), *p[1:], 4)
    refused(api.byte_desc, wide[0], *p[1:], 4)                                        # two page strides
    refused(api.byte_desc, *p, 4, 128, torch.zeros(2, 2))
    refused(api.byte_desc, *p, 4, 128, torch.zeros(4, dtype=torch.int32))
    refused(api.byte_desc, *pools(page=40), 4)


def test_binding_rejects_tensors():
    c, x, p = api.byte_desc(*pools(), 4), torch.zeros(4, 2, 128), torch.zeros(4, dtype=torch.int32)
    r, q = api.Rope([0.1] * 64), torch.zeros(4, 4, 128)
    refused(api.conduit_append_byte, c, p, x, x)                                      # not on the GPU
    refused(api.conduit_append_byte, c, p, x, x[:3])
    refused(api.conduit_append_byte, c, p, x, x.to(torch.bfloat16))
    refused(api.conduit_append_byte, c, p, x.half(), x.half())
    refused(api.conduit_append_byte, c, p, x[:, :, ::2], x)
    refused(api.conduit_append_byte, c, p, x[:, :1], x[:, :1])
    refused(api.conduit_append_byte, c, p, x[0], x[0])
    refused(api.conduit_append_byte, c, p, x, x, q=q)
    refused(api.conduit_append_byte, c, p, x, x, q=q, q_out=q.to(torch.bfloat16))
    refused(api.conduit_append_byte, c, p, x, x, q=q[:, :3], q_out=q[:, :3])
    refused(api.conduit_append_byte, c, p[:2], x, x)
    refused(api.conduit_append_byte, c, p.long(), x, x)
    refused(api.conduit_append_byte, c, p, x, x, n_held=p)
    refused(api.conduit_append_byte, c, p, x, x, n_held=p[:1].long())
    refused(api.conduit_append_byte, c, p, x, x, k_out=torch.zeros(4, 2, 64))
    refused(api.conduit_append_byte, c, p, x, x, v_out=x.to(torch.bfloat16))
    refused(api.conduit_append_byte, c, p, x, x, rope=r)
    refused(api.conduit_append_byte, c, p, x, x, rope=r, rope_pos=p[:3])
    refused(api.conduit_load_byte, c, p, kv(), p[:2])
    refused(api.conduit_attn_byte, c, q, p, torch.zeros(4, 4, 128))                   # not on the GPU
    refused(api.conduit_attn_byte, c, q[:, :2], p, q[:, :2])
    refused(api.conduit_attn_byte, c, q, p, q.to(torch.bfloat16))
    refused(api.conduit_attn_byte, c, q, p.to(torch.int64), q)
    refused(api.conduit_attn_byte, c, q, p, q, lse_out=torch.zeros(4, 5))


@pytest.mark.parametrize("cpu", range(5), ids=["k", "v", "k_scale", "v_scale", "block_table"])
def test_a_pool_on_another_device_is_refused(cpu):
    p = pools(on_gpu) + [on_gpu(1, 2, dtype=torch.int32)]
    p[cpu] = torch.zeros(p[cpu].shape, dtype=p[cpu].dtype)
    with pytest.raises(api.ConduitError, match="different devices"):
        api.byte_desc(*p[:4], 4, 128, p[4])


def test_a_cache_on_another_device_than_its_rows_is_refused():
    x, pos = on_gpu(3, 2, 128), on_gpu(3, dtype=torch.int32)
    with pytest.raises(api.ConduitError, match="different devices"):
        api.conduit_append_byte(api.byte_desc(*pools(), 4), pos, x, x)
    with pytest.raises(api.ConduitError, match="different devices"):
        api.conduit_append_byte(api.byte_desc(*pools(on_gpu), 4), pos, x, torch.zeros(3, 2, 128, dtype=torch.bfloat16))
    flat = [torch.zeros(64, 2, 128, dtype=torch.bfloat16) for _ in range(2)]
    with pytest.raises(api.ConduitError, match="different devices"):
        api.conduit_load_byte(api.byte_desc(*pools(on_gpu), 4), pos, api.kv_desc(*flat, 4), pos)
    with pytest.raises(api.ConduitError, match="different devices"):
        api.conduit_attn_byte(api.byte_desc(*pools(), 4), on_gpu(3, 4, 128), pos, on_gpu(3, 4, 128))


def test_descriptors_keep_their_tensors():
    p = pools() + [torch.zeros(1, 2, dtype=torch.int32)]
    refs = [weakref.ref(t) for t in p]
    c = api.byte_desc(*p[:4], 4, 128, p[4])
    del p
    assert all(r() is not None for r in refs)
    del c
    assert all(r() is None for r in refs)


# ---------------------------------------------------------------------------
# The 64-bit definitions themselves
# ---------------------------------------------------------------------------

def test_codes_are_e4m3():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(B.decoded(torch.arange(256)).nan_to_num(999.0), want.nan_to_num(999.0))
    x = torch.randn(4000, generator=torch.Generator().manual_seed(0), dtype=torch.float64) * 60
    x = torch.cat((x, x / 2 ** 10, B.TABLE, -B.TABLE, (B.TABLE[1:] + B.TABLE[:-1]) / 2))
    x = x[x.abs() <= 448]
    assert torch.equal(B.nearest(x), x.float().to(torch.float8_e4m3fn).view(torch.uint8))
    assert B.nearest(torch.tensor([500.0, -1e9], dtype=torch.float64)).tolist() == [0x7e, 0xfe]


def test_scales_are_the_smallest():
    assert B.needed(0.0) == 10 and B.needed(448.0) == 127 and B.needed(448.001) == 128 and B.needed(3e38) == 247 - 1
    for top in (1e-30, 0.5, 1.0, 447.9, 1e20):
        s = B.needed(top)
        assert top <= 448.0 * 2.0 ** (s - 127) and (s == 10 or top > 448.0 * 2.0 ** (s - 128))


def test_a_block_by_hand():
    """Two tokens, a third with a larger value: the block's scale rises and the kept codes are rounded to it."""
    z = [torch.zeros(1, 1, 64, 4, dtype=torch.uint8), torch.zeros(1, 1, 4, dtype=torch.uint8)]
    p = B.Pools(z[0], z[0], z[1], z[1], torch.zeros(1, 1, dtype=torch.int32), 64, 64)
    x = torch.tensor([[[448.0, 1.0, 0.0, -3.0]], [[17.0, 18.0, 2 ** -9, 2 ** -10]]])
    held, _ = p.append(torch.tensor([0, 1]), x, x)
    assert held[:, 0].tolist() == [[448.0, 1.0, 0.0, -3.0], [16.0, 18.0, 2 ** -9, 0.0]]
    held, _ = p.append(torch.tensor([2]), torch.full((1, 1, 4), 900.0), x[:1])
    assert held[0, 0].tolist() == [896.0] * 4
    assert p.pool["k"][1][0, 0, 0] == 129 and p.pool["v"][1][0, 0, 0] == 127          # 900 > 896: two doublings
    k, v = p.rows(0, 3)
    assert k[1, 0].tolist() == [16.0, 18.0, 0.0, 0.0] and v[1, 0].tolist() == [16.0, 18.0, 2 ** -9, 0.0]
    held, _ = p.append(torch.tensor([3]), torch.full((1, 1, 4), math.nan), x[:1])
    assert held.isnan().all() and (p.rows(0, 4)[1][3] == 0).all()
