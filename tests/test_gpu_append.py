"""Appends to caches of 16, 32 and 4 bits and loads from the 4-bit cache
(conduit_append_kv, conduit_append_mx, conduit_load_mx): bit for bit against
the turn and the packing in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_05821_amd import api
from tests import mx_oracle as M
from tests.gpu_helpers import DEV, bits
from tests.test_gpu_rotary import DT, rope_of

pytestmark = pytest.mark.gpu


def new_rows(n, hq, hkv, d, dtype, seed):
    """q, k, v slices of one fused buffer."""
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(n, hq + 2 * hkv, d, generator=g).to(DT[dtype]).to(DEV)
    return qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]


def turned(x, rope, pos):
    if rope is None:
        return x.clone()
    out = torch.empty(x.shape, dtype=x.dtype, device=DEV)
    api.conduit_rotary(x, rope, pos, out)
    return out


def random_pools(n_pages, hkv, page, d, seed, pad=0):
    """Pools of random bytes, pages `pad` bytes (codes) further apart than dense."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    out = []
    for b in (d // 2, d // 2, d // 32, d // 32):
        dense = hkv * page * b
        buf = torch.randint(0, 256, (n_pages * (dense + pad),), generator=g, device=DEV, dtype=torch.uint8)
        out.append(buf.as_strided((n_pages, hkv, page, b), (dense + pad, page * b, b, 1)))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hq,hkv,d,rot,axes,pairing,page", [
    (1, 28, 4, 128, 128, 3, 0, 64), (1, 8, 8, 64, 64, 1, 0, 0), (77, 6, 2, 64, 32, 2, 0, 64),
    (300, 7, 1, 128, 128, 3, 1, 128), (2100, 4, 4, 128, 16, 4, 0, 0), (65, 5, 5, 64, 0, 1, 0, 256)])
def test_append_kv(dtype, n, hq, hkv, d, rot, axes, pairing, page):
    g = torch.Generator().manual_seed(n)
    n_ctx = n + 131
    q, k, v = new_rows(n, hq, hkv, d, dtype, n + d)
    rope = rope_of(rot // 2, axes, pairing) if rot else None
    rp = torch.randint(0, 9000, (axes, n), generator=g, dtype=torch.int32).to(DEV) if rot else None
    pos = torch.randperm(n_ctx, generator=g)[:n].to(torch.int32)
    if n > 3:
        pos[1], pos[n // 2], pos[-1] = -1, n_ctx, 2 ** 31 - 1            # left out
    rows = n_ctx if not page else -(-n_ctx // page) * page
    ck, cv = (torch.randn(rows, hkv, d, generator=g).to(DT[dtype]).to(DEV) for _ in range(2))
    if page:
        table = torch.randperm(rows // page, generator=g).to(torch.int32)
        tab = table.to(DEV)  # the descriptor holds its address only
        kv = api.kv_desc_paged(ck.view(-1, page, hkv, d), cv.view(-1, page, hkv, d), tab, n_ctx, hq)
    else:
        kv = api.kv_desc(ck, cv, hq)
    wk, wv = ck.clone(), cv.clone()
    live = (pos >= 0) & (pos < n_ctx)
    p = pos[live].long()
    at = (table[p // page].long() * page + p % page if page else p).to(DEV)
    wk[at] = turned(k, rope, rp)[live.to(DEV)]
    wv[at] = v[live.to(DEV)]
    q_out = torch.full((n, hq, d), 7.0, dtype=q.dtype, device=DEV)
    api.conduit_append_kv(kv, pos.to(DEV), k, v, rope=rope, rope_pos=rp, q=q, q_out=q_out)
    assert torch.equal(ck, wk) and torch.equal(cv, wv)
    assert torch.equal(q_out, turned(q, rope, rp))
    # without queries, and into the same rows again
    api.conduit_append_kv(kv, pos.to(DEV), k, v, rope=rope, rope_pos=rp)
    assert torch.equal(ck, wk) and torch.equal(cv, wv)


def test_append_queries_in_place_and_values_bitwise():
    """q_out may be q; values are copied as they are, NaN payloads included."""
    n, hq, hkv, d = 9, 4, 2, 64
    q, k, v = new_rows(n, hq, hkv, d, "bf16", 1)
    v.copy_(torch.randint(-2 ** 15, 2 ** 15, (n, hkv, d), device=DEV, dtype=torch.int16).view(torch.bfloat16))
    rope, rp = rope_of(32, 1), torch.arange(n, dtype=torch.int32, device=DEV)
    want = turned(q, rope, rp)
    ck, cv = (torch.zeros(n, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    api.conduit_append_kv(api.kv_desc(ck, cv, hq), rp, k, v, rope=rope, rope_pos=rp, q=q, q_out=q)
    assert torch.equal(q, want)
    np.testing.assert_array_equal(bits(cv), bits(v))


def test_bad_pages_stay_in_the_pool():
    """Table entries outside the pool are clamped: nothing around the pool changes."""
    page, hkv, d = 64, 2, 64
    buf = torch.full((4, page, hkv, d), 3.0, device=DEV)
    vbuf = buf.clone()
    table = torch.tensor([-7, 10 ** 9], dtype=torch.int32, device=DEV)
    kv = api.kv_desc_paged(buf[1:3], vbuf[1:3], table, 128, 2)
    k = torch.randn(128, hkv, d, device=DEV)
    api.conduit_append_kv(kv, torch.arange(128, dtype=torch.int32, device=DEV), k, k)
    assert (buf[0] == 3).all() and (buf[3] == 3).all() and (vbuf[0] == 3).all() and (vbuf[3] == 3).all()
    pools = random_pools(4, hkv, page, d, 5)
    before = [p.clone() for p in pools]
    mx = api.mx_desc(*(p[1:3] for p in pools), 2, 128, table[None])
    api.conduit_append_mx(mx, torch.arange(128, dtype=torch.int32, device=DEV), k, k)
    for p, b in zip(pools, before):
        assert torch.equal(p[0], b[0]) and torch.equal(p[3], b[3])


def hard_values(n, hkv, d, dtype, seed):
    """Keys or values on the borders of codes and scales, zeros of both signs, denormal
    and huge blocks."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, hkv, d // 32, 32, generator=g)
    ties = torch.tensor([0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 6.5, 7.0, 7.5])
    pick = ties[torch.randint(0, len(ties), x.shape, generator=g)] * torch.where(x < 0, -1.0, 1.0)
    kind = torch.randint(0, 8, x.shape[:3], generator=g)[..., None]
    x = torch.where(kind < 3, pick, x)
    x = x * torch.pow(2.0, torch.randint(-9, 10, x.shape[:3], generator=g).float())[..., None]
    x = torch.where(kind == 5, x * 0.0, x)                                    # zeros of both signs
    x = torch.where(kind == 6, x * 2.0 ** -126 * 2.0 ** -6, x)                # denormal
    x = torch.where(kind == 7, (x * 2.0 ** 120).clamp(-3.3e38, 3.3e38), x)    # up to the largest
    return x.flatten(-2).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,rows,hq,hkv,d,page,pad", [(1, 1, 4, 4, 128, 64, 0), (1, 700, 2, 1, 64, 64, 16),
                                                           (5, 3, 8, 2, 128, 128, 0), (64, 1, 28, 4, 128, 64, 32),
                                                           (3, 40, 6, 6, 64, 256, 0)])
def test_append_mx_packs(dtype, n_seqs, rows, hq, hkv, d, page, pad):
    n = n_seqs * rows
    k, v = hard_values(n, hkv, d, dtype, n), hard_values(n, hkv, d, dtype, n + 1)
    if n > 2:
        k[0, 0, 3], v[1, hkv - 1, d - 1], k[2, 0, 0] = np.inf, np.nan, -np.inf
    g = torch.Generator().manual_seed(n)
    ctx = rows + 200
    per = -(-ctx // page)
    table = torch.randperm(n_seqs * per + 2, generator=g)[:n_seqs * per].to(torch.int32).view(n_seqs, per)
    pools = random_pools(n_seqs * per + 2, hkv, page, d, n, pad)
    mx = api.mx_desc(*pools, hq, ctx, table.to(DEV))
    pos = torch.stack([torch.randperm(ctx, generator=g)[:rows] for _ in range(n_seqs)]).flatten().to(torch.int32)
    if n > 3:
        pos[3], pos[n - 1] = -1, ctx
    want = [p.cpu().clone() for p in pools]
    kc, ks, vc, vs = M.pack_rows(k, v)
    live = (pos >= 0) & (pos < ctx)
    seq = torch.arange(n) // rows
    pg, sl = table[seq[live], pos[live].long() // page].long(), pos[live].long() % page
    for w, x in zip(want, (kc, vc, ks, vs)):
        w[pg, :, sl] = x[live]
    k_out, v_out = (torch.empty(n, hkv, d, dtype=DT[dtype], device=DEV) for _ in range(2))
    api.conduit_append_mx(mx, pos.to(DEV), k.to(DEV), v.to(DEV), k_out=k_out, v_out=v_out)
    for p, w in zip(pools, want):
        assert torch.equal(p.cpu(), w)
    for got, c, s in ((k_out, kc, ks), (v_out, vc, vs)):
        h = M.held(c, s)
        assert torch.equal(got.cpu().isnan(), h.isnan())
        assert torch.equal(got.cpu().double().nan_to_num(0.0), h.nan_to_num(0.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,pairing", [(128, 128, 0), (64, 64, 1), (128, 32, 0)])
def test_append_mx_turns_like_the_wide_cache(dtype, d, rot, pairing):
    """The 4-bit cache holds the packed rows of what the 16/32-bit append holds, and
    bits agree with a turn in 64 bits."""
    n, hq, hkv, page = 1030, 6, 3, 64
    q, k, v = new_rows(n, hq, hkv, d, dtype, d)
    rope = rope_of(rot // 2, 3, pairing)
    rp = torch.randint(0, 2 ** 20, (3, n), generator=torch.Generator().manual_seed(2), dtype=torch.int32).to(DEV)
    pools = random_pools(17, hkv, page, d, 3)
    mx = api.mx_desc(*pools, hq)
    pos = torch.arange(n, dtype=torch.int32, device=DEV) + 5
    q_out = torch.empty(n, hq, d, dtype=q.dtype, device=DEV)
    api.conduit_append_mx(mx, pos, k, v, rope=rope, rope_pos=rp, q=q, q_out=q_out)
    assert torch.equal(q_out, turned(q, rope, rp))
    exact = M.rounded(M.turned(k.cpu(), rope.inv_freq, rope.axis, rp.cpu(), pairing == 1), DT[dtype])
    for rows in (turned(k, rope, rp).cpu(), exact):
        kc, ks, vc, vs = M.pack_rows(rows, v.cpu())
        table = torch.arange(17)[None]
        zero = torch.zeros(n, dtype=torch.long)
        for p, w in zip(pools, (kc, vc, ks, vs)):
            assert torch.equal(M.gather(p.cpu(), table, zero, pos.cpu().long(), page), w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot,pairing", [(128, 0), (64, 0), (128, 1)])
def test_append_mx_turns_no_infinity_into_a_number(dtype, rot, pairing):
    """Infinities and NaN among keys that turn (by nothing, by a quarter, by any angle)
    and values: NaN keys, zero values; the other heads as without them."""
    n, hkv, page, d = 64, 3, 64, 128
    _, k, v = new_rows(n, hkv, hkv, d, dtype, 4)
    bad = torch.zeros(n, hkv, dtype=torch.bool)
    for t, row, h, dim, value in ((k, 0, 0, 0, math.inf), (k, 1, 1, 63, -math.inf), (v, 2, 2, 64, math.nan),
                                  (k, 3, 0, 127, math.inf), (k, 9, 1, 40, math.inf), (k, 9, 1, 104, math.inf),
                                  (v, 20, 2, 5, -math.inf), (k, 21, 0, 1, math.nan)):
        t[row, h, dim] = value
        bad[row, h] = True
    inv = np.full(rot // 2, 1.0, np.float32)
    rope = api.Rope(inv, np.zeros(rot // 2, np.int32), n_axes=1, pairing=pairing)
    rp = torch.arange(n, dtype=torch.int32, device=DEV)[None].contiguous()
    rp[0, 3] = 0
    pools = random_pools(1, hkv, page, d, 5)
    mx = api.mx_desc(*pools, hkv)
    api.conduit_append_mx(mx, torch.arange(n, dtype=torch.int32, device=DEV), k, v, rope=rope, rope_pos=rp)
    kc, vc, ks, vs = (p.cpu()[0].transpose(0, 1) for p in pools)          # [n, hkv, bytes]
    assert (ks[bad] == 255).all() and (kc[bad] == 0).all() and (vc[bad] == 0).all()
    assert (ks[~bad] <= 252).all() and (vs <= 252).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hkv,d,rot,pairing,page,paged", [(1, 1, 64, 64, 0, 64, False), (333, 4, 128, 128, 0, 64, True),
                                                            (1025, 2, 64, 32, 0, 128, False), (65, 3, 128, 128, 1, 64, True),
                                                            (200, 2, 128, 0, 0, 64, False)])
def test_load_mx(dtype, n, hkv, d, rot, pairing, page, paged):
    g = torch.Generator().manual_seed(n)
    ctx = n + 70
    n_pages = -(-ctx // page)
    pools = random_pools(n_pages, hkv, page, d, n)
    for p in pools[2:]:
        p.copy_((p % 60) + 100)                                               # scales of ordinary size
    pools[2][0, 0, 1] = 255                                                   # a NaN key
    table = torch.randperm(n_pages, generator=g).to(torch.int32)[None]
    mx = api.mx_desc(*pools, hkv, ctx, table.to(DEV))
    src = torch.randperm(ctx, generator=g)[:n].to(torch.int32)
    n_dst = n + 40
    dst = torch.randperm(n_dst, generator=g)[:n].to(torch.int32)
    if n > 5:
        src[1], src[2], dst[3], dst[4] = -1, ctx, -3, n_dst
    rope = rope_of(rot // 2, 2, pairing) if rot else None
    rp = torch.randint(-5000, 5000, (2, n), generator=g, dtype=torch.int32).to(DEV) if rot else None
    rows = -(-n_dst // 64) * 64
    ck, cv = (torch.randn(rows, hkv, d, generator=g).to(DT[dtype]).to(DEV) for _ in range(2))
    if paged:
        pt = torch.randperm(rows // 64, generator=g).to(torch.int32)
        tab = pt.to(DEV)  # the descriptor holds its address only
        kv = api.kv_desc_paged(ck.view(-1, 64, hkv, d), cv.view(-1, 64, hkv, d), tab, n_dst, hkv)
    else:
        kv = api.kv_desc(ck[:n_dst], cv[:n_dst], hkv)
    live = (src >= 0) & (src < ctx) & (dst >= 0) & (dst < n_dst)
    s, t = src[live].long(), dst[live].long()
    at = pt[t // 64].long() * 64 + t % 64 if paged else t
    zero = torch.zeros(len(s), dtype=torch.long)
    kk = M.held(M.gather(pools[0].cpu(), table, zero, s, page), M.gather(pools[2].cpu(), table, zero, s, page))
    vv = M.held(M.gather(pools[1].cpu(), table, zero, s, page), M.gather(pools[3].cpu(), table, zero, s, page))
    if rope:
        kk = M.turned(kk, rope.inv_freq, rope.axis, rp.cpu()[:, live], pairing == 1)
    wk, wv = ck.cpu().clone(), cv.cpu().clone()
    wk[at], wv[at] = M.rounded(kk, DT[dtype]), M.rounded(vv, DT[dtype])
    api.conduit_load_mx(mx, src.to(DEV), kv, dst.to(DEV), rope=rope, rope_pos=rp)
    assert torch.equal(ck.cpu().isnan(), wk.isnan())
    assert torch.equal(ck.cpu().nan_to_num(0.0), wk.nan_to_num(0.0)) and torch.equal(cv.cpu(), wv)


def test_no_rows():
    pools = random_pools(2, 2, 64, 64, 1)
    before = [p.clone() for p in pools]
    mx = api.mx_desc(*pools, 2)
    e = torch.empty(0, 2, 64, device=DEV)
    i = torch.empty(0, dtype=torch.int32, device=DEV)
    ck = torch.ones(64, 2, 64, device=DEV)
    api.conduit_append_mx(mx, i, e, e)
    api.conduit_append_kv(api.kv_desc(ck, ck, 2), i, e, e)
    api.conduit_load_mx(mx, i, api.kv_desc(ck, ck, 2), i)
    assert all(torch.equal(p, b) for p, b in zip(pools, before)) and (ck == 1).all()


def test_pool_past_32_bits():
    """Pages spread over more than 4 GiB: append, load, attention on the last page."""
    hkv, page, d, n_pages = 1, 64, 128, 70
    stride = 1 << 26
    pools = []
    for b in (d // 2, d // 2, d // 32, d // 32):
        buf = torch.zeros(n_pages * stride, dtype=torch.uint8, device=DEV)
        pools.append(buf.as_strided((n_pages, hkv, page, b), (stride, page * b, b, 1)))
    mx = api.mx_desc(*pools, hkv, 64, torch.tensor([[n_pages - 1]], dtype=torch.int32, device=DEV))
    k, v = (torch.randn(64, 1, d, device=DEV).to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(64, dtype=torch.int32, device=DEV)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    api.conduit_append_mx(mx, pos, k, v, k_out=ko, v_out=vo)
    ck, cv = torch.empty_like(k), torch.empty_like(v)
    api.conduit_load_mx(mx, pos, api.kv_desc(ck, cv, 1), pos)
    assert torch.equal(ck, ko) and torch.equal(cv, vo)
    o = torch.empty(1, 1, d, device=DEV)
    api.conduit_attn_mx(mx, torch.zeros(1, 1, d, device=DEV), pos[-1:].contiguous(), o)
    mean = vo.float().double().mean(0)
    assert ((o[0].double() - mean).abs() <= 200 * 2.0 ** -24 * vo.float().double().abs().mean(0) + 1e-30).all()
