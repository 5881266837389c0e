"""Appends to and loads from the 8-bit cache (conduit_append_byte, conduit_load_byte): byte
for byte against the turn and the rounding in 64 bits."""
import math

import pytest
import torch

from paper_2609_05821_amd import api
from tests import byte_oracle as B
from tests import mx_oracle as M
from tests.gpu_helpers import DEV
from tests.test_gpu_append import new_rows
from tests.test_gpu_rotary import DT, rope_of

pytestmark = pytest.mark.gpu


class Cache:
    """Pools of random codes and scales on the GPU, pages `pad` bytes further apart than
    dense, with the oracle's copy."""

    def __init__(self, n_seqs, ctx, hq, hkv, d, page=64, seed=0, pad=0, spare=2, lo=115, hi=125):
        g = torch.Generator().manual_seed(seed)
        per = -(-ctx // page)
        n_pages = n_seqs * per + spare
        self.ctx, self.page, self.hkv, self.d = ctx, page, hkv, d
        self.table = torch.randperm(n_pages, generator=g)[:n_seqs * per].to(torch.int32).view(n_seqs, per)
        self.dev = []
        for inner, low, high in (((hkv, page, d), 0, 256), ((hkv, page, d), 0, 256),
                                 ((hkv, page // 16), lo, hi), ((hkv, page // 16), lo, hi)):
            dense = math.prod(inner)
            extra = pad if len(inner) == 3 else pad // 4
            buf = torch.randint(low, high, (n_pages * (dense + extra),), generator=g).to(torch.uint8)
            if len(inner) == 3:
                buf[(buf & 127) == 127] = 1                                  # no NaN to begin with
            strides = tuple(math.prod(inner[i + 1:]) for i in range(len(inner)))
            self.dev.append(buf.to(DEV).as_strided((n_pages, *inner), (dense + extra, *strides)))
        self.desc = api.byte_desc(*self.dev, hq, ctx, self.table.to(DEV))
        k, v, ks, vs = (t.cpu().contiguous() for t in self.dev)
        self.want = B.Pools(k, v, ks, vs, self.table, page, ctx)

    def check(self):
        """Every byte is the oracle's (any NaN code for another)."""
        got = [t.cpu() for t in self.dev]
        want = [self.want.pool["k"][0], self.want.pool["v"][0], self.want.pool["k"][1], self.want.pool["v"][1]]
        assert torch.equal(got[2], want[2]) and torch.equal(got[3], want[3]), "scale bytes"
        for g, w in zip(got[:2], want[:2]):
            nan = ((g & 127) == 127) & ((w & 127) == 127)
            same = (g == w) | nan
            assert same.all(), f"{(~same).sum()} code bytes differ"


def append(c, pos, k, v, n_held=None, rope=None, rp=None, held=True, **kw):
    """The call and the oracle on the same rows; returns the rows as held."""
    ko, vo = (torch.full(k.shape, 9.0, dtype=k.dtype, device=DEV) for _ in range(2)) if held else (None, None)
    api.conduit_append_byte(c.desc, pos.to(DEV), k, v, n_held=None if n_held is None else n_held.to(DEV), rope=rope,
                            rope_pos=rp, k_out=ko, v_out=vo, **kw)
    kt = k.cpu()
    if rope is not None:
        kt = M.rounded(M.turned(kt, rope.inv_freq, rope.axis, rp.cpu(), rope.desc.pairing == 1), k.dtype)
    wk, wv = c.want.append(pos, kt, v.cpu(), n_held)
    c.check()
    if held:
        # a row whose position a later row of its sequence has is not written
        r, last = len(pos) // c.want.table.shape[0], {}
        for i, t in enumerate(pos.tolist()):
            if 0 <= t < c.ctx:
                last[(i // r, t)] = i
        gone = torch.tensor([0 <= t < c.ctx and last[(i // r, t)] != i for i, t in enumerate(pos.tolist())])
        for got, want in ((ko, wk), (vo, wv)):
            want[gone] = 9.0
            got, want = got.cpu().double(), want.float().to(k.dtype).double()
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))
    return wk, wv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,rot,axes,pairing,page", [
    (1, 1, 28, 4, 128, 128, 3, 0, 64), (3, 1, 8, 8, 64, 64, 1, 0, 64), (1, 77, 6, 2, 64, 32, 2, 0, 64),
    (2, 50, 7, 1, 128, 128, 3, 1, 128), (1, 130, 4, 4, 128, 16, 4, 0, 64), (5, 9, 5, 5, 64, 0, 1, 0, 256),
    (1, 40, 6, 6, 128, 64, 1, 1, 64), (1, 33, 3, 3, 64, 48, 1, 0, 64)])
def test_append(dtype, n_seqs, r, hq, hkv, d, rot, axes, pairing, page):
    """New rows behind the others, from positions that begin within a block."""
    n, ctx = n_seqs * r, r + 150
    g = torch.Generator().manual_seed(n + d)
    c = Cache(n_seqs, ctx, hq, hkv, d, page, seed=n)
    q, k, v = new_rows(n, hq, hkv, d, dtype, n)
    rope = rope_of(rot // 2, axes, pairing) if rot else None
    rp = torch.randint(0, 9000, (axes, n), generator=g, dtype=torch.int32).to(DEV) if rot else None
    start = torch.randint(0, 150, (n_seqs, 1), generator=g)
    pos = (start + torch.arange(r)).flatten().to(torch.int32)
    q_out = torch.full((n, hq, d), 7.0, dtype=q.dtype, device=DEV)
    append(c, pos, k, v, rope=rope, rp=rp, q=q, q_out=q_out)
    want = q.clone()
    if rope is not None:
        api.conduit_rotary(q, rope, rp, want)
    assert torch.equal(q_out, want)
    append(c, pos, k, v, rope=rope, rp=rp, held=False)       # the same rows once more, without queries


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 40), (25, 300), (140, 700), (300, 300)])
def test_overwritten_rows(dtype, r, ctx):
    """Rows here and there over what the sequence holds, some of it behind n_held; scales
    below, at and above what the rows need."""
    c = Cache(2, ctx, 4, 2, 128, seed=ctx, pad=64)
    g = torch.Generator().manual_seed(r)
    pos = torch.cat([torch.randperm(ctx, generator=g)[:r].sort().values for _ in range(2)]).to(torch.int32)
    _, k, v = new_rows(2 * r, 4, 2, 128, dtype, r)
    append(c, pos, k * 0.01, v, n_held=torch.tensor([ctx, ctx // 2], dtype=torch.int32))
    append(c, pos, k * 3.0, v * 20.0, n_held=torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32))
    append(c, pos, k * 40.0, v, n_held=torch.tensor([7, ctx - 3], dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_token_by_token(dtype):
    """A sequence that grows by one to four tokens a call, its scales rising on the way: what
    is held is within one step of the last scale of every token."""
    c = Cache(1, 200, 2, 2, 64, seed=3)
    g = torch.Generator().manual_seed(4)
    at, rows = 0, []
    while at < 150:
        m = int(torch.randint(1, 5, (1,), generator=g))
        _, k, v = new_rows(m, 2, 2, 64, dtype, at)
        k, v = k * (1.0 + at / 10), v * 2.0 ** (at % 7 - 3)
        append(c, torch.arange(at, at + m, dtype=torch.int32), k, v)
        rows.append((k.cpu().double(), v.cpu().double()))
        at += m
    place = [c.want.place(0, t) for t in range(at)]
    for i, (name, got) in enumerate(zip("kv", c.want.rows(0, at))):
        want = torch.cat([x[i] for x in rows])
        f = torch.stack([B.factor(c.want.pool[name][1][pg, :, sl // 16]) for pg, sl in place])[..., None]
        # half a step of 2^-3 of the value once; below the smallest normal code half a step of
        # 2^-9 of each scale on the way, of which the last is f and each is at most half the next
        assert ((got - want).abs() <= want.abs() * 2.0 ** -4 + 2.0 ** -9 * f).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_call_or_many(dtype):
    """Rows of one magnitude: a sequence appended at once and in pieces of any size has the
    same bytes (no scale rises by so much that a code becomes subnormal)."""
    n = 137
    _, k, v = new_rows(n, 2, 2, 128, dtype, 1)
    k = torch.where(k.abs() < 0.25, torch.full_like(k, 0.25), k)
    v = torch.where(v.abs() < 0.25, torch.full_like(v, 0.25), v)
    caches = [Cache(1, 300, 2, 2, 128, seed=5) for _ in range(3)]
    for c, step in zip(caches, (n, 1, 23)):
        for at in range(0, n, step):
            m = min(step, n - at)
            api.conduit_append_byte(c.desc, torch.arange(at, at + m, dtype=torch.int32, device=DEV), k[at:at + m],
                                    v[at:at + m])
    for a, b in ((0, 1), (0, 2)):
        for x, y in zip(caches[a].dev, caches[b].dev):
            assert torch.equal(x, y)


@pytest.mark.parametrize("gaps", ["front", "behind", "between", "all", "long"])
def test_rows_left_out(gaps):
    """Rows outside the cache before, behind and between the rows of a block, and more of
    them than a wave looks at once."""
    c = Cache(2, 400, 2, 2, 64, seed=6)
    live = torch.arange(21, 60)
    out = dict(front=[-1] * 70 + live.tolist(), behind=live.tolist() + [400, 2 ** 31 - 1, -2 ** 31] * 30,
               between=[x for t in live.tolist() for x in (t, -1, 405)], all=[-1] * 33,
               long=[5] + [-1] * 700 + [6, 7] + [-1] * 70 + [8, 40])[gaps]
    pos = torch.tensor([out, out[:1] + [-1] * (len(out) - 2) + out[-1:]], dtype=torch.int32).flatten()
    _, k, v = new_rows(len(pos), 2, 2, 64, "bf16", 2)
    append(c, pos, k, v)
    append(c, pos, k, v * 9, held=False, n_held=torch.tensor([30, 400], dtype=torch.int32))


@pytest.mark.parametrize("n", [511, 512, 2047, 2050, 4500, 8191, 8192, 10000])
@pytest.mark.parametrize("hkv", [1, 5])
def test_many_rows(n, hkv):
    """Either side of the number of rows from which workgroups take 16 each; first positions
    within a block; rows of several sequences in one window."""
    g = torch.Generator().manual_seed(n)
    r = n // 5 if n % 5 == 0 else n
    ctx = r + 40
    c = Cache(n // r, ctx, hkv, hkv, 64, page=256, seed=n)
    q, k, v = new_rows(n, hkv, hkv, 64, "bf16", n)
    start = torch.randint(0, 40, (n // r, 1), generator=g)
    pos = (start + torch.arange(r)).flatten().to(torch.int32)
    pos[r // 2: r // 2 + 3] = -1
    rp = torch.randint(0, 9000, (1, n), generator=g, dtype=torch.int32).to(DEV)
    rope = rope_of(32, 1, 0)
    q_out = torch.empty(n, hkv, 64, dtype=q.dtype, device=DEV)
    append(c, pos, k, v, rope=rope, rp=rp, q=q, q_out=q_out)
    want = torch.empty_like(q_out)
    api.conduit_rotary(q, rope, rp, want)
    assert torch.equal(q_out, want)


@pytest.mark.parametrize("n,ctx,hkv,d", [(900, 9000, 2, 64), (800, 1100, 6, 128), (2600, 20000, 6, 128),
                                           (4100, 6000, 5, 64), (8300, 30000, 1, 64)])
def test_scattered_rows_in_windows(n, ctx, hkv, d):
    """Windows that begin many runs, short and long ones, runs that begin in one window and end
    in the next; more heads than a workgroup takes."""
    g = torch.Generator().manual_seed(0)
    c = Cache(1, ctx, hkv, hkv, d, page=1024, seed=1)
    pos = torch.randperm(ctx, generator=g)[:n].sort().values.to(torch.int32)
    _, k, v = new_rows(n, hkv, hkv, d, "bf16", 3)
    rope, rp = rope_of(d // 4, 1, 0), torch.randint(0, 9000, (1, n), generator=g, dtype=torch.int32).to(DEV)
    append(c, pos, k, v * 5, n_held=torch.tensor([ctx - 100], dtype=torch.int32), rope=rope, rp=rp)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r,ctx,hkv", [(3, 200, 700, 3), (3, 700, 3000, 5), (1, 2100, 2500, 2),
                                              (40, 60, 300, 4)])
def test_windows_of_every_kind_of_run(dtype, n_seqs, r, ctx, hkv):
    """Rows here and there, some of them twice, one in four left out, in windows of 4 and of 16 rows."""
    g = torch.Generator().manual_seed(r)
    c = Cache(n_seqs, ctx, hkv, hkv, 64, seed=r)
    pos = torch.randint(0, ctx, (n_seqs, r), generator=g).sort(1).values
    pos[torch.rand(n_seqs, r, generator=g) < 0.25] = -1
    pos = pos.flatten().to(torch.int32)
    _, k, v = new_rows(n_seqs * r, hkv, hkv, 64, dtype, 4)
    held = torch.randint(0, ctx, (n_seqs,), generator=g, dtype=torch.int32)
    rope, rp = rope_of(16, 1, 0), torch.randint(0, 99, (1, n_seqs * r), generator=g, dtype=torch.int32).to(DEV)
    append(c, pos, k, v * 3, n_held=held, rope=rope, rp=rp)
    pos[1:][pos[1:] == pos[:-1]] = -1
    append(c, pos, k * 2, v, n_held=held, rope=rope, rp=rp)


def test_the_last_of_rows_with_one_position():
    """Rows that share a position, in a short run, a long one and across windows."""
    c = Cache(1, 200, 2, 2, 64, seed=12)
    pos = torch.tensor([3, 3, 20, 21, 21, 22, 22, 22, 40, 41, 42, 43, 44, 45, 46, 46, 47, 48, 48], dtype=torch.int32)
    _, k, v = new_rows(len(pos), 2, 2, 64, "bf16", 5)
    append(c, pos, k, v, held=False, n_held=torch.tensor([200], dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hard_values(dtype):
    """Ties, borders of scales, zeros of both signs, denormal and the largest numbers,
    infinities and NaNs, in blocks of their own and beside others."""
    n, hkv, d = 320, 2, 64
    g = torch.Generator().manual_seed(9)
    ties = torch.cat([B.TABLE[:-1], (B.TABLE[1:] + B.TABLE[:-1]) / 2, torch.tensor([448.0, 449.0, 463.0, 480.0])])
    x = ties[torch.randint(0, len(ties), (2, n, hkv, d), generator=g)].float()
    x = x * torch.where(torch.rand(x.shape, generator=g) < 0.5, -1.0, 1.0)
    mag = torch.randint(-135, 119, (2, n // 16, 1, hkv, 1), generator=g).double()
    mag[:, 6] = 0.0
    x = (x.double().view(2, n // 16, 16, hkv, d) * torch.pow(2.0, mag)).float()
    x[:, 3] = 0.0
    x[:, 4] = -0.0
    x[:, 5] = torch.finfo(torch.bfloat16).max
    x[:, 6, ::3] *= 2.0 ** 20
    x = x.view(2, n, hkv, d)
    x[0, 130, 0, 5], x[1, 140, 1, 60], x[0, 199, 1, 0], x[1, 201, 0, 63] = math.inf, math.nan, -math.nan, -math.inf
    k, v = (t.to(DT[dtype]).to(DEV) for t in x)
    c = Cache(1, n + 30, hkv, hkv, d, seed=2, lo=0, hi=256)          # scale bytes that no append writes, too
    append(c, torch.arange(n, dtype=torch.int32), k, v)
    third = torch.arange(0, n, 3, dtype=torch.int32)
    append(c, third, k[::3] * 0.5, v[::3], n_held=torch.tensor([n], dtype=torch.int32))


def test_largest_scales_meet_smallest():
    """Kept tokens of the smallest scale beside new rows of the largest one."""
    c = Cache(1, 64, 1, 1, 64, seed=4, lo=10, hi=11)
    k = torch.full((1, 1, 64), 3e38, device=DEV)
    append(c, torch.tensor([7], dtype=torch.int32), k, -k, n_held=torch.tensor([16], dtype=torch.int32))


def test_bad_pages_stay_in_the_pool():
    c = Cache(1, 128, 2, 2, 64, seed=7)
    before = [t.clone() for t in c.dev]
    table = torch.tensor([[-7, 10 ** 9]], dtype=torch.int32, device=DEV)
    inner = api.byte_desc(*(t[1:3] for t in c.dev), 2, 128, table)
    k = torch.randn(128, 2, 64, device=DEV)
    api.conduit_append_byte(inner, torch.arange(128, dtype=torch.int32, device=DEV), k, k)
    for t, b in zip(c.dev, before):
        assert torch.equal(t[0], b[0]) and torch.equal(t[3], b[3])


def test_queries_in_place_and_strided_rows():
    n, hq, hkv, d = 9, 4, 2, 64
    c = Cache(1, 64, hq, hkv, d)
    q, k, v = new_rows(n, hq, hkv, d, "bf16", 1)
    rope, rp = rope_of(32, 1), torch.arange(n, dtype=torch.int32, device=DEV)
    want = torch.empty(n, hq, d, dtype=q.dtype, device=DEV)
    api.conduit_rotary(q, rope, rp, want)
    append(c, rp.cpu(), k, v, rope=rope, rp=rp[None], q=q, q_out=q)
    assert torch.equal(q, want)


def test_no_rows():
    c = Cache(2, 64, 2, 2, 64)
    before = [t.clone() for t in c.dev]
    e = torch.empty(0, 2, 64, device=DEV)
    api.conduit_append_byte(c.desc, torch.empty(0, dtype=torch.int32, device=DEV), e, e)
    for t, b in zip(c.dev, before):
        assert torch.equal(t, b)


def test_captured_appends():
    """A captured append replayed with new rows and positions, eager work in between."""
    c = Cache(3, 200, 2, 2, 64, seed=11)
    rope = rope_of(32, 1, 0)
    pos = torch.zeros(3, dtype=torch.int32, device=DEV)
    k, v = (torch.randn(3, 2, 64, device=DEV).to(torch.bfloat16) for _ in range(2))
    rp = torch.zeros(1, 3, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        api.conduit_append_byte(c.desc, pos, k, v, rope=rope, rope_pos=rp)
    for step in range(5):
        at = torch.tensor([step, 30 + step, -1 if step % 2 else 199], dtype=torch.int32)
        pos.copy_(at)
        rp.copy_(at[None])
        k.copy_(torch.randn(3, 2, 64) * (step + 1))
        v.copy_(torch.randn(3, 2, 64))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kt = M.rounded(M.turned(k.cpu(), rope.inv_freq, rope.axis, at[None]), torch.bfloat16)
        c.want.append(at, kt, v.cpu())
        c.check()
        eager = Cache(1, 64, 2, 2, 64, seed=step)
        append(eager, torch.tensor([step], dtype=torch.int32), k[:1], v[:1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,hkv,d,rot,axes,pairing,page", [
    (1, 4, 128, 128, 3, 0, 64), (77, 2, 64, 32, 2, 0, 64), (300, 1, 128, 128, 3, 1, 128), (2100, 4, 128, 16, 4, 0, 64),
    (65, 5, 64, 0, 1, 0, 256), (9000, 8, 64, 64, 1, 0, 64)])
def test_load(dtype, n, hkv, d, rot, axes, pairing, page):
    """Rows to a cache of 16 or 32 bits, turned by how far they move; rows left out; the
    rows in any order."""
    g = torch.Generator().manual_seed(n)
    n_src, n_ctx = n + 17, n + 90
    c = Cache(1, n_src, hkv, hkv, d, page, seed=n, pad=32)
    rope = rope_of(rot // 2, axes, pairing) if rot else None
    rp = torch.randint(-9000, 9000, (axes, n), generator=g, dtype=torch.int32).to(DEV) if rot else None
    src = torch.randperm(n_src, generator=g)[:n].to(torch.int32)
    dst = torch.randperm(n_ctx, generator=g)[:n].to(torch.int32)
    if n > 3:
        src[0], dst[1], src[-1] = -1, n_ctx, n_src
    ck, cv = (torch.randn(n_ctx, hkv, d, generator=g).to(DT[dtype]).to(DEV) for _ in range(2))
    wk, wv = ck.cpu().clone(), cv.cpu().clone()
    api.conduit_load_byte(c.desc, src.to(DEV), api.kv_desc(ck, cv, hkv), dst.to(DEV), rope=rope, rope_pos=rp)
    k, v = c.want.rows(0, n_src)
    live = (src >= 0) & (src < n_src) & (dst >= 0) & (dst < n_ctx)
    kk = k[src.clamp(0, n_src - 1).long()]
    if rope is not None:
        kk = M.turned(kk, rope.inv_freq, rope.axis, rp.cpu(), pairing == 1)
    wk[dst[live].long()] = M.rounded(kk, DT[dtype])[live]
    wv[dst[live].long()] = M.rounded(v[src.clamp(0, n_src - 1).long()], DT[dtype])[live]
    assert torch.equal(ck.cpu(), wk) and torch.equal(cv.cpu(), wv)


def test_load_into_pages_and_of_marked_tokens():
    """NaN keys come back as NaN, scale bytes that no append writes as the nearest."""
    c = Cache(2, 100, 2, 2, 64, seed=8, lo=0, hi=256)
    _, k, v = new_rows(2, 2, 2, 64, "bf16", 4)
    k[0, 1, 3] = math.nan
    append(c, torch.tensor([40, 99], dtype=torch.int32), k, v)
    page = 64
    kp, vp = (torch.zeros(4, page, 2, 64, device=DEV) for _ in range(2))
    table = torch.tensor([2, 0, 3], dtype=torch.int32, device=DEV)
    kv = api.kv_desc_paged(kp, vp, table, 180, 2)
    src = torch.cat([torch.arange(80), torch.arange(20, 100)]).to(torch.int32)
    dst = torch.arange(160, dtype=torch.int32)
    api.conduit_load_byte(c.desc, src.to(DEV), kv, dst.to(DEV))
    flat = [p.cpu()[table.cpu().long()].reshape(-1, 2, 64) for p in (kp, vp)]
    for s, lo, hi, base in ((0, 0, 80, 0), (1, 20, 100, 80)):
        for got, want in zip(flat, c.want.rows(s, 100)):
            want = want[lo:hi].float()
            got = got[base:base + hi - lo]
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(3.0), want.nan_to_num(3.0))
    assert flat[0][40, 1].isnan().all() and flat[0][40, 0].isfinite().all()


def test_other_device_and_stream():
    """A pool on the CPU is refused; a call on another stream waits for nothing else."""
    c = Cache(1, 64, 2, 2, 64)
    cpu = api.byte_desc(*(t.cpu().contiguous() for t in c.dev), 2, 64)
    x, pos = torch.zeros(2, 2, 64, device=DEV), torch.arange(2, dtype=torch.int32, device=DEV)
    with pytest.raises(api.ConduitError, match="different devices"):
        api.conduit_append_byte(cpu, pos, x, x)
    with pytest.raises(api.ConduitError, match="different devices"):
        api.conduit_load_byte(cpu, pos, api.kv_desc(x, x.clone(), 2), pos)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    k = torch.randn(2, 2, 64, device=DEV)
    s.wait_stream(torch.cuda.current_stream())
    api.conduit_append_byte(c.desc, pos, k, k, stream=s)
    s.synchronize()
    c.want.append(pos.cpu(), k.cpu(), k.cpu())
    c.check()
