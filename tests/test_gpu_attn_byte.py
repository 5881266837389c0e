"""Attention over an 8-bit cache (conduit_attn_byte) against 64 bits."""
import math

import pytest
import torch

from paper_2609_05821_amd import api
from tests import byte_oracle as B
from tests import mx_oracle as M
from tests.gpu_helpers import DEV
from tests.test_gpu_rotary import DT

pytestmark = pytest.mark.gpu


class Store:
    """A paged 8-bit cache with random contents: every code but NaN, scales around 2^-7."""

    def __init__(self, n_seqs, ctx, hq, hkv, d, page=64, seed=0, contiguous=False):
        g = torch.Generator().manual_seed(seed)
        self.n_seqs, self.ctx, self.hq, self.hkv, self.d, self.page = n_seqs, ctx, hq, hkv, d, page
        per = -(-ctx // page)
        n_pages = n_seqs * per + (0 if contiguous else 3)
        codes = [torch.randint(0, 256, (n_pages, hkv, page, d), generator=g, dtype=torch.uint8) for _ in range(2)]
        for x in codes:
            x[(x & 127) == 127] = 0x31
        self.cpu = codes + [torch.randint(116, 121, (n_pages, hkv, page // 16), generator=g, dtype=torch.uint8)
                            for _ in range(2)]
        self.table = torch.arange(n_pages)[None].to(torch.int32).view(n_seqs, per) if contiguous else \
            torch.randperm(n_pages, generator=g)[:n_seqs * per].to(torch.int32).view(n_seqs, per)
        self.contiguous = contiguous
        self.upload()

    def upload(self):
        self.dev = [t.to(DEV) for t in self.cpu]
        self.desc = api.byte_desc(*self.dev, self.hq, self.ctx, None if self.contiguous else self.table.to(DEV),
                                self.n_seqs)

    def wide(self):
        """A descriptor of the same cache with room for 2^18 tokens (pages that no row reaches): calls of many
        pairs are made in blocks of 256 there."""
        per = 2 ** 18 // self.page
        table = torch.zeros(self.n_seqs, per, dtype=torch.int32)
        table[:, :self.table.shape[1]] = self.table
        return api.byte_desc(*self.dev, self.hq, 2 ** 18, table.to(DEV), self.n_seqs)

    def many(self, r, dtype, desc):
        """Whether a call with r rows per sequence takes blocks of 256 pairs."""
        pairs = r * self.hq // self.hkv
        return dtype == torch.bfloat16 and pairs > (64 if self.d == 128 else 128) and \
            self.n_seqs * self.hkv * -(-pairs // 32) * desc.n_ctx >= 2 ** 18

    def descs(self, r, dtype):
        """The cache's descriptor, and the wide one if calls with r rows run otherwise there."""
        wide = self.wide()
        return [self.desc, wide] if self.many(r, dtype, wide) != self.many(r, dtype, self.desc) else [self.desc]

    def rows(self, s, n):
        """Keys and values of tokens 0 .. n - 1 of sequence s, float64."""
        pos = torch.arange(n)
        pages = self.table[s, pos // self.page].long()
        slot = pos % self.page
        return tuple(B.decoded(self.cpu[i][pages, :, slot]) * B.factor(self.cpu[i + 2][pages, :, slot // 16])[..., None]
                     for i in (0, 1))

    def factors(self, s, n):
        """Factors of the value scales of tokens 0 .. n - 1 of sequence s."""
        pos = torch.arange(n)
        return B.factor(self.cpu[3][self.table[s, pos // self.page].long(), :, pos % self.page // 16])

    def set(self, which, s, t, value):
        """Every code of token t of sequence s in pool `which`, or the scales of its block."""
        slot = t % self.page
        self.cpu[which][int(self.table[s, t // self.page]), :, slot if which < 2 else slot // 16] = value


def run(st, q, pos, lse=True, desc=None, **kw):
    o = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
    l = torch.full(q.shape[:2], 9.0, device=DEV) if lse else None
    api.conduit_attn_byte(desc or st.desc, q.to(DEV), pos.to(DEV), o, lse_out=l, **kw)
    return o.cpu(), None if l is None else l.cpu()


def check(st, q, pos, o, lse, scale=None, rows=None, desc=None):
    r = len(pos) // st.n_seqs
    for s in range(st.n_seqs):
        p = pos[s * r:(s + 1) * r]
        n = max(0, min(int(p.max()) + 1, st.ctx))
        k, v = st.rows(s, n)
        sel = range(r) if rows is None else rows
        qq = q[s * r:(s + 1) * r][list(sel)]
        want = M.attention(qq, k, v, p[list(sel)], scale)
        bo, bl = B.attention_bounds(*want, n, st.d, q.dtype == torch.bfloat16)
        if st.many(r, q.dtype, desc or st.desc):
            bo = bo + B.weight_floor(qq, k, v, st.factors(s, n), p[list(sel)], want[1], scale)
        go, gl = o[s * r:(s + 1) * r][list(sel)].double(), lse[s * r:(s + 1) * r][list(sel)].double()
        err = (go - want[0]).abs()
        assert (err <= bo).all(), f"sequence {s}: output {(err / bo).max():.3g} of the bound"
        empty = p[list(sel)] < 0
        assert (gl[empty] == -math.inf).all() and (go[empty] == 0).all()
        err = (gl - want[1]).abs()[~empty]
        assert (err <= bl[~empty]).all(), f"sequence {s}: log-sum-exp {(err / bl[~empty]).max():.3g} of the bound"


def queries(n, hq, d, dtype, seed, spread=1.0):
    return (torch.randn(n, hq, d, generator=torch.Generator().manual_seed(seed)) * spread).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,ctx,page", [
    (1, 1, 1, 1, 64, 1, 64), (1, 1, 8, 8, 64, 672, 64), (1, 1, 28, 4, 128, 1500, 64), (3, 1, 7, 1, 128, 300, 128),
    (5, 5, 8, 2, 128, 1300, 64), (2, 3, 6, 6, 64, 129, 64), (4, 1, 16, 1, 64, 2000, 256), (2, 1, 20, 1, 128, 900, 64),
    (1, 57, 8, 8, 64, 672, 64), (1, 40, 7, 1, 128, 1250, 64), (2, 33, 4, 4, 64, 700, 64), (1, 130, 6, 2, 128, 200, 64),
    (9, 2, 10, 2, 128, 1100, 64), (1, 301, 2, 2, 64, 1400, 64), (1, 90, 14, 2, 128, 2600, 64)])
def test_attention(dtype, n_seqs, r, hq, hkv, d, ctx, page):
    st = Store(n_seqs, ctx, hq, hkv, d, page, seed=ctx + r)
    g = torch.Generator().manual_seed(ctx)
    q = queries(n_seqs * r, hq, d, dtype, r)
    pos = torch.randint(0, ctx, (n_seqs * r,), generator=g, dtype=torch.int32)
    pos[-1] = ctx - 1
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, q, pos, desc=desc)
        check(st, q, pos, o, lse, desc=desc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1024, 1025, 1153])
def test_lengths(dtype, length):
    """Last tokens around the borders of wave steps, workgroup steps, pages and parts, in
    a cache just large enough and in a larger one."""
    for ctx in (length, 4000):
        st = Store(1, ctx, 4, 2, 128, seed=length)
        q, pos = queries(1, 4, 128, dtype, length), torch.tensor([length - 1], dtype=torch.int32)
        o, lse = run(st, q, pos)
        check(st, q, pos, o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_contiguous_pool(dtype):
    st = Store(3, 500, 4, 2, 64, seed=5, contiguous=True)
    q, pos = queries(6, 4, 64, dtype, 1), torch.tensor([3, 499, 64, 63, 0, 200], dtype=torch.int32)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx", [200, 3000])
@pytest.mark.parametrize("r", [1, 4, 60])
def test_empty_rows_and_sequences(dtype, ctx, r):
    n_seqs = 4
    st = Store(n_seqs, ctx, 6, 2, 128, seed=r)
    q = queries(n_seqs * r, 6, 128, dtype, 2)
    pos = torch.randint(0, ctx, (n_seqs, r), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    pos[1] = -1                                  # a padded sequence
    pos[2, r // 2] = -2 ** 31                    # a padded row
    pos[3, r - 1] = 0
    pos = pos.flatten()
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, q, pos, desc=desc)
        check(st, q, pos, o, lse, desc=desc)
        o, lse = run(st, q, torch.full_like(pos, -1), desc=desc)   # nothing at all
        assert (o == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 3000), (5, 400), (80, 1500)])
def test_masked_keys_may_hold_anything(dtype, r, ctx):
    """Bytes of every kind past every row of a sequence, in its last block too; NaN keys
    between its rows reach exactly the rows that attend to them."""
    st = Store(1, ctx, 4, 2, 128, seed=ctx)
    q = queries(r, 4, 128, dtype, 4)
    pos = torch.randint(0, ctx // 2, (r,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    pos[0] = ctx // 2
    clean = [run(st, q, pos, desc=desc) for desc in st.descs(r, q.dtype)]
    for desc, got in zip(st.descs(r, q.dtype), clean):
        check(st, q, pos, *got, desc=desc)
    last = ctx // 2
    for t in range(last + 1, ctx):
        st.set(0, 0, t, (127, 255, 126, 3)[t % 4])
        st.set(1, 0, t, (255, 127, 254, 126)[t % 4])
        if t // 16 > last // 16:
            st.set(2, 0, t, (255, 0, 246, 9)[t // 16 % 4])
            st.set(3, 0, t, (0, 255, 247, 246)[t // 16 % 4])
    st.upload()
    for desc, (co, cl) in zip(st.descs(r, q.dtype), clean):
        o, lse = run(st, q, pos, desc=desc)
        assert torch.equal(o, co) and torch.equal(lse, cl)
    nan_at = int(pos.sort().values[r // 2]) if r > 1 else last
    st.set(0, 0, nan_at, 0x7f)
    st.upload()
    hit = pos >= nan_at
    for desc, (co, cl) in zip(st.descs(r, q.dtype), clean):
        o, lse = run(st, q, pos, desc=desc)
        assert o[hit].isnan().all() and lse[hit].isnan().all()
        assert torch.equal(o[~hit], co[~hit]) and torch.equal(lse[~hit], cl[~hit])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_positions_past_the_cache(dtype):
    """No key past n_ctx - 1 is read; the other rows keep their results."""
    st = Store(2, 150, 4, 2, 64, seed=8)
    q = queries(6, 4, 64, dtype, 5)
    pos = torch.tensor([149, 3, 40, 149, 60, 7], dtype=torch.int32)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)
    far = pos.clone()
    far[0], far[3] = 150, 2 ** 31 - 1
    o2, lse2 = run(st, q, far)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)


@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,ctx", [(1, 150, 4, 2, 128, 14011), (2, 60, 9, 3, 64, 7501)])
def test_positions_past_a_cache_of_many_pairs(n_seqs, r, hq, hkv, d, ctx):
    """The same with blocks of 256 pairs, whose last tile the cache ends in."""
    st = Store(n_seqs, ctx, hq, hkv, d, seed=8)
    assert st.many(r, torch.bfloat16, st.desc)
    for i in (0, 1):                              # what is behind the last token is in no sequence
        for s in range(n_seqs):
            for t in range(ctx, -(-ctx // 64) * 64):
                st.set(i, s, t, 0x7f)
    st.upload()
    q = queries(n_seqs * r, hq, d, "bf16", 5)
    pos = torch.randint(0, ctx, (n_seqs * r,), generator=torch.Generator().manual_seed(6), dtype=torch.int32)
    pos[::7] = ctx - 1
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse, rows=[0, 1, 6, 7, r - 1])
    far = pos.clone()
    far[::7], far[7] = ctx, 2 ** 31 - 1
    o2, lse2 = run(st, q, far)
    assert torch.equal(o2, o) and torch.equal(lse2, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [1, 3, 70])
def test_sharp_and_rising_logits(dtype, r):
    """Maxima that rise step by step, logits of hundreds, and a scale of one's own."""
    ctx, hq, hkv, d = 2500, 4, 2, 128
    st = Store(1, ctx, hq, hkv, d, seed=6)
    for t in range(ctx):                          # scales grow with the token: 2^-17 .. 2^-5
        st.set(2, 0, t, 110 + 12 * t // ctx)
    st.upload()
    q = queries(r, hq, d, dtype, 7, spread=3.0)
    pos = torch.linspace(ctx - 1, ctx // 3, r).to(torch.int32)
    for scale in (None, 0.3):
        for desc in st.descs(r, q.dtype):
            o, lse = run(st, q, pos, scale=scale, desc=desc)
            check(st, q, pos, o, lse, scale=scale, desc=desc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_sequence_among_short_ones(dtype):
    st = Store(6, 20000, 8, 2, 128, page=256, seed=9)
    pos = torch.tensor([19999, 0, 130, -1, 5000, 64], dtype=torch.int32)
    q = queries(6, 8, 128, dtype, 8)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_rows(dtype):
    """A refresh-sized set of rows, sampled rows checked (the first and last of it too)."""
    ctx, hq, hkv, d, r = 5000, 28, 4, 128, 700
    st = Store(1, ctx, hq, hkv, d, seed=10)
    g = torch.Generator().manual_seed(10)
    pos = torch.randperm(ctx, generator=g)[:r].sort().values.to(torch.int32)
    q = queries(r, hq, d, dtype, 9)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse, rows=[0, 1, 5, 36, 37, 350, 351, 511, 698, 699])
    mixed = pos[torch.randperm(r, generator=g)]       # any order of rows
    o, lse = run(st, q, mixed)
    check(st, q, mixed, o, lse, rows=[0, 7, 300, 699])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r", [1, 25, 45])
def test_a_workgroup_per_block(dtype, d, r):
    """More blocks than CUs, short caches: every block by one workgroup."""
    n = 300
    st = Store(n, 260, 3, 1, d, page=64, seed=21)
    g = torch.Generator().manual_seed(4)
    pos = torch.randint(-1, 260, (n * r,), generator=g, dtype=torch.int32)
    q = queries(n * r, 3, d, dtype, 5)
    o, lse = run(st, q, pos)
    for s in (0, 1, 63, 150, 298, 299):
        p = pos[s * r:(s + 1) * r]
        m = max(int(p.max()) + 1, 0)
        k, v = st.rows(s, m)
        want = M.attention(q[s * r:(s + 1) * r], k, v, p)
        bo, bl = B.attention_bounds(*want, m, d, dtype == "bf16")
        assert ((o[s * r:(s + 1) * r].double() - want[0]).abs() <= bo).all()
        live = p >= 0
        assert ((lse[s * r:(s + 1) * r].double() - want[1]).abs()[live] <= bl[live]).all()
        assert (lse[s * r:(s + 1) * r][~live] == -math.inf).all()


def test_many_rows_of_small_heads():
    """Heads of 64 dims, as many blocks as merge by groups of pairs."""
    ctx, hq, hkv, d, r = 1500, 32, 8, 64, 600
    st = Store(1, ctx, hq, hkv, d, seed=22)
    pos = torch.randperm(ctx, generator=torch.Generator().manual_seed(3))[:r].sort().values.to(torch.int32)
    q = queries(r, hq, d, "bf16", 6)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse, rows=[0, 1, 31, 32, 33, 300, 567, 599])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r", [2, 90])
def test_keys_past_a_row_hold_anything(dtype, d, r):
    """Rows of one block at tokens 95 and 600, whatever bytes follow token 95."""
    st = Store(1, 640, 4, 2, d, page=64, seed=23)
    g = torch.Generator().manual_seed(8)
    k, v = st.rows(0, 96)
    for t in range(96, 640):
        at = int(st.table[0, t // 64])
        for i in (0, 1):
            st.cpu[i][at, :, t % 64] = torch.randint(0, 256, (2, d), generator=g, dtype=torch.uint8)
            st.cpu[i][at, :, t % 64, t % d] = 127
        for i in (2, 3):
            st.cpu[i][at, :, t % 64 // 16] = torch.randint(0, 256, (2,), generator=g, dtype=torch.uint8)
    st.upload()
    pos = torch.tensor([95, 600] * (r // 2), dtype=torch.int32)
    q = queries(r, 4, d, dtype, 9)
    want = M.attention(q[::2], k, v, pos[::2])
    bo, bl = B.attention_bounds(*want, 96, d, dtype == "bf16")
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, q, pos, desc=desc)
        assert ((o[::2].double() - want[0]).abs() <= bo).all()
        assert ((lse[::2].double() - want[1]).abs() <= bl).all()


@pytest.mark.parametrize("n_seqs,hkv", [(9, 8), (60, 8), (64, 5), (65, 5)])
def test_ragged_sequences_share_workgroups(n_seqs, hkv):
    """Few blocks (parts end with their block), many (parts go on into the next),
    and either side of the list that a wave holds."""
    st = Store(n_seqs, 2100, hkv, hkv, 64, page=64, seed=24)
    g = torch.Generator().manual_seed(10)
    pos = torch.randint(0, 2100, (n_seqs,), generator=g, dtype=torch.int32)
    pos[0], pos[3], pos[4], pos[-1] = 2099, -1, -1, 0
    q = queries(n_seqs, hkv, 64, "bf16", 11)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)


def test_many_sequences():
    """More sequence blocks than the list of parts holds: one workgroup per block."""
    n = 4500
    st = Store(n, 1100, 1, 1, 64, page=64, seed=11)
    pos = torch.randint(-1, 1100, (n,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    q = queries(n, 1, 64, "bf16", 3)
    o, lse = run(st, q, pos)
    for s in (0, 1, 17, 2048, 4095, 4096, 4499):
        m = max(int(pos[s]) + 1, 0)
        k, v = st.rows(s, m)
        want = M.attention(q[s:s + 1], k, v, pos[s:s + 1])
        bo, bl = B.attention_bounds(*want, m, 64, True)
        assert ((o[s:s + 1].double() - want[0]).abs() <= bo).all()
        if m:
            assert ((lse[s:s + 1].double() - want[1]).abs() <= bl).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 9000), (1, 200), (120, 3000), (160, 8000)])
def test_repeatable_and_workspace(dtype, r, ctx):
    """Bit for bit the same on repeated calls, on a workspace full of NaN, on one that
    another call has used, and without the log-sum-exp."""
    st = Store(2, ctx, 7, 1, 128, seed=12)
    q = queries(2 * r, 7, 128, dtype, 1)
    pos = torch.randint(0, ctx, (2 * r,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    o, lse = run(st, q, pos)
    need = api.attn_byte_workspace_bytes(st.desc, q)
    ws = torch.full((need + 1024,), 255, dtype=torch.uint8, device=DEV)
    guard = ws[need:].clone()
    for _ in range(2):
        o2, lse2 = run(st, q, pos, ws=ws)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    run(st, q, pos.flip(0), ws=ws)
    o2, lse2 = run(st, q, pos, ws=ws)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    assert torch.equal(ws[need:], guard)
    assert torch.equal(run(st, q, pos, lse=False)[0], o)


@pytest.mark.parametrize("r,ctx", [(1, 6000), (60, 1500), (110, 9000)])
def test_captured_calls(r, ctx):
    """Two captured calls that share one workspace, replayed with new positions and
    cache contents, eager calls in between."""
    st = Store(2, ctx, 8, 2, 128, seed=13)
    g = torch.Generator().manual_seed(1)
    q = [queries(2 * r, 8, 128, "bf16", i).to(DEV) for i in range(2)]
    pos = [torch.randint(0, ctx, (2 * r,), generator=g, dtype=torch.int32).to(DEV) for _ in range(2)]
    o = [torch.zeros_like(x) for x in q]
    lse = [torch.zeros(x.shape[:2], device=DEV) for x in q]
    ws = torch.empty(max(1, api.attn_byte_workspace_bytes(st.desc, q[0])), dtype=torch.uint8, device=DEV)
    graphs = []
    api.conduit_attn_byte(st.desc, q[0], pos[0], o[0], lse_out=lse[0], ws=ws)  # loads the kernels
    torch.cuda.synchronize()
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            api.conduit_attn_byte(st.desc, q[i], pos[i], o[i], lse_out=lse[i], ws=ws)
        graphs.append(gr)
    for step in range(4):
        for i in range(2):
            pos[i].copy_(torch.randint(-1, ctx, (2 * r,), generator=g, dtype=torch.int32))
        st.dev[0].random_(0, 120)
        torch.cuda.synchronize()
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for i in range(2):
            oe, le = torch.empty_like(o[i]), torch.empty_like(lse[i])
            api.conduit_attn_byte(st.desc, q[i], pos[i], oe, lse_out=le)
            torch.cuda.synchronize()
            assert torch.equal(o[i], oe) and torch.equal(lse[i], le), f"replay {step}, call {i}"


def test_two_streams():
    """Calls that run at the same time on streams and workspaces of their own."""
    st = Store(4, 8000, 8, 2, 128, seed=14)
    qs = [queries(4, 8, 128, "bf16", i).to(DEV) for i in range(2)]
    pos = [torch.tensor(p, dtype=torch.int32, device=DEV) for p in ([7999, 10, 3000, 0], [5, 7000, -1, 7999])]
    want = [run(st, q, p) for q, p in zip(qs, pos)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [(torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)) for q in qs]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, q, p, (o, l) in zip(streams, qs, pos, outs):
            api.conduit_attn_byte(st.desc, q, p, o, lse_out=l, stream=s)
    torch.cuda.synchronize()
    for (o, l), (wo, wl) in zip(outs, want):
        assert torch.equal(o.cpu(), wo) and torch.equal(l.cpu(), wl)


def test_a_pool_on_another_device_is_refused():
    st = Store(1, 64, 4, 2, 128)
    cpu = api.byte_desc(*st.cpu, 4, 64, None)
    x = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(api.ConduitError, match="different devices"):
        api.conduit_attn_byte(cpu, x, torch.zeros(2, dtype=torch.int32, device=DEV), x.clone())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [1, 9, 70])
def test_value_scales_far_apart(dtype, r):
    """A sink of zero values and small scales that takes nearly all of the weight, blocks of
    values 2^60 times as large that take next to none, rows that see one kind or both."""
    ctx, hq, hkv, d = 1500, 8, 2, 128
    st = Store(1, ctx, hq, hkv, d, seed=31)
    for t in range(0, ctx, 16):
        kind = t // 16 % 5
        st.set(3, 0, t, (118, 60, 178, 118, 90)[kind])
        st.set(2, 0, t, 121 if kind in (1, 4) else 114)
    for t in range(16):
        st.set(1, 0, t, 0)
    st.set(3, 0, 0, 10)
    st.upload()
    pos = torch.linspace(ctx - 1, 12, r).to(torch.int32)
    q = queries(r, hq, d, dtype, 3)
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, q, pos, desc=desc)
        check(st, q, pos, o, lse, desc=desc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r", [(3, 50), (5, 3)])
def test_all_of_a_sequence(dtype, n_seqs, r):
    """Every row sees all of its sequence, as a text's rows an encoder's states."""
    st = Store(n_seqs, 777, 6, 2, 64, seed=41)
    length = torch.tensor([777, 1, 16, 300, 63][:n_seqs])
    pos = (length[:, None] - 1).expand(n_seqs, r).flatten().to(torch.int32)
    q = queries(n_seqs * r, 6, 64, dtype, 5)
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, q, pos, desc=desc)
        check(st, q, pos, o, lse, desc=desc)


def test_outputs_are_rounded_once():
    """bf16 outputs over many keys are as far from 64 bits as their own rounding puts them: up
    to half a step h off, evenly, so h^2 / 3 on average (over the 1,024 values of a row the
    2-norm strays by 2% from that; 20% are allowed), and 2^-12 of the norm for what the
    products round (2^-11 of a weight at most, averaged over 6,000)."""
    st = Store(1, 6000, 8, 2, 128, seed=51)
    k, v = st.rows(0, 6000)
    for r in (1, 40):
        q = queries(r, 8, 128, "bf16", 6)
        pos = torch.full((r,), 5999, dtype=torch.int32)
        o, _ = run(st, q, pos, desc=st.descs(r, q.dtype)[-1])
        for i in range(min(r, 4)):
            want = M.attention(q[i:i + 1], k, v, pos[i:i + 1])[0]
            half = torch.ldexp(torch.ones((), dtype=torch.float64), torch.frexp(want)[1] - 9)
            err = (o[i:i + 1].double() - want).norm()
            assert err <= 1.2 * (half.norm() / 3 ** 0.5) + 2.0 ** -12 * want.norm()
