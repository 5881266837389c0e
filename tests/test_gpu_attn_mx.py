"""Attention over a 4-bit cache (conduit_attn_mx) against 64 bits."""
import math

import pytest
import torch

from paper_2609_05821_amd import api
from tests import mx_oracle as M
from tests.gpu_helpers import DEV
from tests.test_gpu_rotary import DT

pytestmark = pytest.mark.gpu


class Store:
    """A paged 4-bit cache with random contents: normal-like codes, scales around 1."""

    def __init__(self, n_seqs, ctx, hq, hkv, d, page=64, seed=0, contiguous=False):
        g = torch.Generator().manual_seed(seed)
        self.n_seqs, self.ctx, self.hq, self.hkv, self.d, self.page = n_seqs, ctx, hq, hkv, d, page
        per = -(-ctx // page)
        n_pages = n_seqs * per + (0 if contiguous else 3)
        shape = (n_pages, hkv, page)
        self.cpu = [torch.randint(0, 256, (*shape, d // 2), generator=g, dtype=torch.uint8) for _ in range(2)] + \
                   [torch.randint(124, 127, (*shape, d // 32), generator=g, dtype=torch.uint8) for _ in range(2)]
        self.table = torch.arange(n_pages)[None].to(torch.int32).view(n_seqs, per) if contiguous else \
            torch.randperm(n_pages, generator=g)[:n_seqs * per].to(torch.int32).view(n_seqs, per)
        self.contiguous = contiguous
        self.upload()

    def upload(self):
        self.dev = [t.to(DEV) for t in self.cpu]
        self.mx = api.mx_desc(self.dev[0], self.dev[1], self.dev[2], self.dev[3], self.hq, self.ctx,
                              None if self.contiguous else self.table.to(DEV), self.n_seqs)

    def rows(self, s, n):
        """Keys and values of tokens 0 .. n - 1 of sequence s, float64."""
        pos = torch.arange(n)
        seq = torch.full((n,), s)
        return tuple(M.held(M.gather(self.cpu[i], self.table, seq, pos, self.page),
                            M.gather(self.cpu[i + 2], self.table, seq, pos, self.page)) for i in (0, 1))

    def set(self, which, s, t, value):
        """Every byte of token t of sequence s in pool `which`."""
        self.cpu[which][int(self.table[s, t // self.page]), :, t % self.page] = value


def run(st, q, pos, lse=True, **kw):
    o = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
    l = torch.full(q.shape[:2], 9.0, device=DEV) if lse else None
    api.conduit_attn_mx(st.mx, q.to(DEV), pos.to(DEV), o, lse_out=l, **kw)
    return o.cpu(), None if l is None else l.cpu()


def check(st, q, pos, o, lse, scale=None, rows=None):
    r = len(pos) // st.n_seqs
    for s in range(st.n_seqs):
        p = pos[s * r:(s + 1) * r]
        n = max(0, min(int(p.max()) + 1, st.ctx))
        k, v = st.rows(s, n)
        sel = range(r) if rows is None else rows
        qq = q[s * r:(s + 1) * r][list(sel)]
        want = M.attention(qq, k, v, p[list(sel)], scale)
        bo, bl = M.attention_bounds(*want, n, st.d, q.dtype == torch.bfloat16)
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
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)


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
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)
    o, lse = run(st, q, torch.full_like(pos, -1))   # nothing at all
    assert (o == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 3000), (5, 400), (80, 1500)])
def test_masked_keys_may_hold_anything(dtype, r, ctx):
    """NaN keys, and bytes of every kind, past every row of a sequence; NaN keys between
    its rows reach exactly the rows that attend to them."""
    st = Store(1, ctx, 4, 2, 128, seed=ctx)
    q = queries(r, 4, 128, dtype, 4)
    pos = torch.randint(0, ctx // 2, (r,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    pos[0] = ctx // 2
    clean, clean_lse = run(st, q, pos)
    check(st, q, pos, clean, clean_lse)
    for t in range(ctx // 2 + 1, ctx):
        st.set(2, 0, t, 255)
        st.set(3, 0, t, (255, 254, 253, 0)[t % 4])
        st.set(1, 0, t, 119)
    st.upload()
    o, lse = run(st, q, pos)
    assert torch.equal(o, clean) and torch.equal(lse, clean_lse)
    nan_at = int(pos.sort().values[r // 2]) if r > 1 else ctx // 2
    st.set(2, 0, nan_at, 255)
    st.upload()
    o, lse = run(st, q, pos)
    hit = pos >= nan_at
    assert o[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(o[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])


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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r", [1, 3, 70])
def test_sharp_and_rising_logits(dtype, r):
    """Maxima that rise step by step, logits of hundreds, and a scale of one's own."""
    ctx, hq, hkv, d = 2500, 4, 2, 128
    st = Store(1, ctx, hq, hkv, d, seed=6)
    for t in range(ctx):                          # scales grow with the token: 2^-9 .. 2^3
        st.set(2, 0, t, 118 + 12 * t // ctx)
    st.upload()
    q = queries(r, hq, d, dtype, 7, spread=3.0)
    pos = torch.linspace(ctx - 1, ctx // 3, r).to(torch.int32)
    for scale in (None, 0.3):
        o, lse = run(st, q, pos, scale=scale)
        check(st, q, pos, o, lse, scale=scale)


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
@pytest.mark.parametrize("r", [1, 25])
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
        bo, bl = M.attention_bounds(*want, m, d, dtype == "bf16")
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
@pytest.mark.parametrize("r", [2, 60])
def test_keys_past_a_row_hold_anything(dtype, d, r):
    """Rows of one block at tokens 99 and 600, whatever bytes follow token 99."""
    st = Store(1, 640, 4, 2, d, page=64, seed=23)
    g = torch.Generator().manual_seed(8)
    k, v = st.rows(0, 100)
    for t in range(100, 640):
        at = int(st.table[0, t // 64])
        for i in (2, 3):
            st.cpu[i][at, :, t % 64] = torch.randint(0, 256, (2, d // 32), generator=g, dtype=torch.uint8)
            st.cpu[i][at, :, t % 64, t % (d // 32)] = 255
    st.upload()
    pos = torch.tensor([99, 600] * (r // 2), dtype=torch.int32)
    q = queries(r, 4, d, dtype, 9)
    o, lse = run(st, q, pos)
    want = M.attention(q[::2], k, v, pos[::2])
    bo, bl = M.attention_bounds(*want, 100, d, dtype == "bf16")
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
        bo, bl = M.attention_bounds(*want, m, 64, True)
        assert ((o[s:s + 1].double() - want[0]).abs() <= bo).all()
        if m:
            assert ((lse[s:s + 1].double() - want[1]).abs() <= bl).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 9000), (1, 200), (120, 3000)])
def test_repeatable_and_workspace(dtype, r, ctx):
    """Bit for bit the same on repeated calls, on a workspace full of NaN, on one that
    another call has used, and without the log-sum-exp."""
    st = Store(2, ctx, 7, 1, 128, seed=12)
    q = queries(2 * r, 7, 128, dtype, 1)
    pos = torch.randint(0, ctx, (2 * r,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    o, lse = run(st, q, pos)
    need = api.attn_mx_workspace_bytes(st.mx, q)
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


@pytest.mark.parametrize("r,ctx", [(1, 6000), (60, 1500)])
def test_captured_calls(r, ctx):
    """Two captured calls that share one workspace, replayed with new positions and
    cache contents, eager calls in between."""
    st = Store(2, ctx, 8, 2, 128, seed=13)
    g = torch.Generator().manual_seed(1)
    q = [queries(2 * r, 8, 128, "bf16", i).to(DEV) for i in range(2)]
    pos = [torch.randint(0, ctx, (2 * r,), generator=g, dtype=torch.int32).to(DEV) for _ in range(2)]
    o = [torch.zeros_like(x) for x in q]
    lse = [torch.zeros(x.shape[:2], device=DEV) for x in q]
    ws = torch.empty(max(1, api.attn_mx_workspace_bytes(st.mx, q[0])), dtype=torch.uint8, device=DEV)
    graphs = []
    api.conduit_attn_mx(st.mx, q[0], pos[0], o[0], lse_out=lse[0], ws=ws)  # loads the kernels
    torch.cuda.synchronize()
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            api.conduit_attn_mx(st.mx, q[i], pos[i], o[i], lse_out=lse[i], ws=ws)
        graphs.append(gr)
    for step in range(4):
        for i in range(2):
            pos[i].copy_(torch.randint(-1, ctx, (2 * r,), generator=g, dtype=torch.int32))
        st.dev[0].random_(0, 256)
        torch.cuda.synchronize()
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for i in range(2):
            oe, le = torch.empty_like(o[i]), torch.empty_like(lse[i])
            api.conduit_attn_mx(st.mx, q[i], pos[i], oe, lse_out=le)
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
            api.conduit_attn_mx(st.mx, q, p, o, lse_out=l, stream=s)
    torch.cuda.synchronize()
    for (o, l), (wo, wl) in zip(outs, want):
        assert torch.equal(o.cpu(), wo) and torch.equal(l.cpu(), wl)


def test_a_pool_on_another_device_is_refused():
    st = Store(1, 64, 4, 2, 128)
    cpu = api.mx_desc(*st.cpu, 4, 64, None)
    x = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)
    kv, pos = x[:, :2], torch.zeros(2, dtype=torch.int32, device=DEV)
    cache = torch.zeros(64, 2, 128, dtype=torch.bfloat16, device=DEV)
    for call in (lambda: api.conduit_attn_mx(cpu, x, pos, x.clone()),
                 lambda: api.conduit_append_mx(cpu, pos, kv, kv),
                 lambda: api.conduit_load_mx(cpu, pos, api.kv_desc(cache, cache, 4), pos)):
        with pytest.raises(api.ConduitError, match="different devices"):
            call()
