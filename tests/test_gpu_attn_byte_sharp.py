"""Attention over an 8-bit cache with bounds that show a lost key, a lost step of keys, or
probabilities of few bits, and with queries and keys of every magnitude.

Sequences share their pages here (a reused image), so that long caches stay small."""
import math

import pytest
import torch

from paper_2609_05821_amd import api
from tests import byte_oracle as B
from tests import mx_oracle as M
from tests.gpu_helpers import DEV
from tests.test_gpu_attn_byte import Store, check, queries, run
from tests.test_gpu_attn_mx_sharp import half_step
from tests.test_gpu_rotary import DT

pytestmark = pytest.mark.gpu


class Shared:
    """n_seqs sequences over the same pages: keys of magnitude 0.5 to 1.9, random values with
    scales of 2^-9 to 2^-7."""

    def __init__(self, n_seqs, ctx, hq, hkv, d, page=64, seed=0):
        g = torch.Generator().manual_seed(seed)
        per = -(-ctx // page)
        shape = (per + 2, hkv, page)
        self.n_seqs, self.ctx, self.hq, self.hkv, self.d = n_seqs, ctx, hq, hkv, d
        k = torch.randint(0x30, 0x40, (*shape, d), generator=g) + 128 * torch.randint(0, 2, (*shape, d), generator=g)
        v = torch.randint(0, 256, (*shape, d), generator=g)
        v[(v & 127) == 127] = 0x31
        scales = (per + 2, hkv, page // 16)
        cpu = [k.to(torch.uint8), v.to(torch.uint8), torch.full(scales, 127, dtype=torch.uint8),
               torch.randint(118, 121, scales, generator=g, dtype=torch.uint8)]
        table = torch.randperm(per + 2, generator=g)[:per].to(torch.int32)
        pages, slot = table[torch.arange(ctx) // page].long(), torch.arange(ctx) % page
        self.factors = B.factor(cpu[3][pages, :, slot // 16])                # of the values, [ctx, hkv]
        self.k = B.decoded(cpu[0][pages, :, slot])                           # float64 [ctx, hkv, d]
        self.v = B.decoded(cpu[1][pages, :, slot]) * self.factors[..., None]
        table = table[None].expand(n_seqs, per).contiguous()
        self.cache = api.byte_desc(*(t.to(DEV) for t in cpu), hq, ctx, table.to(DEV))

    def many(self, r, dtype):
        pairs = r * self.hq // self.hkv
        return dtype == torch.bfloat16 and pairs > (64 if self.d == 128 else 128) and \
            self.n_seqs * self.hkv * -(-pairs // 32) * self.ctx >= 2 ** 18

    def run(self, q, pos, scale=None):
        o = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
        lse = torch.full(q.shape[:2], 9.0, device=DEV)
        api.conduit_attn_byte(self.cache, q.to(DEV), pos.to(DEV), o, lse_out=lse, scale=scale)
        return o.cpu().double(), lse.cpu().double()


# (sequences, rows of each, query heads, KV heads, dims, keys): a workgroup of eight and of
# four waves per block, workgroups that share the steps, 32 pairs a block, 256 pairs, heads of
# 64 dims, more blocks than a wave lists, and of 256 pairs a workgroup per block, lists
# in LDS, as many blocks as a list holds and more; a row of more than 256 pairs, and 256 KV heads.
SHAPES = [(30, 1, 8, 2, 128, 1000), (130, 1, 8, 2, 128, 1000), (2, 4, 8, 2, 128, 9000), (12, 3, 14, 2, 128, 1500),
          (1, 700, 7, 1, 128, 4800), (40, 1, 8, 8, 64, 1000), (2, 4, 8, 2, 64, 6000), (1, 500, 8, 2, 64, 4100),
          (70, 1, 6, 2, 128, 2500), (70, 40, 4, 1, 128, 1100), (70, 40, 4, 1, 64, 1100), (300, 12, 7, 1, 128, 1300),
          (300, 12, 7, 1, 128, 2300), (300, 20, 7, 1, 64, 2300), (4096, 10, 7, 1, 128, 4200),
          (4200, 10, 7, 1, 128, 1100), (3, 1, 300, 1, 128, 30000), (1, 2, 512, 256, 64, 2300)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,ctx", SHAPES)
def test_one_key_of_all(dtype, n_seqs, r, hq, hkv, d, ctx):
    """Every query is one key of its own choice, so far above all others that the output is
    that key's value row: its logit is scale |k|^2, 1,380 in the mean, the others' a sum of d products of mean 0, 350
    below it or more.  Every 32 keys of every head have a target of their own.  (A weight rounded to 2^-11 leaves a
    value of 4 significant bits what it is once the output is rounded to 8.)"""
    st = Shared(n_seqs, ctx, hq, hkv, d, seed=ctx + d)
    n, scale = n_seqs * r, 1024.0 / d
    pos = torch.full((n,), ctx - 1, dtype=torch.int32)
    g = hq // hkv
    heads, pairs = (torch.arange(hq) // g).expand(n, hq), torch.arange(n)[:, None] * g + torch.arange(hq) % g
    apart = max(1, ctx // (n * g))
    for start in {*range(0, apart, 32), ctx // 2}:
        at = (pairs * apart + start) % ctx
        if start == ctx // 2:
            at[-1] = ctx - 1
        q = st.k[at, heads].to(DT[dtype])                                   # (exact)
        o, lse = st.run(q, pos, scale)
        want = st.v[at, heads]
        err = 0.0 if dtype == "bf16" else 2.0 ** -20
        bad = ((o - want).abs() > err * want.abs() + 1e-20).any(-1)
        assert not bad.any(), f"keys {at[bad].tolist()[:20]}"
        logit = scale * (st.k[at, heads] ** 2).sum(-1)
        assert ((lse - logit).abs() <= (2 * (d + 8) + 16) * 2.0 ** -24 * logit).all()


@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,ctx", [
    (4, 1, 8, 2, 128, 300), (3, 5, 8, 2, 128, 250), (1, 80, 4, 2, 128, 330), (4, 1, 8, 2, 64, 300),
    (1, 90, 4, 2, 64, 400), (2, 2, 8, 2, 128, 3000), (1, 400, 4, 2, 128, 5300), (9, 60, 8, 2, 64, 2000)])
def test_bf16_outputs_are_rounded_once(n_seqs, r, hq, hkv, d, ctx):
    """Half a step of the output's own rounding, and 2^-17 of each probability (many pairs: 2^-11, or what fp16 loses
    below its normal numbers): what is left of the error is that of 32-bit logits and sums."""
    st = Shared(n_seqs, ctx, hq, hkv, d, seed=ctx)
    q = queries(n_seqs * r, hq, d, "bf16", r)
    pos = torch.randint(ctx // 2, ctx, (n_seqs * r,), generator=torch.Generator().manual_seed(r), dtype=torch.int32)
    o, _ = st.run(q, pos)
    sel = torch.arange(n_seqs * r)[::max(1, n_seqs * r // 40)]
    want, lse, av, mag = M.attention(q[sel], st.k, st.v, pos[sel])
    bo, _ = B.attention_bounds(want, lse, av, mag, ctx, d, False)            # fp32: logits, exponentials, sums
    many = st.many(r, torch.bfloat16)
    err = bo + 2.0 ** (-11 if many else -17) * av
    if many:
        err = err + B.weight_floor(q[sel], st.k, st.v, st.factors, pos[sel], lse)
    bound = err + half_step(want.abs() + err)
    assert ((o[sel] - want).abs() <= bound).all(), f"{((o[sel] - want).abs() / bound).max():.3g} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r,hq,hkv", [(2, 1, 4, 2), (1, 40, 2, 1), (1, 300, 2, 1)])
def test_a_lost_step_shows(dtype, n_seqs, r, hq, hkv):
    """The log-sum-exp over 20,000 keys, within what its additions can lose: a lane adds an
    eighth of a wave's 32 keys of every 128 at most (n / 16 additions; with many pairs sums of 8 keys, n / 16 too, and 8
    within each), parts are merged after 256 keys at the least (n / 256), lanes, waves and changes of the maximum take
    fewer than 64.  The same bound is passed by none of the log-sum-exps that lack 32 keys side by
    side (the rows' queries are short, so that no key stands out)."""
    ctx, d = 20000, 128
    st = Shared(n_seqs, ctx, hq, hkv, d, page=256, seed=3)
    q = queries(n_seqs * r, hq, d, dtype, 4, spread=0.1)
    pos = torch.full((n_seqs * r,), ctx - 1, dtype=torch.int32)
    _, got = st.run(q, pos)
    pairs = [(i, h) for i in range(0, n_seqs * r, max(1, n_seqs * r // 6)) for h in range(hq)]
    scale = 1.0 / math.sqrt(d)
    for i, h in pairs:
        k = st.k[:, h // (hq // hkv)]
        logits = (k @ q[i, h].double()) * scale
        want = torch.logsumexp(logits, 0)
        mag = (k.abs() @ q[i, h].double().abs()).max() * scale
        bound = 2 * (d + 8) * 2.0 ** -24 * mag + 2 * 2.0 ** -22 + (ctx // 16 + ctx // 256 + 72) * 2.0 ** -24 + \
            2.0 ** -21 * want.abs()
        share = torch.exp(logits - want).view(-1, 32).sum(1)
        assert -torch.log1p(-share.min()) > 2 * bound
        off = (got[i, h] - want).abs()
        assert off <= bound, f"row {i}, head {h}: {off / bound:.3g} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 300), (3, 1500), (60, 1200)])
@pytest.mark.parametrize("log2", [-118, -100, 100, 106])
def test_small_and_large(dtype, r, ctx, log2):
    """Products that are ordinary: down to queries of 2^-118, whose smaller parts are subnormal in bf16."""
    st = Store(1, ctx, 4, 2, 128, seed=ctx)
    st.cpu[2][:] = 118 - log2
    st.upload()
    q = (queries(r, 4, 128, "f32", r).double() * 2.0 ** log2).to(DT[dtype])
    pos = torch.linspace(ctx - 1, ctx // 3, r).to(torch.int32)
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, q, pos, desc=desc)
        check(st, q, pos, o, lse, desc=desc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 300), (3, 1500), (60, 1200)])
def test_largest(dtype, r, ctx):
    """Queries up to the largest finite number (in fp32 it rounds up to an infinity in bf16), keys of subnormal codes
    with the smallest scale; values as large as sums of them allow."""
    st = Store(1, ctx, 4, 2, 128, seed=ctx)
    st.cpu[0] &= 0x87
    st.cpu[2][:] = 10
    st.cpu[3][:] = 225                                                      # 448 2^98 2^8 1,500 < 2^127
    st.upload()
    top = torch.finfo(DT[dtype]).max
    q = ((torch.rand(r, 4, 128, generator=torch.Generator().manual_seed(r), dtype=torch.float64) * 2 - 1) * top)
    q[:, :, ::50], q[:, :, 7::40] = top, -top
    q = q.to(DT[dtype])
    pos = torch.linspace(ctx - 1, ctx // 3, r).to(torch.int32)
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, q, pos, desc=desc)
        check(st, q, pos, o, lse, desc=desc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(3, 500), (60, 1200), (60, 9000)])
def test_smallest_values(dtype, r, ctx):
    """Values of the smallest scale, 2^-117, of which no output is lost: as over the same codes with scales of 1,
    times 2^-117 (codes of 1 to 480, so that outputs are normal numbers)."""
    outs = []
    for scale in (10, 127):
        st = Store(1, ctx, 4, 2, 128, seed=ctx)
        st.cpu[1] = (st.cpu[1] & 0x7f) | 0x38
        st.cpu[1][(st.cpu[1] & 127) == 127] = 0x7e
        st.cpu[3][:] = scale
        st.upload()
        q = queries(r, 4, 128, dtype, r)
        pos = torch.linspace(ctx - 1, ctx // 3, r).to(torch.int32)
        outs.append([run(st, q, pos, desc=desc)[0].double() for desc in st.descs(r, q.dtype)])
    for small, plain in zip(*outs):
        # both within half a step of their own rounding and the sums' 2^-16 and (bf16) weights' 2^-11, of terms that all add up
        assert (plain >= 1).all()
        apart = 2.0 ** -7 + 2.0 ** -10 if dtype == "bf16" else 2.0 ** -15
        assert ((small * 2.0 ** 117 - plain).abs() <= apart * plain).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("r,ctx", [(4, 900), (70, 700)])
def test_queries_that_are_not_finite_stay_in_their_rows(dtype, d, r, ctx):
    """A NaN or an infinity in one head of one row leaves every other output within its bounds."""
    st = Store(1, ctx, 6, 2, d, seed=r)
    q = queries(r, 6, d, dtype, 3)
    pos = torch.randint(0, ctx, (r,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    bad = q.clone()
    bad[1, 2, 5], bad[3, 0, 0], bad[r - 1, 5, 1] = math.nan, math.inf, -math.inf
    for desc in st.descs(r, q.dtype):
        o, lse = run(st, bad, pos, desc=desc)
        for i, h in ((1, 2), (3, 0), (r - 1, 5)):
            assert not lse[i, h].isfinite() and o[i, h].isnan().any()
        clean, clean_lse = run(st, q, pos, desc=desc)
        for i, h in ((1, 2), (3, 0), (r - 1, 5)):
            o[i, h], lse[i, h] = clean[i, h], clean_lse[i, h]
        check(st, q, pos, o, lse, desc=desc)
