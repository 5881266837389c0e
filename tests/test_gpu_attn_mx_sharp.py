"""Attention over a 4-bit cache with bounds that show a lost key, a lost step of keys, or
probabilities of few bits.

Sequences share their pages here (a reused image), so that long caches stay small."""
import math

import pytest
import torch

from paper_2609_05821_amd import api
from tests import mx_oracle as M
from tests.gpu_helpers import DEV
from tests.test_gpu_attn_mx import queries
from tests.test_gpu_rotary import DT

pytestmark = pytest.mark.gpu


class Shared:
    """n_seqs sequences over the same pages: random codes, key scales of 2^-2, value scales of
    2^-3 to 2^-1."""

    def __init__(self, n_seqs, ctx, hq, hkv, d, page=64, seed=0):
        g = torch.Generator().manual_seed(seed)
        per = -(-ctx // page)
        shape = (per + 2, hkv, page)
        self.n_seqs, self.ctx, self.hq, self.hkv, self.d = n_seqs, ctx, hq, hkv, d
        cpu = [torch.randint(0, 256, (*shape, d // 2), generator=g, dtype=torch.uint8) for _ in range(2)] + \
              [torch.full((*shape, d // 32), 125, dtype=torch.uint8),
               torch.randint(124, 127, (*shape, d // 32), generator=g, dtype=torch.uint8)]
        table = torch.randperm(per + 2, generator=g)[:per].to(torch.int32)[None]
        pos, seq = torch.arange(ctx), torch.zeros(ctx, dtype=torch.long)
        self.k, self.v = (M.held(M.gather(cpu[i], table, seq, pos, page), M.gather(cpu[i + 2], table, seq, pos, page))
                          for i in (0, 1))                                   # float64 [ctx, hkv, d]
        self.mx = api.mx_desc(*(t.to(DEV) for t in cpu), hq, ctx, table.expand(n_seqs, per).contiguous().to(DEV))

    def run(self, q, pos, scale=None):
        o = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
        lse = torch.full(q.shape[:2], 9.0, device=DEV)
        api.conduit_attn_mx(self.mx, q.to(DEV), pos.to(DEV), o, lse_out=lse, scale=scale)
        return o.cpu().double(), lse.cpu().double()


# (sequences, rows of each, query heads, KV heads, dims, keys): a workgroup of eight and of
# four waves per block, workgroups that share the steps, 32 pairs a block, many pairs, heads
# of 64 dims, more blocks than a wave lists, many pairs with as many and with more than their
# lists hold.
SHAPES = [(30, 1, 8, 2, 128, 1000), (130, 1, 8, 2, 128, 1000), (2, 4, 8, 2, 128, 9000), (12, 3, 14, 2, 128, 1500),
          (1, 700, 7, 1, 128, 4800), (40, 1, 8, 8, 64, 1000), (2, 4, 8, 2, 64, 6000), (1, 500, 8, 2, 64, 4100),
          (70, 1, 6, 2, 128, 2500), (70, 40, 4, 1, 128, 1100), (70, 40, 4, 1, 64, 1100), (2060, 5, 7, 1, 128, 1100)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,ctx", SHAPES)
def test_one_key_of_all(dtype, n_seqs, r, hq, hkv, d, ctx):
    """Every query is one key of its own choice, so far above all others that the output is
    that key's value row: its logit is scale |k|^2, 550 in the mean, the others' a sum of d
    products of mean 0 (50 at the least below it).  Every 32 keys of every
    head have a target of their own."""
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


def half_step(x):
    """Half a step of bf16 at the magnitude x (8 significant bits)."""
    return torch.pow(2.0, torch.floor(torch.log2(x.clamp_min(2.0 ** -120))) - 8)


@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,ctx", [(4, 1, 8, 2, 128, 300), (3, 5, 8, 2, 128, 250), (1, 80, 4, 2, 128, 330),
                                                   (4, 1, 8, 2, 64, 300), (1, 90, 4, 2, 64, 400), (2, 2, 8, 2, 128, 3000)])
def test_bf16_outputs_are_rounded_once(n_seqs, r, hq, hkv, d, ctx):
    """Half a step of the output's own rounding, and 2^-17 of each probability: what is
    left of the error is that of 32-bit logits and sums."""
    st = Shared(n_seqs, ctx, hq, hkv, d, seed=ctx)
    q = queries(n_seqs * r, hq, d, "bf16", r)
    pos = torch.randint(ctx // 2, ctx, (n_seqs * r,), generator=torch.Generator().manual_seed(r), dtype=torch.int32)
    o, _ = st.run(q, pos)
    want, lse, av, mag = M.attention(q, st.k, st.v, pos)
    bo, _ = M.attention_bounds(want, lse, av, mag, ctx, d, False)            # fp32: logits, exponentials, sums
    err = bo + 2.0 ** -17 * av
    bound = err + half_step(want.abs() + err)
    assert ((o - want).abs() <= bound).all(), f"{((o - want).abs() / bound).max():.3g} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seqs,r,hq,hkv", [(2, 1, 4, 2), (1, 40, 2, 1)])
def test_a_lost_step_shows(dtype, n_seqs, r, hq, hkv):
    """The log-sum-exp over 20,000 keys, within what its additions can lose: a lane adds an
    eighth of a wave's 32 keys of every 128 at most (n / 16 additions), parts are merged after
    256 keys at the least (n / 256), lanes, waves and changes of the maximum take fewer than
    64.  The same bound is passed by none of the log-sum-exps that lack 32 keys side by
    side (the rows' queries are short, so that no key stands out)."""
    ctx, d = 20000, 128
    st = Shared(n_seqs, ctx, hq, hkv, d, page=256, seed=3)
    q = queries(n_seqs * r, hq, d, dtype, 4, spread=0.25)
    pos = torch.full((n_seqs * r,), ctx - 1, dtype=torch.int32)
    _, got = st.run(q, pos)
    pairs = [(i, h) for i in range(0, n_seqs * r, max(1, n_seqs * r // 6)) for h in range(hq)]
    scale = 1.0 / math.sqrt(d)
    for i, h in pairs:
        k = st.k[:, h // (hq // hkv)]
        logits = (k @ q[i, h].double()) * scale
        want = torch.logsumexp(logits, 0)
        mag = (k.abs() @ q[i, h].double().abs()).max() * scale
        bound = 2 * (d + 8) * 2.0 ** -24 * mag + 2 * 2.0 ** -22 + (ctx // 16 + ctx // 256 + 64) * 2.0 ** -24 + \
            2.0 ** -21 * want.abs()
        share = torch.exp(logits - want).view(-1, 32).sum(1)
        assert -torch.log1p(-share.min()) > 2 * bound
        assert (got[i, h] - want).abs() <= bound, f"row {i}, head {h}: {(got[i, h] - want).abs() / bound:.3g} of the bound"
