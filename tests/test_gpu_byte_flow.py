"""The 8-bit cache's operators together, as a serving loop uses them: prompts packed, selected
rows of one refreshed, tokens decoded in a batch, a stored image loaded into another
request's cache at another place and scored there, and an encoder's states attended to."""
import numpy as np
import pytest
import torch

from oracle import conduit_oracle as O
from paper_2609_05821_amd import api
from tests import byte_oracle as B
from tests import mx_oracle as M
from tests.gpu_helpers import DEV, assert_scores, to_f64
from tests.test_gpu_rotary import rope_of

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE = 14, 2, 128, 64


def tokens(n, seed, dtype=torch.bfloat16, grow=1.0):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(n, HQ + 2 * HKV, D, generator=g) * grow).to(dtype).to(DEV)
    return qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]


def pools(n_pages):
    return [torch.full((n_pages, HKV, PAGE, D), 255, dtype=torch.uint8, device=DEV) for _ in range(2)] + \
        [torch.full((n_pages, HKV, PAGE // 16), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]


def turned(x, rope, rp):
    """Rows as the cache's dtype holds them turned.  (fp32: conduit_rotary's, whose last bit may differ from that of
    a turn in 64 bits and decide a code.)"""
    if x.dtype == torch.float32:
        out = torch.empty(x.shape, device=DEV)
        api.conduit_rotary(x, rope, rp, out)
        return out.cpu()
    return M.rounded(M.turned(x.cpu(), rope.inv_freq, rope.axis, rp.cpu()), x.dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompt_refresh_decode(dtype):
    lengths, budget, steps = [500, 37, 129], 60, 5
    n_seqs, per = len(lengths), 16
    p = pools(n_seqs * per + 1)                               # one page never used: all bytes 255
    table = torch.randperm(n_seqs * per, generator=torch.Generator().manual_seed(0)).to(torch.int32).view(n_seqs, per)
    rope, tab = rope_of(D // 2, 3), table.to(DEV)
    whole = api.byte_desc(*p, HQ, per * PAGE, tab)
    one = [api.byte_desc(*p, HQ, per * PAGE, tab[s:s + 1]) for s in range(n_seqs)]
    cpu = [x.cpu() for x in p]
    model = [B.Pools(cpu[0], cpu[1], cpu[2], cpu[3], table[s:s + 1], PAGE, per * PAGE) for s in range(n_seqs)]

    def step(desc, q, k, v, rp, pos, held=None):
        """One call of each operator."""
        n = len(pos)
        qo, o = torch.empty(n, HQ, D, dtype=dtype, device=DEV), torch.empty(n, HQ, D, dtype=dtype, device=DEV)
        api.conduit_append_byte(desc, pos, k, v, n_held=held, rope=rope, rope_pos=rp, q=q, q_out=qo)
        api.conduit_attn_byte(desc, qo, pos, o)
        return o

    def follow(s, q, k, v, rp, pos, o, held=None, sample=None):
        """The oracle's cache and attention of sequence s."""
        model[s].append(pos.cpu(), turned(k, rope, rp), v.cpu(), None if held is None else held.cpu())
        sel = torch.arange(len(pos)) if sample is None else sample
        at = pos.cpu()[sel]
        keys, values = model[s].rows(0, int(at.max()) + 1)
        want = M.attention(turned(q, rope, rp)[sel], keys, values, at)
        bo, _ = B.attention_bounds(*want, len(keys), D, dtype == torch.bfloat16)
        assert ((o.cpu()[sel].double() - want[0]).abs() <= bo).all()

    for s, n in enumerate(lengths):                           # prompts, one by one, the first in two pieces
        for lo, hi in ((0, 203), (203, n)) if s == 0 else ((0, n),):
            q, k, v = tokens(hi - lo, 10 * s + lo, dtype)
            at = torch.arange(lo, hi)
            rp = torch.stack([at // 64, at % 64, at]).to(torch.int32).to(DEV)
            pos = at.to(torch.int32).to(DEV)
            o = step(one[s], q, k, v, rp, pos)
            follow(s, q, k, v, rp, pos, o, sample=torch.tensor([0, 1, (hi - lo) // 2, hi - lo - 1]))

    sel = torch.randperm(lengths[0], generator=torch.Generator().manual_seed(1))[:budget].sort().values
    q, k, v = tokens(budget, 77, dtype, grow=3.0)             # the refreshed rows of the first prompt: larger values
    rp = sel.to(torch.int32)[None].repeat(3, 1).to(DEV)
    pos, held = sel.to(torch.int32).to(DEV), torch.tensor([lengths[0]], dtype=torch.int32, device=DEV)
    o = step(one[0], q, k, v, rp, pos, held)
    follow(0, q, k, v, rp, pos, o, held)

    pos = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    for i in range(steps):                                    # a decoding batch; sequence 1 ends after two tokens
        if i == 2:
            pos[1] = -1
        q, k, v = tokens(n_seqs, 1000 + i, dtype, grow=1.0 + i)
        rp = torch.full((3, n_seqs), 600 + i, dtype=torch.int32, device=DEV)
        o = step(whole, q, k, v, rp, pos)
        for s in range(n_seqs):
            if s == 1 and i >= 2:
                assert (o[1] == 0).all()
                continue
            follow(s, q[s:s + 1], k[s:s + 1], v[s:s + 1], rp[:, s:s + 1], pos[s:s + 1], o[s:s + 1])
        pos = torch.where(pos >= 0, pos + 1, pos)
    assert all((x[-1] == 255).all() for x in p)               # the page that no sequence owns
    for s in range(n_seqs):                                   # every byte that a token has is the oracle's
        t = torch.arange(lengths[s] + (2 if s == 1 else steps))
        page, slot = table[s][t // PAGE].long(), t % PAGE
        for name, i in (("k", 0), ("v", 1)):
            codes, scales = model[s].pool[name]
            assert torch.equal(p[i].cpu()[page, :, slot], codes[page, :, slot])
            assert torch.equal(p[i + 2].cpu()[page, :, slot // 16], scales[page, :, slot // 16])


def test_stored_image_moved_and_scored():
    """An image stored in 8 bits is loaded into a request's bf16 cache 300 tokens later; the scoring
    pass reads it there, and the 16-bit refresh attention over the loaded cache agrees with
    attention over the 8-bit one."""
    n, shift, n_q = 256, 300, 8
    rope = rope_of(D // 2, 1)
    p = pools(n // PAGE)
    cache = api.byte_desc(*p, HQ)
    _, k, v = tokens(n, 5)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    api.conduit_append_byte(cache, pos, k, v, rope=rope, rope_pos=pos)
    n_ctx = shift + n + n_q
    _, ck, cv = tokens(n_ctx, 6)
    ck, cv = ck.contiguous(), cv.contiguous()
    kv = api.kv_desc(ck, cv, HQ)
    moved = torch.full((n,), shift, dtype=torch.int32, device=DEV)
    api.conduit_load_byte(cache, pos, kv, pos + shift, rope=rope, rope_pos=moved)
    cpu = [x.cpu() for x in p]
    base, vals = B.Pools(cpu[0], cpu[1], cpu[2], cpu[3], torch.arange(n // PAGE)[None], PAGE, n).rows(0, n)
    want = M.turned(base, rope.inv_freq, rope.axis, moved.cpu()[None])
    assert torch.equal(ck[shift:shift + n].cpu(), M.rounded(want, torch.bfloat16))
    assert torch.equal(cv[shift:shift + n].cpu().double(), vals)
    q = torch.randn(n_q, HQ, D, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    img = api.ImageTable([shift], [0, n])
    s_acc, a_acc = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    api.conduit_score(kv, q.to(DEV), shift + n, img, s_acc, a_acc)
    a, vn, _ = O.score_layer(to_f64(q), to_f64(ck), to_f64(cv), shift + n, np.array([shift]), np.array([0, n]))
    assert_scores(to_f64(a_acc), a, what="a")
    assert_scores(to_f64(s_acc), a * vn, what="s")
    # without a turn the loaded cache holds exactly the 8-bit values: both attentions agree
    lk, lv = (torch.empty(n, HKV, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    api.conduit_load_byte(cache, pos, api.kv_desc(lk, lv, HQ), pos)
    rows = torch.arange(3, n, 17, dtype=torch.int32, device=DEV)
    q = torch.randn(len(rows), HQ, D, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(DEV)
    o16, o8 = torch.empty_like(q), torch.empty_like(q)
    api.conduit_refresh_attn(api.kv_desc(lk, lv, HQ), q, rows, o16)
    api.conduit_attn_byte(cache, q, rows, o8)
    want = M.attention(q.cpu(), lk.cpu().double(), lv.cpu().double(), rows.cpu())
    bo, _ = B.attention_bounds(*want, n, D, True)
    assert ((o8.cpu().double() - want[0]).abs() <= bo).all()
    # (16-bit attention rounds its probabilities to bf16, 2^-8 of each where this one has 2^-11, so its own bound is
    # wider; both are off by their bounds at most)
    b16, _ = M.attention_bounds(*want, n, D, True)
    assert ((o8.cpu().double() - o16.cpu().double()).abs() <= bo + b16).all()


def test_an_encoders_states():
    """States of two requests, of different lengths and without positions, appended once; a text's
    rows attend to all of theirs."""
    lengths, r, per = [700, 90], 40, 12
    p = pools(2 * per)
    table = torch.randperm(2 * per, generator=torch.Generator().manual_seed(3)).to(torch.int32).view(2, per)
    cache = api.byte_desc(*p, HQ, per * PAGE, table.to(DEV))
    n = max(lengths)
    _, k, v = tokens(2 * n, 21)
    at = torch.arange(n)
    pos = torch.cat([torch.where(at < x, at, -1) for x in lengths]).to(torch.int32)
    api.conduit_append_byte(cache, pos.to(DEV), k, v)
    cpu = [x.cpu() for x in p]
    model = B.Pools(cpu[0], cpu[1], cpu[2], cpu[3], table, PAGE, per * PAGE)
    q = torch.randn(2 * r, HQ, D, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    o = torch.empty(2 * r, HQ, D, dtype=torch.bfloat16, device=DEV)
    last = torch.tensor(lengths).repeat_interleave(r).to(torch.int32) - 1
    api.conduit_attn_byte(cache, q.to(DEV), last.to(DEV), o)
    for s, length in enumerate(lengths):
        keys, values = model.rows(s, length)
        fresh = k[s * n:s * n + length].cpu().double()
        assert ((keys - fresh).abs() <= 2.0 ** -4 * fresh.abs() + 2.0 ** -10 * fresh.abs().amax()).all()
        sel = torch.arange(0, r, 7)
        want = M.attention(q[s * r:(s + 1) * r][sel], keys, values, last[s * r:(s + 1) * r][sel])
        bo, _ = B.attention_bounds(*want, length, D, True)
        assert ((o[s * r:(s + 1) * r].cpu()[sel].double() - want[0]).abs() <= bo).all()


@pytest.mark.parametrize("r", [1, 300])
def test_pages_past_32_bits(r):
    """Pages 2^28 bytes apart, 5 GiB of them: every call as over dense pools, whose pages lie together."""
    n, stride, far = 900, 1 << 28, [17, 1, 19, 16, 8, 18, 3, 12, 0, 14, 9, 2, 15, 5, 4]
    table = torch.tensor(far, dtype=torch.int32)[None].to(DEV)
    dense = pools(20)
    flat = [torch.empty(20 * stride, dtype=torch.uint8, device=DEV) for _ in range(2)]
    wide = [x.as_strided((20, HKV, PAGE, D), (stride, PAGE * D, D, 1)) for x in flat] + pools(20)[2:]
    for x in wide[:2]:
        x.fill_(255)
    _, k, v = tokens(n, 31)
    q = torch.randn(r, HQ, D, generator=torch.Generator().manual_seed(r)).to(torch.bfloat16).to(DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    at = torch.arange(r, dtype=torch.int32, device=DEV) * (n // r) + n // r - 1
    got = []
    for p in (dense, wide):
        cache = api.byte_desc(*p, HQ, len(far) * PAGE, table)
        api.conduit_append_byte(cache, pos, k, v)
        o, lse = torch.empty_like(q), torch.empty(r, HQ, device=DEV)
        api.conduit_attn_byte(cache, q, at, o, lse_out=lse)
        room = torch.zeros(1, 512, dtype=torch.int32, device=DEV)          # blocks of 256 pairs, where there are many
        room[:, :len(far)] = table
        o2, lse2 = torch.empty_like(q), torch.empty(r, HQ, device=DEV)
        api.conduit_attn_byte(api.byte_desc(*p, HQ, 512 * PAGE, room), q, at, o2, lse_out=lse2)
        lk, lv = (torch.empty(n, HKV, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        api.conduit_load_byte(cache, pos, api.kv_desc(lk, lv, HQ), pos)
        got.append((p[0].clone(), p[1].clone(), p[2], p[3], o, lse, o2, lse2, lk, lv))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    # both kinds of blocks saw the same keys (a row's sum of |q||k| over sqrt(128) stays below 11 here: log-sum-exps
    # are within 2 * 136 * 2^-24 * 11 + 2^-21 + 2 * 964 * 2^-24 < 3.1e-4 of 64 bits)
    assert (got[0][5] - got[0][7]).abs().max() <= 6.2e-4
