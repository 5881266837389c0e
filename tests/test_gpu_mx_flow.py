"""The operators together, as a serving loop uses them: a prompt packed into a 4-bit
cache, its selected rows refreshed, tokens decoded in a batch, and a stored
image loaded into another request's cache at another place and scored there."""
import numpy as np
import pytest
import torch

from oracle import conduit_oracle as O
from paper_2609_05821_amd import api
from tests import mx_oracle as M
from tests.gpu_helpers import DEV, assert_scores, to_f64
from tests.test_gpu_rotary import rope_of

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE = 14, 2, 128, 64


def tokens(n, seed):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(n, HQ + 2 * HKV, D, generator=g).to(torch.bfloat16).to(DEV)
    return qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]


def pools(n_pages):
    return [torch.full((n_pages, HKV, PAGE, b), 255, dtype=torch.uint8, device=DEV)
            for b in (D // 2, D // 2, D // 32, D // 32)]


def test_prompt_refresh_decode():
    lengths, budget, steps = [500, 37, 129], 60, 5
    n_seqs, per = len(lengths), 16
    p = pools(n_seqs * per + 1)                               # one page never used: all bytes 255
    table = torch.randperm(n_seqs * per, generator=torch.Generator().manual_seed(0)).to(torch.int32).view(n_seqs, per)
    rope = rope_of(D // 2, 3)
    tab = table.to(DEV)
    whole = api.mx_desc(*p, HQ, per * PAGE, tab)
    one = [api.mx_desc(*p, HQ, per * PAGE, tab[s:s + 1]) for s in range(n_seqs)]
    keys, values = [], []                                     # the oracle's cache, float64

    def packed(k, v, rp):
        kc, ks, vc, vs = M.pack_rows(M.rounded(M.turned(k.cpu(), rope.inv_freq, rope.axis, rp.cpu()), torch.bfloat16),
                                     v.cpu())
        return M.held(kc, ks), M.held(vc, vs)

    def attend_check(q, rp, s, pos, got):
        qt = M.rounded(M.turned(q.cpu(), rope.inv_freq, rope.axis, rp.cpu()), torch.bfloat16)
        want = M.attention(qt, keys[s], values[s], pos)
        bo, _ = M.attention_bounds(*want, len(keys[s]), D, True)
        # the queries' own rounding may fall on the other side of a border where the
        # turn in 64 bits is within 2^-40 of it: none of these inputs does
        assert ((got.cpu().double() - want[0]).abs() <= bo).all()

    for s, n in enumerate(lengths):                           # prompts, one by one
        q, k, v = tokens(n, s)
        rp = torch.stack([torch.arange(n) // 64, torch.arange(n) % 64, torch.arange(n)]).to(torch.int32).to(DEV)
        pos = torch.arange(n, dtype=torch.int32, device=DEV)
        qo, o = torch.empty(n, HQ, D, dtype=q.dtype, device=DEV), torch.empty(n, HQ, D, dtype=q.dtype, device=DEV)
        api.conduit_append_mx(one[s], pos, k, v, rope=rope, rope_pos=rp, q=q, q_out=qo)
        api.conduit_attn_mx(one[s], qo, pos, o)
        kk, vv = packed(k, v, rp)
        keys.append(kk)
        values.append(vv)
        rows = torch.tensor([0, 1, n // 2, n - 1])
        attend_check(q[rows.to(DEV)], rp[:, rows.to(DEV)], s, rows, o[rows.to(DEV)])

    sel = torch.randperm(lengths[0], generator=torch.Generator().manual_seed(1))[:budget].sort().values
    q, k, v = tokens(budget, 77)                              # the refreshed rows of the first prompt
    rp = sel.to(torch.int32)[None].repeat(3, 1).to(DEV)
    qo, o = torch.empty(budget, HQ, D, dtype=q.dtype, device=DEV), torch.empty(budget, HQ, D, dtype=q.dtype, device=DEV)
    pos = sel.to(torch.int32).to(DEV)
    api.conduit_append_mx(one[0], pos, k, v, rope=rope, rope_pos=rp, q=q, q_out=qo)
    api.conduit_attn_mx(one[0], qo, pos, o)
    kk, vv = packed(k, v, rp)
    keys[0][sel], values[0][sel] = kk, vv
    attend_check(q, rp, 0, sel, o)

    pos = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    for step in range(steps):                                 # a decoding batch; sequence 1 ends after two tokens
        if step == 2:
            pos[1] = -1
        q, k, v = tokens(n_seqs, 1000 + step)
        rp = torch.full((3, n_seqs), 600 + step, dtype=torch.int32, device=DEV)
        qo, o = torch.empty(n_seqs, HQ, D, dtype=q.dtype, device=DEV), torch.empty(n_seqs, HQ, D, dtype=q.dtype, device=DEV)
        api.conduit_append_mx(whole, pos, k, v, rope=rope, rope_pos=rp, q=q, q_out=qo)
        api.conduit_attn_mx(whole, qo, pos, o)
        kk, vv = packed(k, v, rp)
        for s in range(n_seqs):
            if s == 1 and step >= 2:
                assert (o[1] == 0).all()
                continue
            keys[s], values[s] = torch.cat((keys[s], kk[s:s + 1])), torch.cat((values[s], vv[s:s + 1]))
            attend_check(q[s:s + 1], rp[:, s:s + 1], s, pos[s:s + 1].cpu(), o[s:s + 1])
        pos = torch.where(pos >= 0, pos + 1, pos)
    assert all((x[-1] == 255).all() for x in p)               # the page that no sequence owns


def test_stored_image_moved_and_scored():
    """An image stored in 4 bits is loaded into a request's bf16 cache 300 tokens later;
    its keys there equal a turn by the sum of both positions up to the cache's
    roundings, the scoring pass reads them, and the 16-bit refresh attention over
    the loaded cache agrees with attention over the 4-bit one."""
    n, shift, n_q = 256, 300, 8
    rope = rope_of(D // 2, 1)
    p = pools(n // PAGE)
    mx = api.mx_desc(*p, HQ)
    _, k, v = tokens(n, 5)
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    api.conduit_append_mx(mx, pos, k, v, rope=rope, rope_pos=pos)
    n_ctx = shift + n + n_q
    _, ck, cv = tokens(n_ctx, 6)
    ck, cv = ck.contiguous(), cv.contiguous()
    kv = api.kv_desc(ck, cv, HQ)
    moved = torch.full((n,), shift, dtype=torch.int32, device=DEV)
    api.conduit_load_mx(mx, pos, kv, pos + shift, rope=rope, rope_pos=moved)
    base = M.held(p[0].cpu(), p[2].cpu()).transpose(1, 2).reshape(n, HKV, D)
    want = M.turned(base, rope.inv_freq, rope.axis, moved.cpu()[None])
    assert torch.equal(ck[shift:shift + n].cpu(), M.rounded(want, torch.bfloat16))
    # scoring reads the loaded rows
    q = torch.randn(n_q, HQ, D, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    img = api.ImageTable([shift], [0, n])
    s_acc, a_acc = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    api.conduit_score(kv, q.to(DEV), shift + n, img, s_acc, a_acc)
    a, vn, _ = O.score_layer(to_f64(q), to_f64(ck), to_f64(cv), shift + n, np.array([shift]), np.array([0, n]))
    assert_scores(to_f64(a_acc), a, what="a")
    assert_scores(to_f64(s_acc), a * vn, what="s")
    # without a turn the loaded cache holds exactly the 4-bit values: both attentions agree
    lk, lv = torch.empty(n, HKV, D, dtype=torch.bfloat16, device=DEV), torch.empty(n, HKV, D, dtype=torch.bfloat16, device=DEV)
    api.conduit_load_mx(mx, pos, api.kv_desc(lk, lv, HQ), pos)
    rows = torch.arange(3, n, 17, dtype=torch.int32, device=DEV)
    q = torch.randn(len(rows), HQ, D, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(DEV)
    o16, o4 = torch.empty_like(q), torch.empty_like(q)
    api.conduit_refresh_attn(api.kv_desc(lk, lv, HQ), q, rows, o16)
    api.conduit_attn_mx(mx, q, rows, o4)
    want = M.attention(q.cpu(), lk.cpu().double(), lv.cpu().double(), rows.cpu())
    bo, _ = M.attention_bounds(*want, n, D, True)
    assert ((o4.cpu().double() - want[0]).abs() <= bo).all()
    assert ((o4.cpu().double() - o16.cpu().double()).abs() <= 2 * bo).all()


def test_positions_then_scatter_equals_append():
    """conduit_append_kv is conduit_rotary followed by conduit_scatter_kv, bit for bit."""
    n = 100
    q, k, v = tokens(n, 3)
    rope, rp = rope_of(D // 2, 3), torch.randint(0, 999, (3, n), generator=torch.Generator().manual_seed(1),
                                                 dtype=torch.int32).to(DEV)
    caches = [torch.zeros(200, HKV, D, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    pos = torch.randperm(200, generator=torch.Generator().manual_seed(2))[:n].to(torch.int32).to(DEV)
    kt = torch.empty(n, HKV, D, dtype=torch.bfloat16, device=DEV)
    api.conduit_rotary(k, rope, rp, kt)
    api.conduit_scatter_kv(api.kv_desc(caches[0], caches[1], HQ), pos, kt, v.contiguous())
    api.conduit_append_kv(api.kv_desc(caches[2], caches[3], HQ), pos, k, v, rope=rope, rope_pos=rp)
    assert torch.equal(caches[0], caches[2]) and torch.equal(caches[1], caches[3])


def test_captured_decode_step():
    """Append and attention of a decoding step in one captured graph, positions moved by
    the program between replays; the eager loop gives the same bits."""
    n_seqs, per, steps = 3, 4, 6
    tab = torch.randperm(n_seqs * per, generator=torch.Generator().manual_seed(3)).to(torch.int32).view(n_seqs, per).to(DEV)
    rope = rope_of(D // 2, 1)
    start = [100, 5, 63]

    def loop(graphed):
        p = pools(n_seqs * per)
        mx = api.mx_desc(*p, HQ, per * PAGE, tab)
        for s in range(n_seqs):
            t1 = tab[s:s + 1].contiguous()
            m1 = api.mx_desc(*p, HQ, per * PAGE, t1)
            _, k, v = tokens(start[s], 50 + s)
            ids = torch.arange(start[s], dtype=torch.int32, device=DEV)
            api.conduit_append_mx(m1, ids, k, v, rope=rope, rope_pos=ids)
            torch.cuda.synchronize()
        pos = torch.tensor(start, dtype=torch.int32, device=DEV)
        buf = torch.empty(n_seqs, HQ + 2 * HKV, D, dtype=torch.bfloat16, device=DEV)
        q, k, v = buf[:, :HQ], buf[:, HQ:HQ + HKV], buf[:, HQ + HKV:]
        qo, o = (torch.empty(n_seqs, HQ, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ws = torch.empty(max(1, api.attn_mx_workspace_bytes(mx, qo)), dtype=torch.uint8, device=DEV)

        def step():
            api.conduit_append_mx(mx, pos, k, v, rope=rope, rope_pos=pos, q=q, q_out=qo)
            api.conduit_attn_mx(mx, qo, pos, o, ws=ws)
        if graphed:
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr):
                step()
        outs = []
        for i in range(steps):
            buf.copy_(torch.cat([t for t in tokens(n_seqs, 200 + i)], 1))
            torch.cuda.synchronize()
            gr.replay() if graphed else step()
            torch.cuda.synchronize()
            outs.append(o.clone())
            pos += 1
        return outs, p

    eager, pe = loop(False)
    graphed, pg = loop(True)
    for a, b in zip(eager, graphed):
        assert torch.equal(a, b)
    assert all(torch.equal(a, b) for a, b in zip(pe, pg))
