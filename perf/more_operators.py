"""A cache held in 8 bits, as cases that can be timed and checked.

A case is a dict of plain values; ``prepare`` makes its inputs on the GPU from a
seed, ``run`` makes one pass, and ``exact`` gives the outputs of that pass from
the definitions in 64 bits.  With ``own`` false ``run`` computes the operators
in elementary torch operations; with ``own`` true it calls the package.  The
kinds of case:

  append_byte  new (or recomputed) keys and values into a cache held in 8 bits,
               quantised as they are written, the keys (and the queries of the
               same tokens) rotated on the way;
  load_byte    rows of such a cache into a cache of 16 or 32 bits, the keys
               rotated by the distance that they move;
  attn_byte    attention over such a cache.

The 8-bit cache: a scale byte s for each block of 16 tokens and head, and codes
c in e4m3 (sign, 4 exponent bits, 3 mantissa bits, up to 448); the value is
c * 2^(s - 127).  The rows that an append writes into a block need the smallest
s with max|x| <= 448 * 2^(s - 127), kept between 10 and 246; where the block
keeps tokens from before, its scale never falls, and where it rises the kept
codes are rounded to it.  Kept are the tokens below the sequence's ``n_held``,
or, where that is not given, those before the last row that the block receives.
Codes are the nearest, ties to the even code.  Pools are [page][head][slot][d]
codes and [page][head][slot / 16] scales.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
HALVES, ADJACENT = 0, 1
BLOCK = 16                      # tokens that share a scale
SCALE_MIN, SCALE_MAX = 10, 246
CODE_MAX = 448.0


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _case(kind, **kw):
    c = dict(kind=kind, dtype="bf16", n_seqs=1, rows=1, hq=28, hkv=4, d=128, ctx=0, page=64, rot=128, axes=3,
             pairing=HALVES, with_q=True, held=False, spread=False, ragged=False, cross=False, pad=0)
    c.update(kw)
    return c


def listed():
    return [
        # A decoding batch: one token each of 64 sequences of up to 1,024 tokens (two of them padding), handed
        # back as the cache holds them.
        _case("append_byte", name="append_decode", n_seqs=64, rows=1, ctx=1024, ragged=True, pad=2, held=True),
        # A refresh step's rows (10% of 16k visual tokens) written over stale ones: blocks of kept and new tokens.
        _case("append_byte", name="append_refresh", rows=1638, ctx=17024, spread=True),
        # A whole 16k multi-image prompt, one layer.
        _case("append_byte", name="append_prompt", rows=17024, ctx=17024),
        # A long document's fp32 keys and values packed for reuse.
        _case("append_byte", name="append_document_f32", dtype="f32", rows=65536, ctx=65536, with_q=False),
        # One image of a store loaded into a request's fp32 cache, its keys moved to their new place.
        _case("load_byte", name="load_image_f32", dtype="f32", rows=1024, ctx=1344),
        # A long document loaded into a bf16 cache.
        _case("load_byte", name="load_document", rows=65536, ctx=66048),
        # One token, fp32, one image of context, 8 heads of 64: the smallest attention.
        _case("attn_byte", name="attn_token_f32", dtype="f32", hq=8, hkv=8, d=64, ctx=672),
        # A decoding batch of 64 ragged sequences of up to 32k tokens (two of them padding).
        _case("attn_byte", name="attn_decode", n_seqs=64, ctx=32768, ragged=True, pad=2),
        # One token of a single very long sequence.
        _case("attn_byte", name="attn_long", hq=32, hkv=8, ctx=131072),
        # Five drafted tokens of each of 8 sequences verified at once, an odd context.
        _case("attn_byte", name="attn_draft", n_seqs=8, rows=5, hq=32, hkv=8, ctx=8211, ragged=True),
        # Text rows of 4 requests attending to all of an encoder's states, whose number differs by request.
        _case("attn_byte", name="attn_cross", n_seqs=4, rows=333, hq=32, hkv=8, ctx=4100, ragged=True, cross=True),
        # The refresh step's selected rows (10% of 16k visual tokens).
        _case("attn_byte", name="attn_refresh", rows=1638, ctx=17024, spread=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["append_byte", "append_byte", "load_byte", "attn_byte", "attn_byte", "attn_byte"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 5, 7, 8])
    page = rng.choice([64, 128, 256])
    axes = rng.choice([1, 2, 3, 4])
    pairing = rng.choice([HALVES, HALVES, ADJACENT])
    if kind != "attn_byte":
        with_q = kind == "append_byte" and rng.random() < 0.6
        per_row = (hq if with_q else 0) + 2 * hkv
        rot = rng.choice([d, d, d // 2])
        spread, n_seqs, how = False, 1, rng.random()
        if kind == "append_byte" and how < 0.4:            # a decoding batch
            n_seqs, rows = _log_int(rng, 2, 256), rng.choice([1, 1, 2, 4])
            ctx = rows + _log_int(rng, 1, 1024)
        elif kind == "append_byte" and how < 0.6:          # rows recomputed here and there
            ctx = _log_int(rng, 64, 16384)
            rows, spread = _log_int(rng, 1, max(1, ctx // 3)), True
        else:
            rows = _log_int(rng, 1, min(65536, 2 ** 25 // (per_row * d)))
            ctx = rows + _log_int(rng, 1, 1024)
        return _case(kind, dtype=dtype, n_seqs=n_seqs, rows=rows, hq=hq, hkv=hkv, d=d, ctx=ctx, page=page, rot=rot,
                     axes=axes, pairing=pairing, with_q=with_q, held=kind == "append_byte" and rng.random() < 0.4,
                     spread=spread, ragged=n_seqs > 1, pad=rng.choice([0, 0, 1]) if n_seqs > 1 else 0)
    how = rng.random()
    if how < 0.35:                                       # rows of one sequence
        ctx = _log_int(rng, 64, 16384)
        rows = _log_int(rng, 1, min(ctx, 1500, 2 ** 23 // (hq * d)))
        return _case(kind, dtype=dtype, rows=rows, hq=hq, hkv=hkv, d=d, ctx=ctx, page=page, spread=True)
    if how < 0.5:                                        # an encoder's states
        n_seqs, ctx = _log_int(rng, 1, 16), _log_int(rng, 16, 4096)
        rows = _log_int(rng, 1, max(1, min(512, 2 ** 21 // (n_seqs * hq * d))))
        return _case(kind, dtype=dtype, n_seqs=n_seqs, rows=rows, hq=hq, hkv=hkv, d=d, ctx=ctx, page=page, ragged=True,
                     cross=True, pad=rng.choice([0, 0, 1]) if n_seqs > 1 else 0)
    n_seqs, rows = _log_int(rng, 1, 128), rng.choice([1, 1, 1, 3, 5])
    ctx = max(rows, _log_int(rng, max(rows, 2), max(16, min(65536, 2 ** 22 // (n_seqs * hkv)))))
    return _case(kind, dtype=dtype, n_seqs=n_seqs, rows=rows, hq=hq, hkv=hkv, d=d, ctx=ctx, page=page, ragged=True,
                 pad=rng.choice([0, 0, 1]) if n_seqs > 1 else 0)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _frequencies(case):
    """inv_freq [rot / 2] (fp32) and the axis of each: contiguous sections, the
    first axis (time) with half the share of the others."""
    half = case["rot"] // 2
    inv = (1e6 ** (-np.arange(half, dtype=np.float64) / half)).astype(np.float32)
    shares = np.array([1.0] if case["axes"] == 1 else [1.0] + [2.0] * (case["axes"] - 1))
    ends = np.floor(np.cumsum(shares) / shares.sum() * half + 1e-9).astype(np.int64)
    return inv, np.searchsorted(ends, np.arange(half), side="right").clip(0, case["axes"] - 1).astype(np.int32)


def _grid_positions(case, n, rng, base):
    """Positions of n tokens on up to four axes: one time step per image of 32 x 32
    places, from `base` on."""
    i = np.arange(n)
    axes = [i // 1024, (i // 32) % 32, i % 32, i % 7]
    if case["axes"] == 1:
        axes = [i]
    out = np.stack(axes[: case["axes"]]) + base + rng.integers(0, 64)
    return torch.from_numpy(out.astype(np.int32)).to(DEV)


def _lengths(case, rng):
    """Tokens of every sequence: spread evenly from a few to ctx, in random order."""
    n, lo = case["n_seqs"], 1 if case["cross"] else case["rows"]
    if not case["ragged"]:
        return np.full(n, case["ctx"], np.int64)
    out = lo + ((case["ctx"] - lo) * (np.arange(n) + 1.0) / n).astype(np.int64)
    return rng.permutation(out)


def _positions(case, rng):
    """Row positions [n_seqs * rows]: the last rows of every sequence, rows spread over
    it, or its last token for every row; -1 in padded sequences."""
    r = case["rows"]
    out = []
    for length in _lengths(case, rng):
        if case["cross"]:
            out.append(np.full(r, length - 1))
        elif case["spread"]:
            out.append(np.sort(rng.choice(length, size=r, replace=False)))
        else:
            out.append(np.arange(length - r, length))
    out = np.stack(out)
    if case["pad"]:
        out[rng.choice(case["n_seqs"], size=case["pad"], replace=False)] = -1
    return torch.from_numpy(out.reshape(-1).astype(np.int32)).to(DEV)


def _table(case, rng):
    """Block table [n_seqs][pages] over a pool in random order, and the pool's pages."""
    per = -(-case["ctx"] // case["page"])
    n_pages = case["n_seqs"] * per
    return torch.from_numpy(rng.permutation(n_pages).astype(np.int32).reshape(case["n_seqs"], per)).to(DEV), n_pages


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _random_pool(case, n_pages, gen):
    """Codes and scales like those of normal keys and values: the largest of a block
    between half and all of the largest code, scales around 2^-7."""
    shape = (n_pages, case["hkv"], case["page"], case["d"])
    code = torch.empty(shape, dtype=torch.uint8, device=DEV)
    for p in range(0, n_pages, 512):  # in pieces: one byte per element is kept, four are drawn
        x = (_normal(gen, *code[p:p + 512].shape) * 85.0).clamp(-CODE_MAX, CODE_MAX)
        code[p:p + 512] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    scale = torch.randint(119, 122, (*shape[:2], case["page"] // BLOCK), generator=gen, device=DEV, dtype=torch.uint8)
    return code, scale


def _inputs(case, seed):
    rng = np.random.default_rng([seed, 23])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt, d, hq, hkv = _torch_dtype(case), case["d"], case["hq"], case["hkv"]
    n = case["n_seqs"] * case["rows"]
    table, n_pages = _table(case, rng)
    st = dict(case=case, table=table)
    if case["kind"] != "attn_byte":
        inv, axis = _frequencies(case)
        st.update(inv=inv, axis=axis, inv_dev=torch.from_numpy(inv).to(DEV),
                  axis_dev=torch.from_numpy(axis.astype(np.int64)).to(DEV))
    st["k8"], st["k8s"] = _random_pool(case, n_pages, gen)
    st["v8"], st["v8s"] = _random_pool(case, n_pages, gen)
    if case["kind"] == "append_byte":
        st["pos"] = _positions(case, rng)
        # the projections' output: queries, keys and values of a token side by side
        width = (hq if case["with_q"] else 0) + 2 * hkv
        qkv = _normal(gen, n, width, d).to(dt)
        st["q"] = qkv[:, :hq] if case["with_q"] else None
        st["k_new"], st["v_new"] = qkv[:, -2 * hkv:-hkv], qkv[:, -hkv:]
        st["q_out"] = torch.empty(n, hq, d, dtype=dt, device=DEV) if case["with_q"] else None
        st["k_held"], st["v_held"] = ((torch.empty(n, hkv, d, dtype=dt, device=DEV) for _ in range(2))
                                      if case["held"] else (None, None))
        st["rope_pos"] = _grid_positions(case, n, rng, case["ctx"] - case["rows"])
        # rows written over others: all of the sequence is there already
        st["n_held"] = (torch.full((case["n_seqs"],), case["ctx"], dtype=torch.int32, device=DEV)
                        if case["spread"] else None)
    if case["kind"] == "load_byte":
        # the first `rows` tokens of the store go to the request's tokens from a shift on
        shift = case["ctx"] - case["rows"]
        st["pos"] = torch.arange(n, dtype=torch.int32, device=DEV)
        st["dst_pos"] = st["pos"] + shift
        st["rope_pos"] = torch.full((case["axes"], n), shift, dtype=torch.int32, device=DEV)
        st["k"], st["v"] = (torch.zeros(case["ctx"], hkv, d, dtype=dt, device=DEV) for _ in range(2))
    if case["kind"] == "attn_byte":
        st["pos"] = _positions(case, rng)
        st["q"] = _normal(gen, n, hq, d).to(dt)
        st["o"] = torch.empty(n, hq, d, dtype=dt, device=DEV)
        st["lse"] = torch.empty(n, hq, dtype=torch.float32, device=DEV)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if not own:
        return st
    from paper_2609_05821_amd import api
    if case["kind"] != "attn_byte":
        st["rope"] = api.Rope(st["inv"], st["axis"], n_axes=case["axes"],
                              pairing=api.PAIR_ADJACENT if case["pairing"] == ADJACENT else api.PAIR_HALVES)
    if case["kind"] == "load_byte":
        st["kv"] = api.kv_desc(st["k"], st["v"], case["hq"])
    st["cache"] = api.byte_desc(st["k8"], st["v8"], st["k8s"], st["v8s"], case["hq"], case["ctx"], st["table"])
    if case["kind"] == "attn_byte":
        need = api.attn_byte_workspace_bytes(st["cache"], st["q"])
        st["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _pools(st):
    """The cache's state: codes as the e4m3 numbers that they are, and scale bytes."""
    return [st["k8"].view(torch.float8_e4m3fn), st["k8s"], st["v8"].view(torch.float8_e4m3fn), st["v8s"]]


def _run_own(st):
    from paper_2609_05821_amd import api
    kind = st["case"]["kind"]
    if kind == "append_byte":
        api.conduit_append_byte(st["cache"], st["pos"], st["k_new"], st["v_new"], n_held=st["n_held"], rope=st["rope"],
                              rope_pos=st["rope_pos"], q=st["q"], q_out=st["q_out"], k_out=st["k_held"],
                              v_out=st["v_held"])
        return _pools(st) + [t for t in (st["q_out"], st["k_held"], st["v_held"]) if t is not None]
    if kind == "load_byte":
        api.conduit_load_byte(st["cache"], st["pos"], st["kv"], st["dst_pos"], rope=st["rope"], rope_pos=st["rope_pos"])
        return [st["k"], st["v"]]
    api.conduit_attn_byte(st["cache"], st["q"], st["pos"], st["o"], lse_out=st["lse"], ws=st["ws"])
    return [st["o"], st["lse"]]


def _rotated(st, x, wide):
    """x [n, heads, d] turned by its rows' angles, in 32 bits (64 when `wide`; the
    angles always in 64)."""
    c = st["case"]
    theta = st["rope_pos"].double()[st["axis_dev"]].t() * st["inv_dev"].double()
    t = torch.float64 if wide else torch.float32
    cos, sin = theta.cos().to(t)[:, None], theta.sin().to(t)[:, None]
    x = x.to(t)
    half = c["rot"] // 2
    y = x.clone()
    if c["pairing"] == HALVES:
        a, b = x[..., :half], x[..., half:2 * half]
        y[..., :half], y[..., half:2 * half] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a * cos - b * sin, a * sin + b * cos
    return y


def _two_to(e):
    """2^e (fp32) from its bits: exact, where a power of the device need not be.  Below
    2^-126, where nothing of a code is left, 2^-126."""
    return ((e.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _e4m3(y):
    """y (fp32) rounded to e4m3, ties to even, as fp32."""
    e = torch.frexp(y)[1].clamp(min=-5) - 4
    return ((y * _two_to(-e)).round() * _two_to(e)).clamp(-CODE_MAX, CODE_MAX)


def _needed(top):
    """The smallest scale byte that holds magnitudes up to `top`: 448 is 0.875 * 2^9."""
    m, e = torch.frexp(top)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(m == 0, SCALE_MIN, e + 127).clamp(SCALE_MIN, SCALE_MAX)


def _numbers(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _held(codes, scales):
    """Values (fp32) of codes [..., slot, d] and scale bytes [..., slot / 16]."""
    f = _two_to(scales.int() - 127)
    return (_numbers(codes).unflatten(-2, (-1, BLOCK)) * f[..., None, None]).flatten(-3, -2)


def _run_plain(st):
    c = st["case"]
    kind = c["kind"]
    if kind == "attn_byte":
        return _plain_attention(st)
    n, page = st["pos"].numel(), c["page"]
    p = st["pos"].long()
    if kind == "load_byte":
        at_page, at_slot = st["table"][0, p // page].long(), p % page
        k, v = (_numbers(codes[at_page, :, at_slot]) *
                _two_to(scales[at_page, :, at_slot // BLOCK].int() - 127)[..., None]
                for codes, scales in ((st["k8"], st["k8s"]), (st["v8"], st["v8s"])))
        st["k"][st["dst_pos"].long()] = _rotated(st, k, False).to(st["k"].dtype)
        st["v"][st["dst_pos"].long()] = v.to(st["v"].dtype)
        return [st["k"], st["v"]]
    return _plain_append(st)


def _plain_append(st):
    c = st["case"]
    n_seqs, r, page, hkv, d = c["n_seqs"], c["rows"], c["page"], c["hkv"], c["d"]
    n, p, dt = n_seqs * r, st["pos"].long(), st["k_new"].dtype
    n_blocks = st["table"].shape[1] * page // BLOCK
    seq = torch.arange(n, device=DEV) // r
    # which row goes to each token (-1: none; padded rows to a place of their own)
    tokens = n_blocks * BLOCK
    row_at = torch.full((n_seqs * tokens + 1,), -1, dtype=torch.int64, device=DEV)
    row_at[torch.where(p >= 0, seq * tokens + p, n_seqs * tokens)] = torch.arange(n, device=DEV)
    # the blocks that rows may go to, some more than once
    if c["spread"]:
        bs, bb = seq, p // BLOCK
    else:
        first = p.view(n_seqs, r)[:, :1].clamp(min=0) // BLOCK
        bb = (first + torch.arange(r // BLOCK + 2, device=DEV)).clamp(max=n_blocks - 1)
        bs = torch.arange(n_seqs, device=DEV)[:, None].expand_as(bb).flatten()
        bb = bb.flatten()
    slot = torch.arange(BLOCK, device=DEV)
    token = bb[:, None] * BLOCK + slot
    src = row_at[bs[:, None] * tokens + token]
    written = src >= 0
    if st["n_held"] is None:
        kept = ~written & (slot < (written * slot).amax(1, keepdim=True))
    else:
        kept = ~written & (token < st["n_held"][bs][:, None])
    at_page = st["table"][bs, bb * BLOCK // page].long()
    at_block = bb % (page // BLOCK)
    at_slot = at_block[:, None] * BLOCK + slot
    any_written, any_kept = written.any(1)[:, None], kept.any(1)[:, None]
    # a rounding to 8 bits is a border: the keys are turned in 64 bits, then rounded like a 16-bit cache's
    k = _rotated(st, st["k_new"], True).float().to(dt).float()
    held = []
    for codes, scales, new in ((st["k8"], st["k8s"], k), (st["v8"], st["v8s"], st["v_new"].float())):
        x = torch.where(written[..., None, None], new[src.clamp(min=0)], 0.0)          # [blocks, 16, heads, d]
        old = scales[at_page, :, at_block].int().clamp(SCALE_MIN, SCALE_MAX)             # [blocks, heads]
        s = _needed(x.abs().amax((1, 3)))
        s = torch.where(any_kept, torch.maximum(s, old), s)
        before = codes[at_page[:, None], :, at_slot]
        y = torch.where(written[..., None, None], x * _two_to(127 - s)[:, None, :, None],
                        _numbers(before) * _two_to(old - s)[:, None, :, None])
        y = _e4m3(y).to(torch.float8_e4m3fn).view(torch.uint8)
        changes = (written | kept)[..., None, None]
        codes[at_page[:, None], :, at_slot] = torch.where(changes, y, before)
        byte = torch.where(any_written, s, scales[at_page, :, at_block].int()).to(torch.uint8)
        scales[at_page, :, at_block] = byte
        if c["held"]:
            # a left-out row as it would be held in a block of its own
            at = torch.where(p >= 0, p, 0)
            pg = st["table"][seq, at // page].long()
            e = torch.where((p >= 0)[:, None], scales[pg, :, at % page // BLOCK].int(), _needed(new.abs().amax(-1)))
            e = (e - 127)[..., None]
            held.append((_e4m3(new * _two_to(-e)) * _two_to(e)).to(dt))
    out = _pools(st)
    if c["with_q"]:
        out.append(_rotated(st, st["q"], False).to(dt))
    return out + held


def _plain_attention(st):
    c = st["case"]
    n_seqs, r, hq, hkv, d = c["n_seqs"], c["rows"], c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    ctx = st["table"].shape[1] * c["page"]
    per = max(1, min(n_seqs, 2 ** 27 // (ctx * hkv * d)))  # sequences at once
    pos = st["pos"].view(n_seqs, r)
    q = st["q"].float().view(n_seqs, r, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n_seqs, hkv, r * g, d)
    o, lse = [], []
    for s in range(0, n_seqs, per):
        pages = st["table"][s:s + per].long()
        kv = []
        for codes, scales in ((st["k8"], st["k8s"]), (st["v8"], st["v8s"])):
            x = _held(codes[pages], scales[pages])           # [s, pages, hkv, page, d]
            kv.append(x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], hkv, ctx, d))
        logits = torch.matmul(q[s:s + per], kv[0].transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
        seen = torch.arange(ctx, device=DEV) <= pos[s:s + per].repeat_interleave(g, 1)[:, None, :, None]
        logits = logits.masked_fill(~seen, -math.inf)
        top = logits.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        w = (logits - top).exp()
        total = w.sum(-1, keepdim=True)
        out = torch.matmul(w, kv[1]) / torch.where(total == 0, 1.0, total)
        o.append(out.view(-1, hkv, r, g, d).permute(0, 2, 1, 3, 4).reshape(-1, hq, d))
        lse.append((total.log() + top).view(-1, hkv, r, g).permute(0, 2, 1, 3).reshape(-1, hq))
    return [torch.cat(o).to(st["q"].dtype), torch.cat(lse)]


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    st = _inputs(case, seed)
    page = case["page"]
    if case["kind"] == "attn_byte":
        return _exact_attention(st)
    if case["kind"] == "load_byte":
        at = [(int(t) // page, int(t) % page) for t in st["pos"].tolist()]
        pg = st["table"][0].long()[torch.tensor([a for a, _ in at], device=DEV)]
        sl = torch.tensor([b for _, b in at], device=DEV)
        k, v = st["k"].double(), st["v"].double()
        k[st["dst_pos"].long()] = _turned(st, _decoded(st["k8"][pg, :, sl]) * _power(st["k8s"][pg, :, sl // BLOCK]))
        v[st["dst_pos"].long()] = _decoded(st["v8"][pg, :, sl]) * _power(st["v8s"][pg, :, sl // BLOCK])
        return [k, v]
    return _exact_append(st)


def _power(scales):
    return _double_power(scales.long()[..., None] - 127)


def _double_power(e):
    """2^e in 64 bits, made from its exponent's bits."""
    return ((e + 1023) << 52).view(torch.float64)


def _decoded(codes):
    """Values of code bytes from their bits: sign, four exponent bits, three of mantissa."""
    b = codes.long()
    expo, man = (b // 8) % 16, (b % 8).double()
    mag = torch.where(expo == 0, man * 2.0 ** -9, (1 + man / 8) * _double_power(expo - 7))
    return torch.where(b >= 128, -mag, mag)


def _turned(st, x):
    """Pairs as complex numbers times e^(i theta)."""
    c = st["case"]
    rot = c["rot"]
    theta = torch.stack([st["rope_pos"][int(a)].double() * float(f) for a, f in zip(st["axis"], st["inv"])], -1)
    turn = torch.polar(torch.ones_like(theta), theta)[:, None]
    x = x.double()
    head = x[..., :rot].unflatten(-1, (2, -1) if c["pairing"] == HALVES else (-1, 2))
    dim = -2 if c["pairing"] == HALVES else -1
    z = torch.complex(head.select(dim, 0).contiguous(), head.select(dim, 1).contiguous()) * turn
    return torch.cat((torch.stack((z.real, z.imag), dim).flatten(-2), x[..., rot:]), -1)


def _nearest(y):
    """y (float64) as the nearest e4m3 number by distance, the even code of two."""
    table = _decoded(torch.arange(127, dtype=torch.uint8, device=DEV))
    out = []
    for part in y.reshape(-1).split(1 << 24):
        up = torch.bucketize(part.abs(), table).clamp(1, 126)
        lo, hi = table[up - 1], table[up]
        below, above = part.abs() - lo, hi - part.abs()
        take = (below < above) | ((below == above) & (up % 2 == 1))        # (up - 1 is the even one)
        out.append(torch.copysign(torch.where(take, lo, hi), part))
    return torch.cat(out).view(y.shape)


def _smallest(top):
    """The smallest scale byte whose largest code is not below `top`."""
    s = torch.full(top.shape, SCALE_MAX, dtype=torch.int64, device=DEV)
    for byte in range(SCALE_MAX - 1, SCALE_MIN - 1, -1):
        s = torch.where(top <= CODE_MAX * 2.0 ** (byte - 127), byte, s)
    return s


def _exact_append(st):
    c = st["case"]
    r, page, hkv, d = c["rows"], c["page"], c["hkv"], c["d"]
    live = torch.nonzero(st["pos"] >= 0).flatten()
    p, seq = st["pos"][live].long(), live // r
    blocks, of = torch.unique(seq * (1 << 32) + p // BLOCK, return_inverse=True)
    b_seq, b_at = blocks >> 32, blocks & ((1 << 32) - 1)
    pg = st["table"][b_seq, b_at * BLOCK // page].long()
    in_page = b_at % (page // BLOCK)
    row = torch.full((blocks.numel(), BLOCK), -1, dtype=torch.int64, device=DEV)
    row[of, p % BLOCK] = live
    token = b_at[:, None] * BLOCK + torch.arange(BLOCK, device=DEV)
    if st["n_held"] is None:
        last = torch.where(row >= 0, token, -1).amax(1)
    else:
        last = st["n_held"].long()[b_seq]
    keep = (row < 0) & (token < last[:, None])
    dt = st["k_new"].dtype
    keys = _turned(st, st["k_new"]).float().to(dt).double()       # as a cache of this type would hold them
    outs, held = [], []
    for codes, scales, new in ((st["k8"], st["k8s"], keys), (st["v8"], st["v8s"], st["v_new"].double())):
        top = torch.zeros(blocks.numel(), hkv, dtype=torch.float64, device=DEV)
        for j in range(BLOCK):
            there = row[:, j] >= 0
            top[there] = torch.maximum(top[there], new[row[there, j]].abs().amax(-1))
        was = scales[pg, :, in_page].long().clamp(SCALE_MIN, SCALE_MAX)
        now = _smallest(top)
        now = torch.where(keep.any(1)[:, None], torch.maximum(now, was), now)
        number = _decoded(codes)
        for j in range(BLOCK):
            sl = in_page * BLOCK + j
            k = keep[:, j]
            number[pg[k], :, sl[k]] = _nearest(number[pg[k], :, sl[k]] * _double_power(was[k] - now[k])[..., None])
            w = row[:, j] >= 0
            number[pg[w], :, sl[w]] = _nearest(new[row[w, j]] * _double_power(127 - now[w])[..., None])
        scales[pg, :, in_page] = now.to(torch.uint8)
        outs += [number, scales]
        if c["held"]:
            x = torch.empty_like(new)
            s = _smallest(new.abs().amax(-1))
            s[live] = now[of]
            f = _power(s)
            for i in range(0, x.shape[0], 4096):
                x[i:i + 4096] = _nearest(new[i:i + 4096] / f[i:i + 4096]) * f[i:i + 4096]
            held.append(x)
    if c["with_q"]:
        outs.append(_turned(st, st["q"]))
    return outs + held


def _exact_attention(st):
    c = st["case"]
    r, hq, hkv, page = c["rows"], c["hq"], c["hkv"], c["page"]
    g = hq // hkv
    n = c["n_seqs"] * r
    o = torch.zeros(n, hq, c["d"], dtype=torch.float64, device=DEV)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=DEV)
    pos = st["pos"].view(-1, r).tolist()
    for s in range(c["n_seqs"]):
        length = max(pos[s]) + 1
        if length == 0:
            continue
        pages = st["table"][s, : -(-length // page)].long()
        hidden = torch.arange(length, device=DEV)[None] > st["pos"].view(-1, r)[s][:, None]
        for h in range(hkv):
            k, v = ((_decoded(codes[pages, h]) * _power(scales[pages, h].repeat_interleave(BLOCK, -1)))
                    .reshape(-1, c["d"])[:length] for codes, scales in ((st["k8"], st["k8s"]), (st["v8"], st["v8s"])))
            for j in range(h * g, (h + 1) * g):
                w = (st["q"][s * r:(s + 1) * r, j].double() @ k.t()) / math.sqrt(c["d"])
                w[hidden] = -math.inf
                total = torch.logsumexp(w, -1)
                some = total > -math.inf
                w = torch.where(some[:, None], torch.exp(w - torch.where(some, total, 0.0)[:, None]), 0.0)
                o[s * r:(s + 1) * r, j] = w @ v
                lse[s * r:(s + 1) * r, j] = total
    return [o, lse]


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    n_seqs, r, hq, hkv, d = case["n_seqs"], case["rows"], case["hq"], case["hkv"], case["d"]
    n, live = n_seqs * r, (n_seqs - case["pad"]) * r
    kind = case["kind"]
    ids = 4 * (case["axes"] + 1) * n
    if kind == "append_byte":
        q = 2 * n * hq * d * es if case["with_q"] else 0
        q_flops = 3 * n * hq * case["rot"] if case["with_q"] else 0
        held = 2 * n * hkv * d * es if case["held"] else 0
        blocks = live if case["spread"] or r < BLOCK else live / BLOCK
        return {"bytes": int(2 * live * hkv * d * (es + 1) + 2 * blocks * hkv + held + q + ids),
                "flops": live * hkv * (3 * case["rot"] + 4 * d) + q_flops}
    if kind == "load_byte":
        return {"bytes": int(2 * n * hkv * (d + 1 / BLOCK + d * es) + ids),
                "flops": n * hkv * (3 * case["rot"] + 2 * d)}
    lo = 1 if case["cross"] else r
    lengths = [case["ctx"]] * n_seqs
    if case["ragged"]:
        lengths = [lo + int((case["ctx"] - lo) * (i + 1.0) / n_seqs) for i in range(n_seqs)]
    share = (n_seqs - case["pad"]) / n_seqs
    keys = sum(lengths)
    if case["cross"]:
        pairs = sum(length * r for length in lengths)
    elif case["spread"]:
        pairs = sum(length * r / 2 for length in lengths)
    else:
        pairs = sum(length * r - r * (r - 1) / 2 for length in lengths)
    return {"bytes": int(share * keys * 2 * hkv * (d + 1 / BLOCK)) + 2 * n * hq * d * es + 4 * n * hq + 4 * n,
            "flops": int(share * pairs) * 4 * hq * d}
