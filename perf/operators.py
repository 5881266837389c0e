"""Positions, growing caches and 4-bit caches, as cases that can be timed and checked.

A case is a dict of plain values; ``prepare`` makes its inputs on the GPU from a
seed, ``run`` makes one pass, and ``exact`` gives the outputs of that pass from
the definitions in 64 bits.  With ``own`` false ``run`` computes the operators
in elementary torch operations; with ``own`` true it calls the package.  The
kinds of case:

  rotary     rotary positions with one to four axes, forward and inverse (the
             inverse rotation of a gradient is the operator's backward pass);
  append     new keys and values into a cache of 16 or 32 bits, the keys (and
             the queries of the same tokens) rotated on the way;
  append_mx  the same into a cache held in 4 bits;
  load_mx    rows of a 4-bit cache into a cache of 16 or 32 bits, the keys
             rotated by the distance that they move;
  attn_mx    causal attention over a 4-bit cache.

The 4-bit cache: 32 consecutive dims of one token and head share one scale
byte s and hold codes c of sign and magnitude {0, 0.5, 1, 1.5, 2, 3, 4, 6}; the
value is c * 2^(s - 127).  s is the smallest with max|x| <= 6 * 2^(s - 127),
kept between 2 and 252; codes are the nearest, ties to the even code.  Code
bytes hold dim 2i in the low four bits.  Pools are [page][head][slot][d / 2] codes
and [page][head][slot][d / 32] scales.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
HALVES, ADJACENT = 0, 1
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# Borders between neighbouring magnitudes, and whether the border itself goes
# up (to the even code).
BORDERS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------

def _case(kind, **kw):
    c = dict(kind=kind, dtype="bf16", n_seqs=1, rows=1, hq=28, hkv=4, d=128, ctx=0, page=64, rot=128, axes=3,
             pairing=HALVES, inverse=False, with_q=True, held=False, spread=False, ragged=False, pad=0)
    c.update(kw)
    return c


def listed():
    return [
        # One generated token of a grouped-head model, its queries turned before attention: pure latency.
        _case("rotary", name="rotary_token", rows=1),
        # The backward pass of a vision encoder's two-axis positions, heads of 80 dims, fp32 gradients.
        _case("rotary", name="rotary_patches_grad_f32", dtype="f32", rows=16384, hq=16, d=80, rot=80, axes=2,
              inverse=True),
        # A decoding batch: one token each of 64 sequences into the shared page pool (two of them padding).
        _case("append", name="append_decode", n_seqs=64, rows=1, ctx=1024, pad=2),
        # A whole 16k multi-image prompt into a paged cache, one layer.
        _case("append", name="append_prompt", rows=17024, ctx=17024),
        # The decoding batch again, cache in 4 bits.
        _case("append_mx", name="append_mx_decode", n_seqs=64, rows=1, ctx=1024, pad=2, held=True),
        # A long document's keys and values packed for reuse, and handed back as the cache holds them.
        _case("append_mx", name="append_mx_document", rows=65536, ctx=65536, with_q=False, held=True),
        # One image of a 4-bit store loaded into a request's cache, its keys moved to their new place.
        _case("load_mx", name="load_image", rows=1024, ctx=1344),
        # A long document loaded likewise.
        _case("load_mx", name="load_document", rows=65536, ctx=66048),
        # One token, fp32, one image of context, 8 heads of 64: the smallest attention.
        _case("attn_mx", name="attn_token_f32", dtype="f32", hq=8, hkv=8, d=64, ctx=672),
        # A decoding batch of 64 ragged sequences of up to 32k tokens (two of them padding).
        _case("attn_mx", name="attn_decode", n_seqs=64, ctx=32768, ragged=True, pad=2),
        # Five drafted tokens of each of 8 sequences verified at once, an odd context.
        _case("attn_mx", name="attn_draft", n_seqs=8, rows=5, hq=32, hkv=8, ctx=8211, ragged=True),
        # The refresh step's selected rows (10% of 16k visual tokens) over a 4-bit cache.
        _case("attn_mx", name="attn_refresh", rows=1638, ctx=17024, spread=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "append_mx", "load_mx", "attn_mx", "attn_mx"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 5, 7, 8])
    page = rng.choice([64, 128, 256])
    axes = rng.choice([1, 2, 3, 4])
    pairing = rng.choice([HALVES, HALVES, ADJACENT])
    if kind == "rotary":
        d = rng.choice([64, 72, 80, 96, 128, 128, 256])
        rot = rng.choice([d, d, d // 2])
        rows = _log_int(rng, 1, max(1, 2 ** 26 // (hq * d)))
        return _case(kind, dtype=dtype, rows=rows, hq=hq, d=d, rot=rot, axes=axes, pairing=pairing,
                     inverse=rng.random() < 0.4)
    if kind in ("append", "append_mx", "load_mx"):
        with_q = kind != "load_mx" and rng.random() < 0.6
        per_row = (hq if with_q else 0) + 2 * hkv
        rot = rng.choice([d, d, d // 2])
        if kind != "load_mx" and rng.random() < 0.4:  # a decoding batch
            n_seqs, rows = _log_int(rng, 2, 256), rng.choice([1, 1, 2, 4])
        else:
            n_seqs, rows = 1, _log_int(rng, 1, min(65536, 2 ** 25 // (per_row * d)))
        ctx = rows + _log_int(rng, 1, 1024)
        return _case(kind, dtype=dtype, n_seqs=n_seqs, rows=rows, hq=hq, hkv=hkv, d=d, ctx=ctx, page=page, rot=rot,
                     axes=axes, pairing=pairing, with_q=with_q, held=kind == "append_mx" and rng.random() < 0.5,
                     pad=rng.choice([0, 0, 1]) if n_seqs > 1 else 0)
    if rng.random() < 0.4:  # rows of one sequence
        ctx = _log_int(rng, 64, 16384)
        rows = _log_int(rng, 1, min(ctx, 1500, 2 ** 23 // (hq * d)))
        return _case(kind, dtype=dtype, rows=rows, hq=hq, hkv=hkv, d=d, ctx=ctx, page=page, spread=True)
    n_seqs, rows = _log_int(rng, 1, 128), rng.choice([1, 1, 1, 3, 5])
    ctx = _log_int(rng, max(rows, 2), max(16, min(32768, 2 ** 22 // (n_seqs * hkv))))
    ctx = max(ctx, rows)
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
    n, lo = case["n_seqs"], case["rows"]
    if not case["ragged"]:
        return np.full(n, case["ctx"], np.int64)
    out = lo + ((case["ctx"] - lo) * (np.arange(n) + 1.0) / n).astype(np.int64)
    return rng.permutation(out)


def _positions(case, rng):
    """Row positions [n_seqs * rows]: the last rows of every sequence, or rows spread
    over it; -1 in padded sequences."""
    r = case["rows"]
    out = []
    for length in _lengths(case, rng):
        if case["spread"]:
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
    """Codes and scales like those of normal keys and values: codes by their share
    under the borders for max|x| around 4.5 units, scales around 1/2."""
    shape = (n_pages, case["hkv"], case["page"])
    edges = torch.tensor([b for b, _ in BORDERS], device=DEV)
    code = torch.empty(*shape, case["d"], dtype=torch.uint8, device=DEV)
    for p in range(0, n_pages, 512):  # in pieces: one byte per element is kept, four are drawn
        x = _normal(gen, *code[p:p + 512].shape) * 1.9
        code[p:p + 512] = torch.bucketize(x.abs(), edges).to(torch.uint8) + (x < 0).to(torch.uint8) * 8
    packed = code[..., 0::2] | (code[..., 1::2] << 4)
    scale = torch.randint(125, 128, (*shape, case["d"] // 32), generator=gen, device=DEV, dtype=torch.uint8)
    return packed.contiguous(), scale


def _inputs(case, seed):
    rng = np.random.default_rng([seed, 17])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt, d, hq, hkv = _torch_dtype(case), case["d"], case["hq"], case["hkv"]
    n = case["n_seqs"] * case["rows"]
    st = dict(case=case)
    if case["kind"] != "attn_mx":
        inv, axis = _frequencies(case)
        st.update(inv=inv, axis=axis, inv_dev=torch.from_numpy(inv).to(DEV),
                  axis_dev=torch.from_numpy(axis.astype(np.int64)).to(DEV))
    if case["kind"] == "rotary":
        st.update(x=_normal(gen, n, hq, d).to(dt), rope_pos=_grid_positions(case, n, rng, 1000),
                  out=torch.empty(n, hq, d, dtype=dt, device=DEV))
        return st
    table, n_pages = _table(case, rng)
    pool = (n_pages, case["page"], hkv, d)
    st["table"] = table
    if case["kind"] in ("append", "append_mx"):
        st["pos"] = _positions(case, rng)
        # the projections' output: queries, keys and values of a token side by side
        width = (hq if case["with_q"] else 0) + 2 * hkv
        qkv = _normal(gen, n, width, d).to(dt)
        st["q"] = qkv[:, :hq] if case["with_q"] else None
        st["k_new"], st["v_new"] = qkv[:, -2 * hkv:-hkv], qkv[:, -hkv:]
        st["q_out"] = torch.empty(n, hq, d, dtype=dt, device=DEV) if case["with_q"] else None
        st["rope_pos"] = _grid_positions(case, n, rng, case["ctx"] - case["rows"])
    if case["kind"] == "append":
        st["k"], st["v"] = (torch.zeros(pool, dtype=dt, device=DEV) for _ in range(2))
        # rows of the pool: where each token goes (-1: padding)
        page = case["page"]
        p = st["pos"].long()
        seq = torch.arange(n, device=DEV) // case["rows"]
        row = table[seq, p.clamp(min=0) // page].long() * page + p.clamp(min=0) % page
        st["slots"] = torch.where(p >= 0, row, -1).to(torch.int32)
    if case["kind"] in ("append_mx", "load_mx", "attn_mx"):
        st["k4"], st["k4s"] = _random_pool(case, n_pages, gen)
        st["v4"], st["v4s"] = _random_pool(case, n_pages, gen)
    if case["kind"] == "append_mx":
        st["k_held"], st["v_held"] = ((torch.empty(n, hkv, d, dtype=dt, device=DEV) for _ in range(2))
                                      if case["held"] else (None, None))
    if case["kind"] == "load_mx":
        # the first `rows` tokens of the store go to the request's tokens from a shift on
        shift = case["ctx"] - case["rows"]
        st["pos"] = torch.arange(n, dtype=torch.int32, device=DEV)
        st["dst_pos"] = st["pos"] + shift
        st["rope_pos"] = torch.full((case["axes"], n), shift, dtype=torch.int32, device=DEV)
        st["k"], st["v"] = (torch.zeros(case["ctx"], hkv, d, dtype=dt, device=DEV) for _ in range(2))
    if case["kind"] == "attn_mx":
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
    if case["kind"] != "attn_mx":
        st["rope"] = api.Rope(st["inv"], st["axis"], n_axes=case["axes"],
                              pairing=api.PAIR_ADJACENT if case["pairing"] == ADJACENT else api.PAIR_HALVES)
    if case["kind"] == "append":
        pool = (-1, case["hkv"], case["d"])
        st["kv"] = api.kv_desc(st["k"].view(pool), st["v"].view(pool), case["hq"])
    if case["kind"] == "load_mx":
        st["kv"] = api.kv_desc(st["k"], st["v"], case["hq"])
    if case["kind"] in ("append_mx", "load_mx", "attn_mx"):
        st["mx"] = api.mx_desc(st["k4"], st["v4"], st["k4s"], st["v4s"], case["hq"], case["ctx"], st["table"])
    if case["kind"] == "attn_mx":
        need = api.attn_mx_workspace_bytes(st["mx"], st["q"])
        st["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    from paper_2609_05821_amd import api
    kind = st["case"]["kind"]
    if kind == "rotary":
        api.conduit_rotary(st["x"], st["rope"], st["rope_pos"], st["out"], inverse=st["case"]["inverse"])
        return [st["out"]]
    if kind == "append":
        api.conduit_append_kv(st["kv"], st["slots"], st["k_new"], st["v_new"], rope=st["rope"],
                              rope_pos=st["rope_pos"], q=st["q"], q_out=st["q_out"])
        return [t for t in (st["k"], st["v"], st["q_out"]) if t is not None]
    if kind == "append_mx":
        api.conduit_append_mx(st["mx"], st["pos"], st["k_new"], st["v_new"], rope=st["rope"],
                              rope_pos=st["rope_pos"], q=st["q"], q_out=st["q_out"], k_out=st["k_held"],
                              v_out=st["v_held"])
        return [t for t in (st["k4"], st["k4s"], st["v4"], st["v4s"], st["q_out"], st["k_held"], st["v_held"])
                if t is not None]
    if kind == "load_mx":
        api.conduit_load_mx(st["mx"], st["pos"], st["kv"], st["dst_pos"], rope=st["rope"], rope_pos=st["rope_pos"])
        return [st["k"], st["v"]]
    api.conduit_attn_mx(st["mx"], st["q"], st["pos"], st["o"], lse_out=st["lse"], ws=st["ws"])
    return [st["o"], st["lse"]]


def _rotated(st, x, wide):
    """x [n, heads, d] turned by its rows' angles, in 32 bits (64 when `wide`; the
    angles always in 64)."""
    c = st["case"]
    theta = st["rope_pos"].double()[st["axis_dev"]].t() * st["inv_dev"].double()
    if c["inverse"]:
        theta = -theta
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


def _packed(x):
    """Code bytes, scale bytes and held values of x [n, heads, d] (fp32)."""
    blocks = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(blocks.abs().amax(-1))
    e = torch.where(m <= 0.75, e - 3, e - 2)
    e = torch.where(m == 0, -125, e).clamp(-125, 125)
    y = torch.ldexp(blocks, -e[..., None])
    mag = y.abs()
    code = torch.zeros_like(mag, dtype=torch.uint8)
    for border, up in BORDERS:
        code += (mag >= border if up else mag > border)
    held = torch.tensor(MAGNITUDES, device=x.device)[code.long()] * torch.where(torch.signbit(y), -1.0, 1.0)
    held = torch.ldexp(held, e[..., None]).flatten(-2)
    code = (code + torch.signbit(y).to(torch.uint8) * 8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8), held


def _held(codes, scales):
    """Values (fp32) of code bytes [..., d / 2] and scale bytes [..., d / 32]."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    x = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * torch.exp2(scales.float() - 127.0)[..., None]).flatten(-2)


def _run_plain(st):
    c = st["case"]
    kind = c["kind"]
    if kind == "rotary":
        return [_rotated(st, st["x"], False).to(st["x"].dtype)]
    if kind == "attn_mx":
        return _plain_attention(st)
    n, page = st["pos"].numel(), c["page"]
    seq = torch.arange(n, device=DEV) // c["rows"]
    p = st["pos"].long()
    if kind == "load_mx":
        at_page, at_slot = st["table"][seq, p // page].long(), p % page
        k = _rotated(st, _held(st["k4"][at_page, :, at_slot], st["k4s"][at_page, :, at_slot]), False)
        v = _held(st["v4"][at_page, :, at_slot], st["v4s"][at_page, :, at_slot])
        st["k"][st["dst_pos"].long()] = k.to(st["k"].dtype)
        st["v"][st["dst_pos"].long()] = v.to(st["v"].dtype)
        return [st["k"], st["v"]]
    dt = st["k_new"].dtype
    if c["pad"]:  # padded rows write the first live row's data to its place once more
        src = torch.where(p >= 0, torch.arange(n, device=DEV), (p >= 0).to(torch.uint8).argmax())
    else:
        src = slice(None)
    q = [_rotated(st, st["q"], False).to(dt)] if c["with_q"] else []
    if kind == "append":
        k = _rotated(st, st["k_new"], False).to(dt)
        for cache, new in ((st["k"], k), (st["v"], st["v_new"])):
            cache.view(-1, c["hkv"], c["d"])[st["slots"][src].long()] = new[src]
        return [st["k"], st["v"]] + q
    # a rounding to 4 bits is a border: the keys are turned in 64 bits, then rounded like a 16-bit cache's
    k = _rotated(st, st["k_new"], True).float().to(dt).float()
    at_page, at_slot = st["table"][seq[src], p[src] // page].long(), p[src] % page
    held = []
    for codes, scales, new in ((st["k4"], st["k4s"], k), (st["v4"], st["v4s"], st["v_new"].float())):
        code, scale, values = _packed(new)
        codes[at_page, :, at_slot] = code[src]
        scales[at_page, :, at_slot] = scale[src]
        held.append(values.to(dt))
    return [st["k4"], st["k4s"], st["v4"], st["v4s"]] + q + (held if c["held"] else [])


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
        for codes, scales in ((st["k4"], st["k4s"]), (st["v4"], st["v4s"])):
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
    kind, d, page = case["kind"], case["d"], case["page"]
    dt = _torch_dtype(case)
    if kind == "rotary":
        return [_turned(st, st["x"])]
    if kind == "attn_mx":
        return _exact_attention(st)
    if kind == "load_mx":
        places = [(int(t) // page, int(t) % page) for t in st["pos"].tolist()]
        pg = st["table"][0].long()[torch.tensor([a for a, _ in places], device=DEV)]
        sl = torch.tensor([b for _, b in places], device=DEV)
        k, v = st["k"].double(), st["v"].double()
        k[st["dst_pos"].long()] = _turned(st, _value(st["k4"][pg, :, sl], st["k4s"][pg, :, sl]))
        v[st["dst_pos"].long()] = _value(st["v4"][pg, :, sl], st["v4s"][pg, :, sl])
        return [k, v]
    live = torch.nonzero(st["pos"] >= 0).flatten()
    k, v = _turned(st, st["k_new"]), st["v_new"].double()
    outs = []
    if kind == "append":
        for cache, new in ((st["k"], k), (st["v"], v)):
            flat = cache.double().view(-1, case["hkv"], d)
            flat[st["slots"][live].long()] = new[live]
            outs.append(flat.view(cache.shape))
    else:
        held = []
        p = st["pos"][live].long()
        pg = st["table"][live // case["rows"], p // page].long()
        for codes, scales, new in ((st["k4"], st["k4s"], k.float().to(dt).double()), (st["v4"], st["v4s"], v)):
            code, scale = _nearest(new)
            codes[pg, :, p % page] = code[live]
            scales[pg, :, p % page] = scale[live]
            held.append(_value(code, scale))
            outs += [codes, scales]
    if case["with_q"]:
        outs.append(_turned(st, st["q"]))
    if kind == "append_mx" and case["held"]:
        outs += held
    return outs


def _turned(st, x):
    """Pairs as complex numbers times e^(i theta)."""
    c = st["case"]
    rot, sign = c["rot"], -1.0 if c["inverse"] else 1.0
    theta = torch.stack([st["rope_pos"][int(a)].double() * float(f) for a, f in zip(st["axis"], st["inv"])], -1)
    turn = torch.polar(torch.ones_like(theta), sign * theta)[:, None]
    x = x.double()
    head = x[..., :rot].unflatten(-1, (2, -1) if c["pairing"] == HALVES else (-1, 2))
    dim = -2 if c["pairing"] == HALVES else -1
    z = torch.complex(head.select(dim, 0).contiguous(), head.select(dim, 1).contiguous()) * turn
    return torch.cat((torch.stack((z.real, z.imag), dim).flatten(-2), x[..., rot:]), -1)


def _value(codes, scales):
    """Values of code and scale bytes from their bits: sign, two exponent bits, one
    mantissa bit."""
    nib = torch.stack((codes % 16, codes // 16), -1).flatten(-2).long()
    sign, expo, man = 1.0 - 2.0 * (nib // 8).double(), (nib // 2) % 4, (nib % 2).double()
    mag = torch.where(expo == 0, man / 2, (1 + man / 2) * 2.0 ** (expo - 1).double())
    return sign * mag * 2.0 ** (scales.double().repeat_interleave(32, -1) - 127.0)


def _nearest(x):
    """Code and scale bytes of x by distance: the smallest scale that holds the
    block's largest value, then the nearest magnitude (the even code of two)."""
    blocks = x.unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    s = torch.full_like(top, 252.0)
    low = torch.floor(torch.log2(top.clamp(min=1e-300))) - 4
    for step in range(5, -1, -1):  # candidates from large to small, the smallest that holds
        cand = low + step
        s = torch.where(top <= 6.0 * 2.0 ** cand, cand + 127.0, s)
    s = s.clamp(2.0, 252.0)
    y = blocks / 2.0 ** (s - 127.0)[..., None]
    best, code = torch.full_like(y, math.inf), torch.zeros_like(y, dtype=torch.uint8)
    for i in (0, 2, 4, 6, 1, 3, 5, 7):  # even codes first: they keep a tie
        dist = (y.abs() - MAGNITUDES[i]).abs()
        code = torch.where(dist < best, torch.full_like(code, i), code)
        best = torch.minimum(best, dist)
    code = (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] + 16 * code[..., 1], s.to(torch.uint8)


def _exact_attention(st):
    c = st["case"]
    r, hq, hkv, d, page = c["rows"], c["hq"], c["hkv"], c["d"], c["page"]
    g = hq // hkv
    n = c["n_seqs"] * r
    o = torch.zeros(n, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=DEV)
    pos = st["pos"].view(-1, r).tolist()
    for s in range(c["n_seqs"]):
        length = max(pos[s]) + 1
        if length == 0:
            continue
        pages = st["table"][s, : -(-length // page)].long()
        at = st["pos"].view(-1, r)[s]
        for h in range(hkv):
            k = _value(st["k4"][pages, h], st["k4s"][pages, h]).reshape(-1, d)[:length]
            v = _value(st["v4"][pages, h], st["v4s"][pages, h]).reshape(-1, d)[:length]
            hidden = torch.arange(length, device=DEV)[None] > at[:, None]
            for j in range(h * g, (h + 1) * g):
                w = (st["q"][s * r:(s + 1) * r, j].double() @ k.t()) / math.sqrt(d)
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
    row4 = hkv * (d // 2 + d // 32)                    # bytes of a token's keys (or values) in 4 bits
    kind = case["kind"]
    if kind == "rotary":
        return {"bytes": 2 * n * hq * d * es + 4 * case["axes"] * n, "flops": 3 * n * hq * case["rot"]}
    q = 2 * n * hq * d * es if case["with_q"] else 0
    q_flops = 3 * n * hq * case["rot"] if case["with_q"] else 0
    ids = 4 * (case["axes"] + 1) * n
    if kind == "append":
        return {"bytes": 4 * live * hkv * d * es + q + ids, "flops": 3 * live * hkv * case["rot"] + q_flops}
    if kind == "append_mx":
        held = 2 * n * hkv * d * es if case["held"] else 0
        return {"bytes": 2 * live * (hkv * d * es + row4) + held + q + ids,
                "flops": live * hkv * (3 * case["rot"] + 4 * d) + q_flops}
    if kind == "load_mx":
        return {"bytes": 2 * n * (row4 + hkv * d * es) + ids, "flops": n * hkv * (3 * case["rot"] + 2 * d)}
    lengths = [case["ctx"]] * n_seqs
    if case["ragged"]:
        lengths = [r + int((case["ctx"] - r) * (i + 1.0) / n_seqs) for i in range(n_seqs)]
    share = (n_seqs - case["pad"]) / n_seqs
    if case["spread"]:
        keys, pairs = sum(lengths), sum(length * r / 2 for length in lengths)
    else:
        keys, pairs = sum(lengths), sum(length * r - r * (r - 1) / 2 for length in lengths)
    return {"bytes": int(share * keys) * 2 * row4 + 2 * n * hq * d * es + 4 * n * hq + 4 * n,
            "flops": int(share * pairs) * 4 * hq * d}
