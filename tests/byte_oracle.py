"""Plain 64-bit definitions of the 8-bit cache on the CPU (torch float64), for the
parity tests: e4m3 codes, a scale byte per 16 tokens and head, and what an append
leaves of a block."""
from __future__ import annotations

import math

import torch

BLOCK, LOW, HIGH, NAN = 16, 10, 246, 0x7f


def decoded(codes):
    """Values (float64) of code bytes."""
    b = codes.long()
    e, m = (b >> 3) & 15, (b & 7).double()
    mag = torch.where(e == 0, m / 512, (8 + m) * torch.pow(2.0, (e - 10).double()))
    mag = torch.where(b & 127 == NAN, math.nan, mag)
    return torch.where(b >= 128, -mag, mag)


TABLE = decoded(torch.arange(127))


def nearest(y):
    """Code bytes of y (float64): the nearest, ties to the even code, the largest above it."""
    a = y.abs().clamp(max=448.0)
    hi = torch.searchsorted(TABLE, a.contiguous()).clamp(1, 126)
    below, above = a - TABLE[hi - 1], TABLE[hi] - a
    lower = (below < above) | ((below == above) & (hi % 2 == 1))
    code = torch.where(lower, hi - 1, hi) + 128 * torch.signbit(y).long()
    return torch.where(y.isnan(), NAN, code).to(torch.uint8)


def needed(top):
    """The smallest scale byte with top <= 448 * 2^(s - 127)."""
    for s in range(LOW, HIGH):
        if top <= 448.0 * 2.0 ** (s - 127):
            return s
    return HIGH


def clamped(scale):
    return min(max(int(scale), LOW), HIGH)


def factor(scales):
    """2^(s - 127) (float64) of scale bytes."""
    return torch.pow(2.0, scales.long().clamp(LOW, HIGH).double() - 127.0)


class Pools:
    """Pools [page][head][slot][d] and [page][head][slot / 16] on the CPU and what appends
    do to them, token by token."""

    def __init__(self, k, v, ks, vs, table, page, ctx):
        self.pool = dict(k=(k.clone(), ks.clone()), v=(v.clone(), vs.clone()))
        self.table, self.page, self.ctx = table, page, ctx

    def place(self, s, t):
        n_pages = self.pool["k"][0].shape[0]
        return min(max(int(self.table[s, t // self.page]), 0), n_pages - 1), t % self.page

    def append(self, pos, k, v, n_held=None):
        """Rows k, v [n, H, d] in their cache dtype, the keys turned.  Returns the rows as
        held (float64)."""
        n, hkv, _ = k.shape
        r = n // self.table.shape[0]
        fine = k.double().isfinite().all(-1) & v.double().isfinite().all(-1)       # [n, H]
        held = dict(k=torch.zeros(k.shape, dtype=torch.float64), v=torch.zeros(v.shape, dtype=torch.float64))
        runs = {}
        for i in range(n):
            t = int(pos[i])
            if 0 <= t < self.ctx:
                runs.setdefault((i // r, t // BLOCK), {})[t % BLOCK] = i
            else:
                runs[("out", i)] = {0: i}
        for (s, b), rows in runs.items():
            out = s == "out"
            if out:
                kept = []
            else:
                end = b * BLOCK + max(rows) if n_held is None else min(max(int(n_held[s]), 0), self.ctx)
                kept = [j for j in range(BLOCK) if j not in rows and b * BLOCK + j < end]
                page, slot0 = self.place(s, b * BLOCK)
            for h in range(hkv):
                for name, new in (("k", k), ("v", v)):
                    codes, scales = self.pool[name]
                    x = {j: new[i, h].double() for j, i in rows.items()}
                    top = max([float(x[j].abs().max()) for j, i in rows.items() if fine[i, h]], default=0.0)
                    now = needed(top)
                    if kept:
                        was = clamped(scales[page, h, slot0 // BLOCK])
                        now = max(now, was)
                        if now > was:
                            for j in kept:
                                old = decoded(codes[page, h, slot0 + j])
                                codes[page, h, slot0 + j] = nearest(old * 2.0 ** (was - now))
                    for j, i in rows.items():
                        c = nearest(x[j] * 2.0 ** (127 - now))
                        if not fine[i, h]:
                            c = torch.full_like(c, NAN if name == "k" else 0)
                        held[name][i, h] = decoded(c) * 2.0 ** (now - 127)
                        if not out:
                            codes[page, h, slot0 + j] = c
                    if not out:
                        scales[page, h, slot0 // BLOCK] = now
        return held["k"], held["v"]

    def rows(self, s, n):
        """Keys and values (float64) of tokens 0 .. n - 1 of sequence s."""
        out = []
        for name in ("k", "v"):
            codes, scales = self.pool[name]
            at = [self.place(s, t) for t in range(n)]
            pg, sl = torch.tensor([a for a, _ in at]).long(), torch.tensor([b for _, b in at]).long()
            out.append(decoded(codes[pg, :, sl]) * factor(scales[pg, :, sl // BLOCK])[..., None])
        return out


def attention_bounds(o, lse, av, mag, n_keys, d, bf16):
    """Elementwise bounds of the kernel's error (o, lse, av, mag of mx_oracle.attention).
    Logits: d products added in fp32, then the scale and the exponent's argument, each
    at most 2^-24 of mag; twice (numerator and denominator).  Exponential 2^-22.  For bf16
    tensors the probabilities enter the product as fp16 numbers or better: of a number in [2^e, 2^(e+1)) fp16 keeps
    11 bits, its steps are 2^(e-10), and half a step is up to 2^-11 of the number.  Sums of
    n_keys terms in fp32 (numerator and denominator), merges of parts within 64 more
    roundings.  Output: one rounding, half a step."""
    es = 2 * (d + 8) * 2.0 ** -24 * mag + 2 * 2.0 ** -22 + 2 * (n_keys + 64) * 2.0 ** -24
    bo = (es + (2.0 ** -11 if bf16 else 0.0))[..., None] * av + (2.0 ** -8 if bf16 else 2.0 ** -24) * o.abs() + 1e-30
    bl = es + 2.0 ** -21 * lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2.0 ** -22
    return bo, bl


def weight_floor(q, k, v, factors, pos, lse, scale=None):
    """bf16 with many pairs: probabilities enter the product in fp16, as p_t f_t (f: the
    factor of the block's scale) over 2^-11 times a power of two that is at most 2^4 below
    and no more than the row's largest p_t f_t above it.  Below fp16's normal numbers a
    weight is off by up to half its smallest step, 2^-25, so by 2^-36 max(p f): times the
    codes, summed over the row's keys.  q [n, Hq, d], k, v [len, Hkv, d], factors [len, Hkv]."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    codes = v.abs() / factors[..., None]
    out = torch.zeros(n, hq, d, dtype=torch.float64)
    for i in range(n):
        m = min(int(pos[i]) + 1, k.shape[0])
        if m > 0:
            logits = (k[:m].repeat_interleave(g, 1) * q[i].double()).sum(-1) * scale        # [m, hq]
            largest = (torch.exp(logits - lse[i]) * factors[:m].repeat_interleave(g, 1)).amax(0)
            out[i] = 2.0 ** -36 * largest[:, None] * codes[:m].sum(0).repeat_interleave(g, 0)
    return out
