"""Plain 64-bit definitions of rotary positions, the 4-bit cache and attention
over it, on the CPU (torch float64), for the parity tests."""
from __future__ import annotations

import math

import torch

MAG = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def turned(x, inv_freq, axis, pos, adjacent=False, inverse=False):
    """x [n, H, d] (any dtype) turned; pos [axes, n]; float64."""
    x = x.double()
    half = len(inv_freq)
    w = torch.as_tensor(inv_freq, dtype=torch.float32).double()
    ax = torch.zeros(half, dtype=torch.long) if axis is None else torch.as_tensor(axis).long()
    theta = pos.double()[ax].t() * w * (-1.0 if inverse else 1.0)          # [n, half]
    c, s = theta.cos()[:, None], theta.sin()[:, None]
    y = x.clone()
    ia = torch.arange(half) * 2 if adjacent else torch.arange(half)
    ib = ia + 1 if adjacent else ia + half
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, a * s + b * c
    return y


def rounded(x, dtype):
    """64 bits -> fp32 -> dtype, the order of roundings of the kernels."""
    return x.float().to(dtype)


def pack(x):
    """(codes [.., d/2], scales [.., d/32]) of rows x [n, H, d] in their cache dtype,
    without the rule for non-finite heads."""
    blocks = x.double().unflatten(-1, (-1, 32))
    top = blocks.abs().amax(-1)
    s = torch.full(top.shape, 252, dtype=torch.long)
    for byte in range(252, 1, -1):
        s = torch.where(top <= 6.0 * 2.0 ** (byte - 127), byte, s)
    y = blocks / torch.pow(2.0, (s - 127).double())[..., None]
    dist = (y.abs()[..., None] - MAG).abs()
    dist = dist + torch.tensor([0, 1, 0, 1, 0, 1, 0, 1]) * 1e-13            # ties to the even code
    code = dist.argmin(-1) + 8 * torch.signbit(y).long()
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), s.to(torch.uint8)


def pack_rows(k, v):
    """pack of keys and values with the rule for heads that hold an infinity or a NaN."""
    bad = ~(torch.isfinite(k.double()).all(-1) & torch.isfinite(v.double()).all(-1))
    zero = torch.zeros((), dtype=k.dtype)
    kc, ks = pack(torch.where(bad[..., None], zero, k))
    vc, vs = pack(torch.where(bad[..., None], zero, v))
    ks[bad] = 255
    return kc, ks, vc, vs


def held(codes, scales):
    """Values (float64) of code and scale bytes; scale byte 255 is NaN."""
    nib = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    x = MAG[nib & 7] * torch.where(nib >= 8, -1.0, 1.0).double()
    f = torch.pow(2.0, scales.double() - 127.0)
    f = torch.where(scales == 255, math.nan, f)
    return x * f.repeat_interleave(32, -1)


def gather(pool, table, seq, pos, page):
    """Rows of a pool [n_pages, H, page, b]: token pos[i] of sequence seq[i]."""
    return pool[table[seq, pos // page].long(), :, pos % page]


def attention(q, k, v, pos, scale=None):
    """One sequence: q [n, Hq, d], k, v [len, Hkv, d] (float64), pos [n] (-1: empty).
    Returns o, lse, and for tolerances: sum p|v| / sum p per output and
    scale * sum |q||k| maximised over the row's keys."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    q = q.double()
    o = torch.zeros(n, hq, d, dtype=torch.float64)
    av = torch.zeros_like(o)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64)
    mag = torch.zeros(n, hq, dtype=torch.float64)
    for i in range(n):
        m = min(int(pos[i]) + 1, k.shape[0])
        if m <= 0:
            continue
        kk = k[:m].repeat_interleave(g, 1)
        vv = v[:m].repeat_interleave(g, 1)
        logits = (kk * q[i]).sum(-1).t() * scale                              # [hq, m]
        lse[i] = torch.logsumexp(logits, -1)
        p = torch.exp(logits - lse[i][:, None])
        o[i] = torch.einsum("hm,mhd->hd", p, vv)
        av[i] = torch.einsum("hm,mhd->hd", p, vv.abs())
        mag[i] = ((kk.abs() * q[i].abs()).sum(-1).t() * scale).amax(-1)
    return o, lse, av, mag


def attention_bounds(o, lse, av, mag, n_keys, d, bf16):
    """Elementwise bounds of the kernel's error.  Logits: d products added in fp32,
    then the scale and the exponent's argument, each at most 2^-24 of mag;
    twice (numerator and denominator).  Probabilities: exponential 2^-22, for
    bf16 rounded to 8 bits (half a step, 2^-8).  Sums of n_keys terms in fp32
    (numerator and denominator), merges of parts within 64 more roundings.
    Output: one rounding."""
    es = 2 * (d + 8) * 2.0 ** -24 * mag + 2 * 2.0 ** -22 + 2 * (n_keys + 64) * 2.0 ** -24
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    bo = (es + (half if bf16 else 0.0))[..., None] * av + half * o.abs() + 1e-30
    bl = es + 2.0 ** -21 * lse.abs().nan_to_num(0.0, 0.0, 0.0) + 2.0 ** -22
    return bo, bl
