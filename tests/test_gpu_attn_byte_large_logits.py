"""Attention over an 8-bit cache with logits up to the largest that the call takes, over values whose
scales differ from block to block: the weights of blocks with different scales stay in proportion."""
import pytest
import torch

from paper_2609_05821_amd import api
from tests import byte_oracle as B
from tests.gpu_helpers import DEV
from tests.test_gpu_rotary import DT

pytestmark = pytest.mark.gpu


class Chosen:
    """One sequence of ctx keys of d dims, every code that of the number 1 and every scale 1 to begin with: a query
    of x in every dim has the logit scale d x f over a key of the scale f, in fp32 exactly."""

    def __init__(self, ctx, d, seed, low, high):
        g = torch.Generator().manual_seed(seed)
        per = -(-ctx // 64)
        self.ctx, self.d = ctx, d
        self.k = torch.full((per, 1, 64, d), 0x38, dtype=torch.uint8)
        self.v = torch.randint(0x20, 0x58, (per, 1, 64, d), generator=g).to(torch.uint8)        # 2^-3 to 15
        self.v |= (128 * torch.randint(0, 2, self.v.shape, generator=g)).to(torch.uint8)
        self.ks = torch.full((per, 1, 4), 127, dtype=torch.uint8)
        self.vs = torch.randint(low, high + 1, (per, 1, 4), generator=g).to(torch.uint8)

    def attend(self, x, pos, wide, scale=1.0):
        """Rows of one head, scale times as large logits as x.  wide: the cache has room for 2^18 tokens, so that 256 (row, head) pairs are a block."""
        pools = [t.to(DEV) for t in (self.k, self.v, self.ks, self.vs)]
        table = torch.zeros(1, 4096, dtype=torch.int32)
        table[0, :len(self.k)] = torch.arange(len(self.k))
        cache = api.byte_desc(*pools, 1, 2 ** 18, table.to(DEV)) if wide else api.byte_desc(*pools, 1, self.ctx)
        q = x[:, None, None].expand(len(x), 1, self.d).contiguous()
        o = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
        lse = torch.full(q.shape[:2], 9.0, device=DEV)
        api.conduit_attn_byte(cache, q.to(DEV), pos.to(DEV), o, lse_out=lse, scale=scale / self.d)
        return o[:, 0].cpu().double(), lse[:, 0].cpu().double()

    def factors(self, scales):
        return B.factor(scales).flatten().repeat_interleave(16)[:self.ctx]

    def values(self):
        """Values, and what a weight held in fp16 is off by below its normal numbers (2^-36 of the largest
        weight times scale) counts: codes times that."""
        code = B.decoded(self.v).reshape(-1, self.d)[:self.ctx]
        return code * self.factors(self.vs)[:, None], code.abs()


def bound(want, magnitudes, dtype, wide):
    """Weights off by 2^-11 (256 pairs a block, bf16), 2^-17 (few), for sums of up to 1,000 terms a lane
    2^-14, for exponents' arguments of up to 2,048 half a step of 2^-13, 2^-14 with the factor ln 2 to a weight; the output rounded once."""
    weights = (2.0 ** -11 if wide and dtype == "bf16" else 2.0 ** -17) + 2.0 ** -14 + 2.0 ** -14
    return weights * magnitudes + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * want.abs()


def check_lse(lse, want):
    assert ((lse - want).abs() <= 2.0 ** -20 * want.abs() + 2.0 ** -12).all()


# rows, keys, and whether the cache is a large one
SHAPES = [(1, 300, False), (40, 700, False), (150, 5300, False), (300, 300, True), (300, 5300, True),
          (300, 16000, True)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,ctx,wide", SHAPES)
@pytest.mark.parametrize("low,high", [(117, 121), (10, 225), (100, 140)])
@pytest.mark.parametrize("sign", [1, -1])
def test_equal_logits_over_values_of_other_scales(dtype, d, rows, ctx, wide, low, high, sign):
    """Every key has the same logit, by row from 2^3 to 2^29 above or below 0: the output is the mean of the
    values, whatever scales their blocks have (sums of up to 16,000 values of 15 2^98 stay below 2^119)."""
    c = Chosen(ctx, d, ctx + low, low, high)
    exponent = 3 + torch.arange(rows) * 7 % 27
    x = sign * torch.pow(2.0, exponent.double())
    o, lse = c.attend(x.to(DT[dtype]), torch.full((rows,), ctx - 1, dtype=torch.int32), wide)
    v, code = c.values()
    want = v.mean(0)
    err = bound(want, v.abs().mean(0), dtype, wide)
    if wide and dtype == "bf16":
        err = err + 2.0 ** -36 * c.factors(c.vs).max() * code.mean(0)
    bad = ~((o - want).abs() <= err)
    assert not bad.any(), f"rows with logits of 2^{sorted(set(exponent[bad.any(1)].tolist()))}"
    check_lse(lse, x + torch.log(torch.tensor(float(ctx), dtype=torch.float64)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,ctx,wide", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_keys_that_stand_out(dtype, d, rows, ctx, wide, sign):
    """Three blocks of the first 32 and two of every 32 after have the largest logit, 2^6 to 2^28 above the others: the
    output is the mean of their values.  (The others weigh less than 16,000 e^-64 15 2^13, 2^-61, in all.)"""
    c = Chosen(ctx, d, ctx, 100, 140)
    top = torch.zeros(c.ks.numel(), dtype=torch.bool)
    top[0] = top[7::32] = top[24::32] = True
    c.ks.view(-1)[top if sign > 0 else ~top] = 128               # keys of 2 among keys of 1
    pos = torch.randint(min(400, ctx // 2), ctx, (rows,), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    exponent = 6 + torch.arange(rows) * 7 % 23
    x = sign * torch.pow(2.0, exponent.double())
    o, lse = c.attend(x.to(DT[dtype]), pos, wide)
    out = top.repeat_interleave(16)[:ctx].double()[:, None]
    v, code = c.values()
    value, magnitude, codes, count = (t.cumsum(0)[pos.long()] for t in (v * out, v.abs() * out, code * out, out))
    want = value / count
    err = bound(want, magnitude / count, dtype, wide) + 2.0 ** -60
    if wide and dtype == "bf16":
        err = err + 2.0 ** -36 * c.factors(c.vs).max() * codes / count
    bad = ~((o - want).abs() <= err)
    assert not bad.any(), f"rows with logits of 2^{sorted(set(exponent[bad.any(1)].tolist()))}"
    check_lse(lse, x * (2 if sign > 0 else 1) + torch.log(count[:, 0]))


@pytest.mark.parametrize("dtype,wide", [("bf16", True), ("bf16", False), ("f32", True)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
@pytest.mark.parametrize("sign", [1, -1])
def test_logits_of_every_size(dtype, wide, d, order, sign):
    """Keys of 21 magnitudes a factor of two apart, 256 keys each or block by block, for rows of magnitudes of their own:
    logits of 2^-3 to 2^28."""
    rows, ctx = 300, 5300
    c = Chosen(ctx, d, 5, 110, 130)
    n = c.ks.numel()
    step = torch.arange(n) // 16
    step = dict(rising=step, falling=20 - step,
                mixed=torch.randint(0, 21, (n,), generator=torch.Generator().manual_seed(6)))[order].clamp(0, 20)
    c.ks.view(-1)[:] = (112 + step).to(torch.uint8)
    pos = torch.randint(0, ctx, (rows,), generator=torch.Generator().manual_seed(4), dtype=torch.int32)
    pos[:4] = torch.tensor([0, 255, 256, ctx - 1])
    exponent = 12 + torch.arange(rows) * 5 % 12
    x = sign * torch.pow(2.0, exponent.double())
    o, lse = c.attend(x.to(DT[dtype]), pos, wide)
    v, code = c.values()
    for i in range(rows):
        seen = int(pos[i]) + 1
        logits = x[i] * c.factors(c.ks)[:seen]
        p = torch.softmax(logits, 0)[:, None]
        want = (p * v[:seen]).sum(0)
        err = bound(want, (p * v[:seen].abs()).sum(0), dtype, wide) + 2.0 ** -90
        if wide and dtype == "bf16":
            err = err + 2.0 ** -36 * (p[:, 0] * c.factors(c.vs)[:seen]).max() * code[:seen].sum(0)
        assert ((o[i] - want).abs() <= err).all(), f"row {i}, queries of 2^{int(exponent[i])}"
        check_lse(lse[i], torch.logsumexp(logits, 0))


@pytest.mark.parametrize("dtype,wide", [("bf16", True), ("bf16", False), ("f32", True)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("order", ["rising", "falling"])
def test_products_near_the_largest_number(dtype, wide, d, order):
    """Sums of products up to 2^126.6 of either sign in one row, whose differences are no finite numbers, with scales that
    make logits of up to 2^28 of them: the output is the mean over the keys with the row's largest."""
    rows, ctx = 300, 2000
    c = Chosen(ctx, d, 7, 110, 130)
    step = torch.arange(c.ks.numel()) * 8 // c.ks.numel()           # keys of -1.5, -1, -0.5, -0, 0, 0.5, 1 and 1.5
    if order == "falling":
        step = 7 - step
    size = torch.tensor([0x3c, 0x38, 0x30, 0, 0, 0x30, 0x38, 0x3c])[step] + 128 * (step < 4)
    c.k[:] = size.repeat_interleave(16).view(-1, 1, 64, 1).to(torch.uint8)
    number = B.decoded(c.k)[:, 0, :, 0].flatten()[:ctx]
    pos = torch.randint(0, ctx, (rows,), generator=torch.Generator().manual_seed(8), dtype=torch.int32)
    largest = 126 - (6 if d == 64 else 7)                            # 1.5 d x = 2^126.6
    x = torch.pow(2.0, (largest - torch.arange(rows) % 10).double()) * (1 - 2 * (torch.arange(rows) // 10 % 2))
    scale = 2.0 ** (27 - largest)
    o, lse = c.attend(x.to(DT[dtype]), pos, wide, scale)
    v, code = c.values()
    for i in range(rows):
        seen = int(pos[i]) + 1
        logits = x[i] * scale * number[:seen]
        p = torch.softmax(logits, 0)[:, None]
        want = (p * v[:seen]).sum(0)
        err = bound(want, (p * v[:seen].abs()).sum(0), dtype, wide)
        if wide and dtype == "bf16":
            err = err + 2.0 ** -36 * (p[:, 0] * c.factors(c.vs)[:seen]).max() * code[:seen].sum(0)
        assert ((o[i] - want).abs() <= err).all(), f"row {i}"
        check_lse(lse[i], torch.logsumexp(logits, 0))
