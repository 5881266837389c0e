"""Attention over an 8-bit cache on either side of the sizes at which calls change from a workgroup per block of 32 (row,
head) pairs to blocks of 256."""
import pytest
import torch

from tests import byte_oracle as B
from tests import mx_oracle as M
from tests.test_gpu_attn_byte import queries
from tests.test_gpu_attn_byte_sharp import Shared
from tests.test_gpu_attn_mx_sharp import half_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_seqs,r,hq,hkv,d,ctx", [(8, 64, 16, 4, 128, 4096), (16, 40, 16, 4, 64, 2048),
                                                   (1, 2049, 4, 4, 128, 1024), (16, 20, 32, 8, 64, 1100)])
@pytest.mark.parametrize("more", [0, 1])
def test_either_side(n_seqs, r, hq, hkv, d, ctx, more):
    """bf16 outputs: half a step of their own rounding, 2^-17 of each probability in blocks of 32 pairs and
    2^-11 or what fp16 loses below its normal numbers in blocks of 256, and the errors of 32-bit logits and sums."""
    pairs = r * hq // hkv
    blocks = n_seqs * hkv * -(-pairs // 32)
    last = (1 << 20) // (-(-blocks // 256) * 256)
    assert 256 <= blocks < 1024 and ctx <= last
    ctx = last + 1 if more else ctx
    st = Shared(n_seqs, ctx, hq, hkv, d, seed=ctx)
    g = torch.Generator().manual_seed(r)
    q, pos = queries(n_seqs * r, hq, d, "bf16", r), torch.randint(-1, ctx, (n_seqs * r,), generator=g, dtype=torch.int32)
    o, lse = st.run(q, pos)
    sel = torch.cat([torch.arange(0, n_seqs * r, max(1, n_seqs * r // 30)), torch.tensor([n_seqs * r - 1])])
    want, want_lse, av, mag = M.attention(q[sel], st.k, st.v, pos[sel])
    err, err_lse = B.attention_bounds(want, want_lse, av, mag, ctx, d, False)
    err = err + 2.0 ** (-11 if more else -17) * av
    if more:
        err = err + B.weight_floor(q[sel], st.k, st.v, st.factors, pos[sel], want_lse)
    bound = err + half_step(want.abs() + err)
    assert ((o[sel] - want).abs() <= bound).all(), f"{((o[sel] - want).abs() / bound).max():.3g} of the bound"
    live = pos[sel] >= 0
    assert ((lse[sel] - want_lse).abs()[live] <= err_lse[live]).all()
    assert (o[pos < 0] == 0).all() and (lse[pos < 0] == -float("inf")).all()
