"""Attention over a 4-bit cache with queries and keys of every magnitude, their products
ordinary."""
import pytest
import torch

from tests.test_gpu_attn_mx import Store, check, queries, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 300), (3, 1500), (60, 1200)])
@pytest.mark.parametrize("log2", [-118, -100, 100, 118])
def test_small_and_large(dtype, r, ctx, log2):
    """Down to queries of 2^-118, whose smaller parts are subnormal in bf16."""
    st = Store(1, ctx, 4, 2, 128, seed=ctx)
    st.cpu[2][:] = 125 - log2
    st.upload()
    q = (queries(r, 4, 128, "f32", r).double() * 2.0 ** log2).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    pos = torch.linspace(ctx - 1, ctx // 3, r).to(torch.int32)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("r,ctx", [(1, 300), (3, 1500), (60, 1200)])
def test_largest(dtype, r, ctx):
    """Queries up to the largest finite number: in fp32 it rounds up to an infinity in bf16."""
    st = Store(1, ctx, 4, 2, 128, seed=ctx)
    st.cpu[2][:] = 2
    st.upload()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    top = torch.finfo(dt).max
    q = ((torch.rand(r, 4, 128, generator=torch.Generator().manual_seed(r), dtype=torch.float64) * 2 - 1) * top).to(dt)
    q[:, :, ::50], q[:, :, 7::40] = top, -top
    pos = torch.linspace(ctx - 1, ctx // 3, r).to(torch.int32)
    o, lse = run(st, q, pos)
    check(st, q, pos, o, lse)
