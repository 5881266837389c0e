"""Memory that a call takes for itself belongs to the stream that uses it."""
import torch

import pytest

from paper_2609_05821_amd import api
from tests.gpu_helpers import DEV
from tests.test_gpu_attn_mx import Store, queries

pytestmark = pytest.mark.gpu


def held_by(stream):
    """Bytes of the allocator's segments that belong to the stream's pool."""
    return sum(s["total_size"] for s in torch.cuda.memory_snapshot() if s["stream"] == stream.cuda_stream)


def taken(call, stream):
    """Bytes by which the pools of the given stream and of the default stream grow in the call."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    streams = (stream, torch.cuda.default_stream())
    before = [held_by(s) for s in streams]
    call()
    torch.cuda.synchronize()
    return [held_by(s) - b for s, b in zip(streams, before)]


def test_attention_over_4_bits():
    """A block of the current stream's pool may be in use there still, and what is queued
    there would overwrite the workspace while the call reads it."""
    st = Store(1, 3000, 4, 2, 128, seed=1)
    q, pos = queries(1, 4, 128, "bf16", 1).to(DEV), torch.tensor([2999], dtype=torch.int32, device=DEV)
    need = api.attn_mx_workspace_bytes(st.mx, q)
    o, want = torch.empty_like(q), torch.empty_like(q)
    api.conduit_attn_mx(st.mx, q, pos, want)
    s = torch.cuda.Stream()
    own, default = taken(lambda: api.conduit_attn_mx(st.mx, q, pos, o, stream=s), s)
    assert need > 0 and own >= need and default == 0
    assert torch.equal(o, want)
