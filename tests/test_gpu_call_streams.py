"""Memory that a call takes for itself belongs to the stream that uses it."""
import numpy as np
import pytest
import torch

from paper_2609_05821_amd import api, workloads as W
from tests.gpu_helpers import DEV, to_dev
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


def scoring_and_refresh():
    """{call: (what it needs, the call on a stream)} over two layers of one cache."""
    w = W.custom(1, 8, 2, 64, 40, 7, [700, 533], 3, "bf16", seed=4)
    L = w.layer(0)
    k, v, q = (to_dev(L[x]) for x in ("k", "v", "q"))
    kv, img = api.kv_desc(k, v, w.n_q_heads), api.ImageTable(w.img_pos, w.img_off)
    sel = np.arange(0, w.n_vis, 5)
    pos = torch.from_numpy(w.vis_positions()[sel].astype(np.int32)).to(DEV)
    kn, vn, qn = (to_dev(np.ascontiguousarray(L[x][sel])) for x in ("k_star", "v_star", "q_star"))
    f32 = dict(dtype=torch.float32, device=DEV)
    s, a, lse = torch.zeros(w.n_vis, **f32), torch.zeros(w.n_vis, **f32), torch.zeros((w.n_q, w.n_q_heads), **f32)
    err, out = torch.zeros((1, w.n_q, w.n_q_heads), **f32), [torch.empty_like(qn) for _ in range(2)]
    idx, at = (torch.zeros(len(sel), dtype=torch.int32, device=DEV) for _ in range(2))
    mask = torch.zeros(w.n_vis, dtype=torch.uint8, device=DEV)
    n = len(sel)
    return {
        "score": (api.score_workspace_bytes(kv, w.n_q, img),
                  lambda st: api.conduit_score(kv, q, w.q_pos0, img, s, a, row_lse_out=lse, stream=st)),
        "score_layers": (api.score_layers_workspace_bytes(kv, w.n_q, img, 2),
                         lambda st: api.conduit_score_layers([kv, kv], [q, q], w.q_pos0, img, s, a, stream=st)),
        "select": (int(api.lib().conduit_select_workspace_bytes(w.n_vis, w.n_images)),
                   lambda st: api.conduit_select_topk(s, a, 1, img, 1.0, n, idx, at, stream=st)),
        "refresh": (api.refresh_workspace_bytes(kv, n),
                    lambda st: api.conduit_refresh_attn(kv, qn, pos, out[0], stream=st)),
        "refresh_layers": (api.refresh_layers_workspace_bytes(kv, n, 2),
                           lambda st: api.conduit_refresh_attn_layers([kv, kv], [qn, qn], pos, out, stream=st)),
        "merge_refresh": (api.refresh_workspace_bytes(kv, n),
                          lambda st: api.conduit_merge_refresh_attn(kv, pos, kn, vn, qn, out[0], stream=st)),
        "residual": (api.residual_workspace_bytes(kv, w.n_q, img, 1, False),
                     lambda st: api.conduit_residual_error(kv, q, w.q_pos0, img, lse, mask, err, stream=st))}


@pytest.mark.parametrize("name", ["score", "score_layers", "select", "refresh", "refresh_layers", "merge_refresh",
                                  "residual"])
def test_scoring_and_refresh(name):
    need, call = scoring_and_refresh()[name]
    s = torch.cuda.Stream()
    own, default = taken(lambda: call(s), s)
    assert own >= need and default == 0
