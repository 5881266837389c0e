"""An append to the 8-bit cache of as many rows as workgroups for every two of them would pass 2^32 threads."""
import pytest
import torch

from paper_2609_05821_amd import api
from tests.gpu_helpers import DEV
from tests.test_gpu_rotary import rope_of

pytestmark = pytest.mark.gpu

HEADS, D, PAGE = 4, 64, 1 << 18


def empty_cache(n):
    per = -(-n // PAGE)
    codes = [torch.zeros(per, HEADS, PAGE, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros(per, HEADS, PAGE // 16, dtype=torch.uint8, device=DEV) for _ in range(2)]
    return codes + scales, api.byte_desc(*codes, *scales, HEADS, n)


def test_more_rows_than_two_a_workgroup():
    """2^24 rows and a few more, 4 heads of keys, values and queries, against calls of a quarter each."""
    n = (1 << 24) + 48
    x, q = (torch.empty(n, HEADS, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for i in range(0, n, 1 << 20):
        x[i:i + (1 << 20)].normal_()
        q[i:i + (1 << 20)].normal_()
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    rope, rp = rope_of(16, 1, 0), (pos % 9001)[None].contiguous()
    want_q = q.clone()
    whole, cache = empty_cache(n)
    api.conduit_append_byte(cache, pos, x, x, rope=rope, rope_pos=rp, q=q, q_out=q)
    parts, cache = empty_cache(n)
    for i in range(0, n, 1 << 22):
        j = min(n, i + (1 << 22))
        api.conduit_append_byte(cache, pos[i:j], x[i:j], x[i:j], rope=rope, rope_pos=rp[:, i:j].contiguous())
        api.conduit_rotary(want_q[i:j], rope, rp[:, i:j].contiguous(), want_q[i:j])
    for a, b in zip(whole, parts):
        for p, r in zip(a, b):
            assert torch.equal(p, r)
    for i in range(0, n, 1 << 22):
        assert torch.equal(q[i:i + (1 << 22)], want_q[i:i + (1 << 22)])
