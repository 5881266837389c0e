"""Which calls of the 8-bit attention take blocks of 256 (row, head) pairs, seen in the workspace that they ask for,
without a GPU."""
import os

import pytest

from paper_2609_05821_amd import api
from tests.test_abi_byte_cpu import parts, workspace

pytestmark = pytest.mark.skipif(not os.path.exists(api.LIB_PATH),
                                reason="libconduit.so not built (run __graft_entry__.build())")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_seqs,hkv,pairs", [(8, 4, 256), (1, 1, 8192), (2, 1, 4096), (16, 4, 160), (1, 8, 1000)])
def test_short_caches_that_fill_the_chip(d, n_seqs, hkv, pairs):
    """256 to 1,023 blocks of 32 pairs, each done by one workgroup (no workspace): where the 256 CUs have up to 2^20 keys
    in all they are done sooner than blocks of 256 pairs."""
    blocks = n_seqs * hkv * -(-pairs // 32)
    assert 256 <= blocks < 1024
    most = (1 << 20) // (-(-blocks // 256) * 256)
    for ctx in (64, -(-(1 << 18) // blocks), most - 1, most):
        assert workspace(n_seqs, pairs, 1, d, ctx=ctx, hkv=hkv) == 0, ctx
    wide = n_seqs * -(-pairs // 256)
    if wide * hkv < 256 and most >= 8 * 128:                 # (their steps are shared)
        assert workspace(n_seqs, pairs, 1, d, ctx=most + 1, hkv=hkv) == shared(wide, hkv, most + 1, d)


def shared(n_sb, hkv, ctx, d):
    """The workspace of blocks of 256 pairs whose steps of 128 keys workgroups share, two steps each or more."""
    return parts(min(256, n_sb * hkv * -(-ctx // 128) // 2), 256, n_sb, d)


@pytest.mark.parametrize("d", [64, 128])
def test_long_caches_and_fewer_blocks(d):
    """As before: from 2^18 keys of all blocks on where those are fewer than 256, and where they fill the chip with longer caches."""
    long = (1 << 18) // 7 + 1
    assert workspace(1, 7 * 32, 1, d, ctx=long) == shared(1, 1, long, d)
    assert workspace(1, 255 * 32, 1, d, ctx=1029) == shared(32, 1, 1029, d)
    assert workspace(64, 256, 1, d, ctx=4096, hkv=4) == shared(64, 4, 4096, d)
    assert workspace(1, 1024 * 32, 1, d, ctx=1025) == shared(128, 1, 1025, d)
