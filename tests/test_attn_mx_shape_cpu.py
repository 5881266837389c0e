"""How conduit_attn_mx cuts a call up, seen from its workspace: memory for parts and their
list where workgroups share the key steps, none where each has a block of its own."""
import ctypes
import os

import pytest

from paper_2609_05821_amd import api

pytestmark = pytest.mark.skipif(not os.path.exists(api.LIB_PATH),
                                reason="libconduit.so not built (run __graft_entry__.build())")

FAKE = 0x100000  # never dereferenced
LDS = 160 * 1024  # of a CU


def workspace(n_seqs, r, group, d, dtype=api.BF16, ctx=2048, hkv=1):
    mx = api.KVMX(FAKE, FAKE, FAKE, FAKE, hkv * 64 * d // 2, hkv * 64 * d // 32, 1 << 20, 64, n_seqs, ctx // 64, ctx,
                  FAKE, group * hkv, hkv, d)
    return int(api.lib().conduit_attn_mx_workspace_bytes(ctypes.byref(mx), n_seqs * r, dtype))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("blocks", [1, 64, 65, 2043, 2044, 2500, 4096, 4097])
def test_lists_leave_two_workgroups_a_cu(blocks, d):
    """128 pairs a block: four tiles of 64 values of d + 16 bf16, and the list."""
    used = 4 * 64 * (d + 16) * 2 + 16 + 4 * (blocks + 1)
    assert (workspace(blocks, 5, 7, d) > 0) == (blocks <= 4096 and 2 * used <= LDS)
    assert (workspace(1, blocks * 128, 1, d) > 0) == (blocks <= 4096 and 2 * used <= LDS)


@pytest.mark.parametrize("dtype", [api.BF16, api.F32])
@pytest.mark.parametrize("blocks,shared", [(4096, True), (4097, False)])
def test_lists_of_few_pairs(blocks, shared, dtype):
    assert (workspace(blocks, 1, 8, 128, dtype, ctx=8192) > 0) == shared


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan"), float("inf"), 1e-40, 2.0 ** 127, 3e38])
def test_scales_that_fp32_cannot_carry(scale):
    """scale * log2(e), by which the logits are multiplied, has to be a normal number."""
    mx = api.KVMX(FAKE, FAKE, FAKE, FAKE, 64 * 64, 64 * 4, 1 << 20, 64, 1, 32, 2048, FAKE, 8, 1, 128)
    st = api.lib().conduit_attn_mx(ctypes.byref(mx), FAKE, api.BF16, FAKE, 3, scale, FAKE, None, FAKE, 1 << 30, None)
    assert st == api.ERR_INVALID_ARG and "scale" in api.lib().conduit_last_error().decode()
