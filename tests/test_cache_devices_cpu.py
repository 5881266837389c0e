"""Where a descriptor's cache lives, and how long: refusals before anything is launched,
so without a GPU (the calls' rows are CPU tensors that say they are on GPU 0)."""
import os
import weakref

import pytest
import torch

from paper_2609_05821_amd import api

pytestmark = pytest.mark.skipif(not os.path.exists(api.LIB_PATH),
                                reason="libconduit.so not built (run __graft_entry__.build())")


class OnGpu(torch.Tensor):
    def get_device(self):
        return 0


def on_gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


def pools(make):
    return [make(2, 2, 64, b, dtype=torch.uint8) for b in (64, 64, 4, 4)]


def caches(cpu):
    """Descriptors of 16-bit caches of which one tensor is on the CPU."""
    make = [torch.zeros if i == cpu else on_gpu for i in range(3)]
    paged = [m(2, 64, 2, 128, dtype=torch.bfloat16) for m in make[:2]] + [make[2](2, dtype=torch.int32)]
    out = [api.kv_desc_paged(*paged, 128, 4)]
    if cpu < 2:
        out.append(api.kv_desc(*(m(128, 2, 128, dtype=torch.bfloat16) for m in make[:2]), 4))
    return out


@pytest.mark.parametrize("cpu", [0, 1, 2], ids=["k", "v", "block_table"])
def test_a_cache_on_another_device_is_refused(cpu):
    x, pos = on_gpu(3, 2, 128), on_gpu(3, dtype=torch.int32)
    for kv in caches(cpu):
        with pytest.raises(api.ConduitError, match="different devices"):
            api.conduit_append_kv(kv, pos, x, x)
        with pytest.raises(api.ConduitError, match="different devices"):
            api.conduit_load_mx(api.mx_desc(*pools(on_gpu), 4), pos, kv, pos)


def test_a_cpu_cache_with_cpu_rows_is_refused():
    x, pos = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    kv = api.kv_desc(torch.zeros(64, 2, 128, dtype=torch.bfloat16), torch.zeros(64, 2, 128, dtype=torch.bfloat16), 4)
    with pytest.raises(api.ConduitError, match="on the GPU"):
        api.conduit_append_kv(kv, pos, x, x)


def test_descriptors_keep_their_tensors():
    k, v = (torch.zeros(2, 64, 2, 128, dtype=torch.bfloat16) for _ in range(2))
    table = torch.zeros(2, dtype=torch.int32)
    flat = [torch.zeros(64, 2, 128, dtype=torch.bfloat16) for _ in range(2)]
    refs = [weakref.ref(t) for t in (k, v, table, *flat)]
    paged, dense = api.kv_desc_paged(k, v, table, 128, 4), api.kv_desc(*flat, 4)
    del k, v, table, flat
    assert all(r() is not None for r in refs)
    del paged, dense
    assert all(r() is None for r in refs)
