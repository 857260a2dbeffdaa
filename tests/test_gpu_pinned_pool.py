"""A pool in pinned host memory is compacted within pinned memory, into device memory, and back."""
import pytest
import torch

from gpu_util import DEV
from paper_2512_11920_amd import kvc

pytestmark = pytest.mark.gpu


def _buffer(n, pinned):
    return torch.full((n,), 0xAB, dtype=torch.uint8, pin_memory=True) if pinned else torch.full((n,), 0xAB, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("blocks", [24, 300])  # by one workgroup, and by the launches for larger pools
@pytest.mark.parametrize("tiers", [(True, True), (True, False), (False, True), (True, True, True)])
def test_compaction_within_and_between_tiers(blocks, tiers):
    x = torch.randn((blocks, 4, 16, 64), generator=torch.Generator(device=DEV).manual_seed(blocks), device=DEV).half()
    codec = kvc.Codec(16, 64, 4)
    codec.alloc_pool(blocks, x.numel() * 2 + 16, DEV, host_pool=tiers[0])
    codec.compress_blocks(x)
    want, left = torch.empty_like(x), list(range(blocks))
    codec.decompress_blocks(want)
    for tier in tiers[1:]:
        gone, left = left[::2], left[1::2]
        codec.free_blocks(torch.tensor(gone, dtype=torch.int32, device=DEV))
        live = codec.stats()["payload_bytes"]
        pool, desc = _buffer(codec.pool.numel(), tier), torch.empty_like(codec.desc)
        used = torch.zeros(1, dtype=torch.int64, device=DEV)
        codec.compact_pool(pool, desc, used, torch.empty(kvc.compact_workspace(codec.pool.numel()), dtype=torch.uint8, device=DEV))
        codec.adopt_pool(pool, desc, used)
        torch.cuda.synchronize()
        assert int(used) == live and (pool[live:] == 0xAB).all() and codec.pool is pool
        ids = torch.tensor(left, dtype=torch.int32, device=DEV)
        got = torch.zeros_like(x)
        codec.decompress_blocks(got, pool_ids=ids, dst_ids=ids)
        assert codec.stats()["status"] == 0 and torch.equal(got[left].view(torch.int16), want[left].view(torch.int16))


def test_pageable_memory_is_refused():
    codec = kvc.Codec(16, 64, 4)
    codec.alloc_pool(4, 4096, DEV)
    with pytest.raises(AssertionError):
        codec.compact_pool(torch.empty(4096, dtype=torch.uint8), torch.empty_like(codec.desc), torch.zeros(1, dtype=torch.int64, device=DEV),
                           torch.empty(kvc.compact_workspace(4096), dtype=torch.uint8, device=DEV))
