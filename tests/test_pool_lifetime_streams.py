"""adopt_pool takes a stream as the other calls take it: anything whose cuda_stream names one, as a number or as one of ctypes' pointers."""
import ctypes
import types

import pytest
import torch

from paper_2512_11920_amd import kvc


@pytest.mark.gpu
@pytest.mark.parametrize("pinned", [False, True])
def test_streams_of_other_kinds(pinned):
    dev = "cuda:0"
    side = torch.cuda.Stream()
    for named in (side.cuda_stream, ctypes.c_void_p(side.cuda_stream), 0, None, ctypes.c_void_p(None)):
        x = torch.randn((8, 4, 16, 64), device=dev).half()
        codec = kvc.Codec(16, 64, 4)
        codec.alloc_pool(8, x.numel() * 2, dev, host_pool=pinned)
        codec.compress_blocks(x)
        want, got = torch.empty_like(x), torch.empty_like(x)
        codec.decompress_blocks(want)
        pool = torch.empty(codec.pool.shape, dtype=torch.uint8, pin_memory=True) if pinned else torch.empty_like(codec.pool)
        desc, used = torch.empty_like(codec.desc), torch.zeros(1, dtype=torch.int64, device=dev)
        work = torch.empty(kvc.compact_workspace(pool.numel()), dtype=torch.uint8, device=dev)
        torch.cuda.synchronize()
        stream = types.SimpleNamespace(cuda_stream=named)
        codec.compact_pool(pool, desc, used, work, stream=stream)
        codec.adopt_pool(pool, desc, used, stream=stream)
        assert codec.pool is pool and codec.desc is desc
        torch.cuda.synchronize()
        codec.decompress_blocks(got)
        assert codec.stats()["pool_bytes_used"] == int(used) and torch.equal(got.view(torch.int16), want.view(torch.int16))
