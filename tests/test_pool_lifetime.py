"""Buffers that adopt_pool replaces stay theirs until what was enqueued has read them: the codec often holds the last reference, and the allocator
would hand the memory out again while a compaction on another stream still reads it."""
import types

import pytest
import torch

from paper_2512_11920_amd import kvc


class _Memory:
    """What adopt_pool looks at of a tensor, and the streams that its memory is kept for."""

    def __init__(self, pinned=False):
        self.is_cuda, self.pinned, self.streams = not pinned, pinned, []

    def is_pinned(self):
        return self.pinned

    def is_contiguous(self):
        return True

    def element_size(self):
        return 1

    def numel(self):
        return 64

    def data_ptr(self):
        return 4096

    def record_stream(self, stream):
        assert self.is_cuda, "host memory is not kept that way"
        self.streams.append(stream)


class _Event:
    passed = False

    def __init__(self, stream=None):
        self.stream, self.waited = stream, False

    def query(self):
        return self.passed

    def synchronize(self):
        self.waited = True


@pytest.fixture
def codec(monkeypatch):
    kvc.load()
    c = kvc.Codec.__new__(kvc.Codec)
    c._L, c._ctx = types.SimpleNamespace(kvc_adopt_pool=lambda *a: 0, kvc_destroy=lambda *a: 0), None
    c._leaving = []
    c.pool, c.desc = _Memory(), _Memory()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0, record_event=lambda: _Event("current")))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return c


def _adopt(c, pool, stream):
    used = _Memory()
    used.element_size, used.numel = lambda: 8, lambda: 1
    c.adopt_pool(pool, _Memory(), used, stream=stream)


def _stream(name):
    return types.SimpleNamespace(cuda_stream=7, record_event=lambda: _Event(name))


def test_old_buffers_are_kept_for_the_stream_of_the_call(codec):
    pool, desc, stream = codec.pool, codec.desc, _stream("side")
    _adopt(codec, _Memory(), stream)
    assert pool.streams == [stream] and desc.streams == [stream]
    assert codec.pool.streams == [] and codec.pool is not pool


def test_without_a_stream_they_are_kept_for_the_current_one(codec):
    pool = codec.pool
    _adopt(codec, _Memory(), None)
    assert len(pool.streams) == 1 and pool.streams[0] is not None


def test_pinned_pools_are_held_until_the_stream_has_passed(codec):
    old = codec.pool = _Memory(pinned=True)
    _adopt(codec, _Memory(), _stream("side"))
    assert [x[1] for x in codec._leaving] == [old] and codec._leaving[0][0].stream == "side"
    _adopt(codec, _Memory(), _stream("side"))
    assert [x[1] for x in codec._leaving] == [old], "its event has not passed"
    codec._leaving[0][0].passed = True
    _adopt(codec, _Memory(), _stream("side"))
    assert codec._leaving == []


def test_close_waits_for_what_is_held(codec):
    codec.pool = _Memory(pinned=True)
    _adopt(codec, _Memory(), _stream("side"))
    event = codec._leaving[0][0]
    codec._ctx = types.SimpleNamespace(value=1)
    codec.close()
    assert event.waited and codec._leaving == []


def test_the_first_pool_replaces_none(codec):
    codec.pool = codec.desc = None
    _adopt(codec, _Memory(), _stream("side"))
    assert codec._leaving == []


@pytest.mark.gpu
@pytest.mark.parametrize("adopted_on", ["side", "current"])
def test_a_compaction_reads_the_old_pool_while_others_allocate(adopted_on):
    """The compaction waits behind a pause on its own stream; in the meantime the program lets go of the old buffers and fills new ones of their sizes."""
    dev, n = "cuda:0", 64
    x = torch.randn((n, 4, 16, 64), generator=torch.Generator(device=dev).manual_seed(1), device=dev).half()
    codec = kvc.Codec(16, 64, 4)
    codec.alloc_pool(n, x.numel() * 2, dev)
    codec.compress_blocks(x)
    want = torch.empty_like(x)
    codec.decompress_blocks(want)
    codec.free_blocks(torch.arange(0, n, 2, dtype=torch.int32, device=dev))
    sizes = codec.pool.numel(), codec.desc.numel()
    pool, desc, used = torch.empty_like(codec.pool), torch.empty_like(codec.desc), torch.zeros(1, dtype=torch.int64, device=dev)
    work = torch.empty(kvc.compact_workspace(pool.numel()), dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    codec.compact_pool(pool, desc, used, work, stream=side)
    if adopted_on == "current":
        torch.cuda.current_stream().wait_stream(side)
    codec.adopt_pool(pool, desc, used, stream=side if adopted_on == "side" else None)
    junk = [torch.full((k,), 0x5A, dtype=torch.uint8, device=dev) for k in sizes for _ in range(3)]
    torch.cuda.synchronize()
    odd = torch.arange(1, n, 2, dtype=torch.int32, device=dev)
    got = torch.zeros_like(x)
    codec.decompress_blocks(got, pool_ids=odd, dst_ids=odd)
    assert codec.stats()["status"] == 0 and all((j == 0x5A).all() for j in junk)
    assert torch.equal(got[1::2].view(torch.int16), want[1::2].view(torch.int16))
