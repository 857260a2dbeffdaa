"""append, copy_blocks, fork_blocks, free_blocks, compact_pool and adopt_pool, bit for bit against plain statements of them."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from gpu_util import DEV, check_pool_invariants, gpu_compress
from paper_2512_11920_amd import kvc

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _bits(x):
    return (x.cpu().numpy() if torch.is_tensor(x) else x).view(np.uint16)


@pytest.mark.parametrize("N,d,kv,new", [(16, 64, 4, 1), (16, 128, 8, 3), (1, 32, 1, 5), (7, 96, 3, 20), (32, 128, 2, 70), (8, 256, 5, 2), (16, 224, 16, 1)])
@pytest.mark.parametrize("separate,token_major", [(False, False), (True, False), (False, True)])
def test_append(N, d, kv, new, separate, token_major):
    rng = np.random.default_rng(N * d + kv)
    S, ppb, blocks, width = 9, kv if separate else 2 * kv, 60, 6 + -(-new // N)
    lens = np.array([0, 1, new, N, N + 1, 2 * N, 3 * N - 1, new + 1, 5 * N], np.int32)
    table = np.full((S, width), -1, np.int32)
    perm = rng.permutation(S * width)[:].astype(np.int32)
    blocks = S * width
    table[:] = perm.reshape(S, width)
    table[4, 0] = -1          # a block that is not there
    table[6, 2] = blocks      # and one that cannot be
    shape = (blocks, N, ppb, d) if token_major else (blocks, ppb, N, d)
    k, v = (rng.integers(0, 1 << 16, shape).astype(np.uint16).view(np.float16) for _ in range(2))
    qkv = rng.integers(0, 1 << 16, (S, new, 3 + 2 * kv, d)).astype(np.uint16).view(np.float16)
    codec = kvc.Codec(N, d, ppb)
    codec.alloc_pool(1, 4096, DEV)
    if token_major:
        codec.set_cache_layout(N * ppb * d, d, ppb * d)
    kt, vt, x = _dev(k), _dev(v), _dev(qkv)
    codec.append(kt, _dev(table), _dev(lens), x[:, :, 3:3 + kv], x[:, :, 3 + kv:], v_cache=vt if separate else None)
    kp, vp = (ref.pages_view(_bits(y), N, d, ppb, token_major) for y in (k, v))
    ref.append(kp, vp if separate else kp, 0 if separate else kv, N, table, lens, _bits(qkv)[:, :, 3:3 + kv], _bits(qkv)[:, :, 3 + kv:])
    assert np.array_equal(_bits(kt), _bits(k)) and np.array_equal(_bits(vt), _bits(v))
    hit = lens[6] - new <= 2 * N + N - 1 and lens[6] > 2 * N
    assert codec.stats()["status"] == (kvc.ST_BAD_INDEX if hit else 0)


@pytest.mark.parametrize("N,d,ppb,layers", [(16, 64, 8, 1), (16, 128, 16, 3), (5, 32, 1, 2), (24, 96, 12, 2), (1, 256, 3, 4)])
@pytest.mark.parametrize("layout", ["dense", "token_major", "padded"])
def test_copy_blocks(N, d, ppb, layers, layout):
    rng = np.random.default_rng(N + d)
    per = 11
    row, page, block = {"dense": (d, N * d, ppb * N * d), "token_major": (ppb * d, d, N * ppb * d), "padded": (d + 8, N * (d + 8) + 16, ppb * (N * (d + 8) + 16) + 32)}[layout]
    x = rng.integers(0, 1 << 16, layers * per * block).astype(np.uint16)
    codec = kvc.Codec(N, d, ppb)
    codec.alloc_pool(1, 4096, DEV)
    codec.set_cache_layout(block, page, row)
    src, dst = np.array([0, 3, 3, -1, 7, 5, per], np.int32), np.array([1, 2, 4, 6, -1, 8, 9], np.int32)
    t = _dev(x.view(np.float16))
    codec.copy_blocks(t, _dev(src), _dev(dst), layers, per)
    at = (np.arange(ppb)[:, None, None] * page + np.arange(N)[:, None] * row + np.arange(d)).reshape(-1)
    for l in range(layers):
        for s, e in zip(src, dst):
            if 0 <= s < per and 0 <= e < per:
                x[(l * per + e) * block + at] = x[(l * per + s) * block + at]
    assert np.array_equal(_bits(t), x)
    assert codec.stats()["status"] == kvc.ST_BAD_INDEX
    if layers == 1 and layout == "dense":  # all blocks there are, by default
        codec.copy_blocks(t, _dev(np.array([10], np.int32)), _dev(np.array([0], np.int32)))
        assert np.array_equal(_bits(t).reshape(per, -1)[0], x.reshape(per, -1)[10])


def _pool(rng, nb=40, N=16, d=128, ppb=4, scheme=3):
    x = (rng.standard_normal((nb, ppb, N, d)) * np.exp(0.5 * rng.standard_normal(d))).astype(np.float16)
    x[1, 0] = 0
    x[2, 1, 3, 7] = np.float16("nan")
    codec, cache = gpu_compress(x, N, d, ppb, scheme)
    return codec, cache


def _compact(codec, out_bytes=None):
    pool, desc = codec.pool, codec.desc
    out = torch.full((out_bytes or pool.numel(),), 0xAB, dtype=torch.uint8, device=DEV)
    desc_out, used = torch.full_like(desc, 0xCD), torch.full((1,), -1, dtype=torch.int64, device=DEV)
    work = torch.full((kvc.compact_workspace(pool.numel()),), 0xEE, dtype=torch.uint8, device=DEV)
    codec.compact_pool(out, desc_out, used, work)
    torch.cuda.synchronize()
    return out, desc_out, used


def _check_compact(codec, out, desc_out, used):
    want, n, moved, status = ref.compact(codec.desc_numpy(), codec.pool.cpu().numpy(), out.numel())
    assert int(used) == n
    got = desc_out.cpu().numpy().view(kvc.DESC_DTYPE)
    assert np.array_equal(got.view(np.uint8), want.view(np.uint8))
    o = out.cpu().numpy()
    assert np.array_equal(o[:n], moved) and (o[n:] == 0xAB).all()
    return status


@pytest.mark.parametrize("scheme", [0, 1, 3])
def test_fork_free_compact_decode(scheme):
    """A forked block decodes as its source does, also after the source is freed; compaction keeps what is left, once."""
    rng = np.random.default_rng(3)
    codec, cache = _pool(rng, scheme=scheme)
    before = torch.empty_like(cache)
    codec.decompress_blocks(before)
    src, dst = np.array([5, 5, 9, -1, 39], np.int32), np.array([10, 11, 12, 13, 14], np.int32)
    codec.fork_blocks(_dev(src), _dev(dst))
    codec.free_blocks(_dev(np.array([5, 0, 20, 21, 22, -1, 30], np.int32)))
    out, desc_out, used = _compact(codec)
    assert _check_compact(codec, out, desc_out, used) == 0
    want = before.clone()
    for s, e in zip(src, dst):
        if s >= 0:
            want[e] = before[s]
    kept = [b for b in range(40) if b not in (5, 0, 20, 21, 22, 30)]
    payloads = {(int(e["off"]), int(e["n16"])) for e in codec.desc_numpy() if e["mode"] != 0xFF}
    assert int(used) == 16 * sum(n for _, n in payloads)
    codec.adopt_pool(out, desc_out, used)
    st = codec.stats()
    assert st["pool_bytes_used"] == int(used) and st["status"] == 0 and st["pages_invalid"] == 6 * 4
    ids = _dev(np.array(kept, np.int32))
    got = torch.zeros_like(cache)
    codec.decompress_blocks(got, pool_ids=ids, dst_ids=ids)
    assert torch.equal(got[ids.long()].view(torch.int16), want[ids.long()].view(torch.int16))
    # the pool goes on: new blocks go behind what was kept
    codec.compress_blocks(cache, n=2, src_ids=_dev(np.array([0, 5], np.int32)), pool_ids=_dev(np.array([0, 5], np.int32)))
    codec.decompress_blocks(got, n=2, pool_ids=_dev(np.array([0, 5], np.int32)), dst_ids=_dev(np.array([0, 5], np.int32)))
    assert torch.equal(got[[0, 5]].view(torch.int16), before[[0, 5]].view(torch.int16)) and codec.stats()["status"] == 0
    assert torch.equal(got[ids.long()].view(torch.int16), want[ids.long()].view(torch.int16))


def test_fork_and_free_in_layers():
    rng = np.random.default_rng(4)
    codec, _ = _pool(rng, nb=36)
    d0 = codec.desc_numpy().reshape(3, 12, 4).copy()
    src, dst = np.array([2, 2, 7, 12, 3], np.int32), np.array([5, 6, 0, 1, -1], np.int32)
    codec.fork_blocks(_dev(src), _dev(dst), 3, 12)
    codec.free_blocks(_dev(np.array([11, -4], np.int32)), 3)  # (all blocks there are, by default)
    d0[:, [5, 6, 0]] = d0[:, [2, 2, 7]]
    d0[:, 11] = np.array((0, 0, 0, 0xFF, 0), kvc.DESC_DTYPE)
    assert np.array_equal(codec.desc_numpy().view(np.uint8), d0.reshape(-1).view(np.uint8))
    assert codec.stats()["status"] == kvc.ST_BAD_INDEX


def test_compaction_of_nothing_and_of_everything():
    rng = np.random.default_rng(5)
    codec, cache = _pool(rng)
    out, desc_out, used = _compact(codec)
    assert _check_compact(codec, out, desc_out, used) == 0 and int(used) == codec.stats()["pool_bytes_used"]
    codec.free_blocks(torch.arange(40, dtype=torch.int32, device=DEV))
    out, desc_out, used = _compact(codec)
    assert _check_compact(codec, out, desc_out, used) == 0 and int(used) == 0
    codec.adopt_pool(out, desc_out, used)
    codec.compress_blocks(cache)
    check_pool_invariants(codec.desc_numpy(), codec.stats()["pool_bytes_used"], out.numel())


def _random_table(rng, pages, units, sizes):
    desc = np.zeros(pages, kvc.DESC_DTYPE)
    desc["n16"] = rng.choice(sizes, pages)
    gaps = rng.integers(0, 3, pages) * rng.integers(0, 40, pages)
    ends = np.cumsum(desc["n16"].astype(np.int64) + gaps)
    off = np.minimum(ends - desc["n16"], units)  # what lies behind the end is corrupt
    desc["off"] = 16 * off[np.argsort(rng.random(pages))] if rng.random() < 0 else 16 * off
    perm = rng.permutation(pages)
    desc = desc[perm]
    desc["mode"] = rng.choice([0, 1, 2, 3, 4, 5, 0xFF], pages)
    desc["scale"] = rng.random(pages)
    return desc


@pytest.mark.parametrize("pages,units,sizes", [(1, 1, [1]), (3, 64, [1, 64]), (64, 4096, [63, 64, 65]), (500, 4097, [1, 2, 5]), (200, 70000, [0, 1, 128, 256, 512]),
                                               (3000, 300001, [3, 64, 100]), (2000, 4096 * 1100, [512, 500])])
@pytest.mark.parametrize("damage", [False, True])
def test_compaction_of_any_table(pages, units, sizes, damage):
    """Tables made by hand: payloads of any size anywhere, several tiles, overlapping and shared ones, corrupt descriptors."""
    rng = np.random.default_rng(pages + damage)
    desc = _random_table(rng, pages, units, sizes)
    if damage and pages > 2:
        n = max(1, pages // 10)
        desc["off"][rng.integers(0, pages, n)] += 8                      # not on a unit
        desc["off"][rng.integers(0, pages, n)] = (1 << 64) - 16          # far away
        desc["off"][rng.integers(0, pages, n)] = 16 * (units - 1)        # the last unit, mostly beyond the end
        desc["mode"][rng.integers(0, pages, n)] = 77
        i = rng.integers(0, pages, n)
        desc[i] = desc[rng.integers(0, pages, n)]                        # shared
        desc["off"][rng.integers(0, pages, n)] = 16 * (units // 3)       # overlapping
    pool = rng.integers(0, 256, 16 * units).astype(np.uint8)
    codec = kvc.Codec(16, 128, 1)
    codec.bind_pool(_dev(pool), _dev(desc.view(np.uint8)))
    for room in (16 * units, max(16, 16 * (units // 5))):
        codec.restore_pool(0)  # (clears the status)
        out, desc_out, used = _compact(codec, room)
        status = _check_compact(codec, out, desc_out, used)
        assert codec.stats()["status"] == status


def test_a_pool_of_more_than_4_gib():
    """Payloads on both sides of 2^32 bytes."""
    units = (1 << 28) + 5000
    pool = torch.zeros(16 * units, dtype=torch.uint8, device=DEV)
    desc = np.zeros(6, kvc.DESC_DTYPE)
    at = [100, (1 << 28) - 130, 1 << 28, (1 << 28) + 4999, (1 << 27) + 3, (1 << 28) + 300]
    desc["off"], desc["n16"], desc["mode"] = 16 * np.array(at, np.int64), [7, 260, 9, 1, 512, 30], 3
    rng = np.random.default_rng(6)
    parts = [rng.integers(0, 256, 16 * int(n)).astype(np.uint8) for n in desc["n16"]]
    for a, p in zip(at, parts):
        pool[16 * a:16 * a + p.size] = _dev(p)
    codec = kvc.Codec(16, 128, 1)
    codec.bind_pool(pool, _dev(desc.view(np.uint8)))
    out, desc_out, used = _compact(codec, 1 << 16)
    new = desc_out.cpu().numpy().view(kvc.DESC_DTYPE)
    # the second and third overlap: 1 << 28 lies inside the second's span, so they share its units
    held = sorted({u for a, n in zip(at, desc["n16"]) for u in range(a, a + int(n))})
    assert int(used) == 16 * len(held)
    rank = {u: i for i, u in enumerate(held)}
    assert [int(o) for o in new["off"]] == [16 * rank[a] for a in at]
    o = out.cpu().numpy()
    whole = pool.view(-1, 16)[torch.tensor(held, device=DEV)].cpu().numpy().reshape(-1)
    assert np.array_equal(o[:whole.size], whole) and (o[whole.size:] == 0xAB).all()


def test_fork_free_and_compact_replay_from_a_graph():
    rng = np.random.default_rng(7)
    codec, _ = _pool(rng)
    start = codec.desc.clone()
    src, dst, ids = (torch.zeros(3, dtype=torch.int32, device=DEV) for _ in range(3))
    out, desc_out, used = torch.empty_like(codec.pool), torch.empty_like(codec.desc), torch.zeros(1, dtype=torch.int64, device=DEV)
    work = torch.empty(kvc.compact_workspace(codec.pool.numel()), dtype=torch.uint8, device=DEV)

    def turn(stream=None):
        codec.fork_blocks(src, dst, stream=stream)
        codec.free_blocks(ids, stream=stream)
        codec.compact_pool(out, desc_out, used, work, stream=stream)

    turn()
    torch.cuda.synchronize()
    cap, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(cap):
        graph.capture_begin()
        turn(cap)
        graph.capture_end()
    for rep in range(4):
        codec.desc.copy_(start)
        pick = rng.permutation(40)[:9].astype(np.int32)
        src.copy_(_dev(pick[:3]))
        dst.copy_(_dev(pick[3:6]))
        ids.copy_(_dev(pick[6:]))
        out.fill_(0xAB)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        d = start.cpu().numpy().view(kvc.DESC_DTYPE).reshape(40, 4).copy()
        d[pick[3:6]] = d[pick[:3]]
        d[pick[6:]] = np.array((0, 0, 0, 0xFF, 0), kvc.DESC_DTYPE)
        assert np.array_equal(codec.desc_numpy().view(np.uint8), d.reshape(-1).view(np.uint8))
        assert _check_compact(codec, out, desc_out, used) == 0


def test_refusals():
    codec = kvc.Codec(16, 64, 4)
    ids, used = torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    byte = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)  # noqa: E731
    for call in (lambda: codec.fork_blocks(ids, ids), lambda: codec.free_blocks(ids), lambda: codec.compact_pool(byte(4096), byte(0), used, byte(4096))):
        with pytest.raises(kvc.KvcError) as e:
            call()
        assert e.value.code == kvc.ERR_NOT_BOUND
    codec.alloc_pool(3, 8192, DEV)
    cache = torch.zeros((6, 4, 16, 64), dtype=torch.float16, device=DEV)
    kv = torch.zeros((2, 1, 2, 64), dtype=torch.float16, device=DEV)
    table, lens = torch.zeros((2, 3), dtype=torch.int32, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV)
    codec.append(cache, table, lens, kv, kv)
    for bad in ((cache.float(), table, lens, kv, kv), (cache, table[:1], lens, kv, kv), (cache, table, lens[:1], kv, kv), (cache, table, lens, kv, kv[:, :, :1]),
                (cache, table, lens, kv[:, :, :1], kv[:, :, :1]), (cache, table, lens, kv[..., :32], kv[..., :32]), (cache, table, lens, kv.float(), kv),
                (cache, table, lens, kv[0], kv[0]), (cache, table.long(), lens, kv, kv), (cache, table, lens, kv.transpose(2, 3), kv.transpose(2, 3))):
        with pytest.raises(AssertionError):
            codec.append(*bad)
    odd = torch.zeros((2, 1, 2, 68), dtype=torch.float16, device=DEV)[..., :64]
    with pytest.raises(kvc.KvcError):
        codec.append(cache, table, lens, odd, kv)
    with pytest.raises(AssertionError):
        codec.append(cache, table, lens, kv, kv, v_cache=cache)  # four heads each then
    with pytest.raises(AssertionError):
        codec.copy_blocks(cache, ids, ids[:1])
    with pytest.raises(AssertionError):
        codec.copy_blocks(cache, ids.long(), ids)
    with pytest.raises(AssertionError):
        codec.copy_blocks(cache, ids, ids, 0)
    for bad in (dict(n_layers=2, blocks_per_layer=4), dict(n_layers=70000, blocks_per_layer=0), dict(blocks_per_layer=-1)):
        with pytest.raises(kvc.KvcError):
            codec.copy_blocks(cache, ids, ids, **bad)
    with pytest.raises(AssertionError):
        codec.fork_blocks(ids, ids[:1])
    with pytest.raises(AssertionError):
        codec.fork_blocks(None, ids)
    with pytest.raises(kvc.KvcError):
        codec.free_blocks(ids, 2, 2)  # three blocks are bound
    need = kvc.compact_workspace(8192)
    good = dict(pool_out=byte(8192), desc_out=byte(16 * 12), used_out=used, work=byte(need))
    codec.compact_pool(**good)
    for bad in (dict(desc_out=byte(16 * 11)), dict(used_out=used.int()), dict(pool_out=byte(8192).float())):
        with pytest.raises(AssertionError):
            codec.compact_pool(**{**good, **bad})
    for bad in (dict(work=byte(need - 1)), dict(pool_out=byte(8190)[:8184]), dict(pool_out=codec.pool), dict(desc_out=codec.desc), dict(pool_out=byte(0))):
        with pytest.raises(kvc.KvcError):
            codec.compact_pool(**{**good, **bad})
    with pytest.raises(AssertionError):
        codec.adopt_pool(good["pool_out"], good["desc_out"], used.cpu())
