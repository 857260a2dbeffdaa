"""append_fp4, unpack_fp4 and evict on both sides of the sizes from which they take other kernels, or go round a loop again: bit for bit against fp4_reference and wide_reference."""
import numpy as np
import pytest
import torch

import fp4_reference as ref
import wide_reference as wide
from gpu_util import DEV
from paper_2512_11920_amd import kvc
from wide_reference import dev

pytestmark = pytest.mark.gpu


def _codec(N, d, ppb):
    c = kvc.Codec(N, d, ppb)
    c.alloc_pool(1, 4096, DEV)
    return c


# sequences, new tokens: 2,047 and 2,048 of a call; so many that 0 to 3 of a sequence are over; one of each
@pytest.mark.parametrize("S,new", [(23, 89), (32, 64), (3, 701), (3, 702), (3, 703), (3, 704), (1, 2049), (2100, 1), (1025, 2)])
@pytest.mark.parametrize("N,d,kv,separate", [(16, 64, 2, False), (5, 32, 3, True)])
def test_append_of_many_tokens(S, new, N, d, kv, separate):
    rng = np.random.default_rng(S * new + N)
    ppb, width = kv if separate else 2 * kv, -(-(new + 40) // N)
    lens = (new + rng.integers(0, 40, S)).astype(np.int32)
    lens[0] = new - 1  # (its first token has no place)
    blocks = S * width
    table = rng.permutation(blocks).astype(np.int32).reshape(S, width)
    table[rng.random(table.shape) < 0.05] = -1
    s = S - 1
    table[s, (int(lens[s]) - 1) // N] = blocks  # (its last block cannot be)
    codec = _codec(N, d, ppb)
    k, v = (rng.integers(0, 256, (blocks, codec.fp4_block_bytes), dtype=np.uint8) for _ in range(2))
    x = (rng.standard_normal((S, new, 1 + 2 * kv, d), dtype=np.float32) * 2.0 ** rng.integers(-20, 12, (S, new, 1 + 2 * kv, 1))).astype(np.float16)
    x[rng.random((S, new, 1 + 2 * kv)) < 0.02] = np.nan
    kt, vt, xt = dev(k), dev(v), dev(x)
    codec.append_fp4(kt, dev(table), dev(lens), xt[:, :, 1:1 + kv], xt[:, :, 1 + kv:], v_cache=vt if separate else None)
    ref.append(k, ppb, 0, N, table, lens, x[:, :, 1:1 + kv])
    ref.append(v if separate else k, ppb, 0 if separate else kv, N, table, lens, x[:, :, 1 + kv:])
    assert np.array_equal(kt.cpu().numpy(), k) and np.array_equal(vt.cpu().numpy(), v)
    assert codec.stats()["status"] == kvc.ST_BAD_INDEX


@pytest.mark.parametrize("N,d,ppb,n", [(16, 128, 16, 512), (16, 128, 16, 513), (5, 96, 6, 6001), (128, 32, 4, 1100)])
@pytest.mark.parametrize("layout", ["dense", "token_major", "padded"])
def test_unpack_of_many_blocks(N, d, ppb, n, layout):
    """32 MB of FP16 and more; blocks twice, no block, and blocks that cannot be."""
    assert n * ppb * N * d * 2 >= 32 << 20
    rng = np.random.default_rng(n)
    row, page, block = {"dense": (d, N * d, ppb * N * d), "token_major": (ppb * d, d, N * ppb * d), "padded": (d + 8, N * (d + 8) + 16, ppb * (N * (d + 8) + 16) + 32)}[layout]
    codec = _codec(N, d, ppb)
    codec.set_cache_layout(block, page, row)
    have = n - 9
    cache = rng.integers(0, 256, (have, codec.fp4_block_bytes), dtype=np.uint8)
    codes, exps = ref.parts(cache, N, d, ppb)
    exps[:] = 101 + exps % 40
    src, dst = rng.integers(-1, have + 1, n).astype(np.int32), rng.permutation(n).astype(np.int32)
    src[:4], dst[4], dst[5] = [have, -1, 0, have - 1], -1, n
    src[4:6] = 1
    want = rng.integers(0, 1 << 16, n * block, dtype=np.uint16)
    out = dev(want.view(np.float16))
    codec.unpack_fp4(out, dev(cache), dev(src), dev(dst))
    with np.errstate(over="ignore"):
        value = ref.values(codes, exps).astype(np.float16).view(np.uint16)
    blocks = np.lib.stride_tricks.as_strided(want, (n, ppb, N, d), (2 * block, 2 * page, 2 * row, 2))
    ok = (src >= 0) & (src < have) & (dst >= 0) & (dst < n)
    blocks[dst[ok]] = value[src[ok]]
    assert np.array_equal(out.cpu().numpy().view(np.uint16), want)
    assert codec.stats()["status"] == kvc.ST_BAD_INDEX


def _evict_check(rng, N, d, kv, lens, slots, keep, recent, fp4, kind, apart):
    lens = np.array(lens, np.int32)
    width = -(-int(lens.max()) // N)
    table, blocks = wide.tables(rng, lens, N, width)
    codec = _codec(N, d, 2 * kv)
    cache = rng.integers(0, 256, (blocks, codec.fp4_block_bytes), dtype=np.uint8) if fp4 else rng.integers(0, 1 << 16, (blocks, 2 * kv, N, d), dtype=np.uint16)
    S = len(lens)
    weights = {"heavy": np.exp(4 * rng.standard_normal((S, kv, slots))), "ties": rng.integers(0, 3, (S, kv, slots)) * 0.25, "later": np.broadcast_to(np.arange(1, slots + 1), (S, kv, slots))}[kind].astype(np.float32)
    seen = lens + rng.integers(0, 50, S).astype(np.int32)
    positions = rng.permuted(np.broadcast_to(np.arange(slots, dtype=np.int32), weights.shape), axis=2) + (seen - lens)[:, None, None].astype(np.int32)
    keep = np.full(S, keep, np.int32)
    ct, wt, pt, lt = dev(cache if fp4 else cache.view(np.float16)), dev(weights), dev(positions), dev(lens)
    w_out, p_out = (torch.full_like(wt, -3.0), torch.full_like(pt, -77)) if apart else (wt, pt)
    new = torch.full_like(lt, -9)
    work = torch.full((kvc.evict_workspace(S, kv, slots),), 0xCC, dtype=torch.uint8, device=DEV)
    codec.evict(ct, dev(table), lt, dev(keep), recent, wt, pt, dev(seen), new, work, weights_out=w_out if apart else None, positions_out=p_out if apart else None)
    parts = ref.parts(cache, N, d, 2 * kv) if fp4 else [cache]
    w, p = weights.copy(), positions.copy()
    want_lens = wide.evict([x[:, a:a + kv] for x in parts for a in (0, kv)], N, table, lens, keep, recent, w, p, seen)
    assert np.array_equal(ct.cpu().numpy().view(cache.dtype), cache)
    assert np.array_equal(new.cpu().numpy(), want_lens) and codec.stats()["status"] == 0
    inside = np.broadcast_to(np.arange(slots) < want_lens[:, None, None], w.shape)
    got_w, got_p = w_out.cpu().numpy(), p_out.cpu().numpy()
    assert np.array_equal(got_w[inside], w[inside]) and np.array_equal(got_p[inside], p[inside])
    assert np.array_equal(got_w[~inside], np.full_like(w, -3.0)[~inside] if apart else weights[~inside]) and np.array_equal(got_p[~inside], np.full_like(p, -77)[~inside] if apart else positions[~inside])


@pytest.mark.parametrize("slots", [1, 2, 511, 512, 513, 1024, 1025, 2560, 2561, 4097, 4608, 4609, 8704, 8705, 16384, 16385, 16400])
@pytest.mark.parametrize("apart", [False, True])
def test_eviction_from_so_many_slots(slots, apart):
    """As many tokens as slots, one less, and few; one leaves, half, and most, which are tied."""
    rng = np.random.default_rng(slots)
    lens = [slots, max(1, slots - 1), max(1, min(slots, 7))]
    for keep, kind, recent in ((slots - 1, "heavy", 100), (slots // 2, "heavy", slots // 8), (slots // 5, "ties", 3)):
        _evict_check(rng, 16, 32, 2, lens, slots, keep, recent, apart, kind, apart)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("N,d", [(16, 32), (5, 96)])
def test_eviction_of_more_rows_than_the_workgroups_move_at_a_time(fp4, N, d):
    """2,048 workgroups, 64 moves at a time: the first half of every head leaves, so each of its slots gets a token."""
    S, kv, n, keep = 9, 8, 4400, 2200
    assert S * kv * keep > 2048 * 64
    _evict_check(np.random.default_rng(N), N, d, kv, [n] * (S - 1) + [n - 300], n, keep, 0, fp4, "later", False)


@pytest.mark.parametrize("fp4", [False, True])
def test_a_length_beyond_slots_and_table(fp4):
    """Nothing of that sequence is read or written, and the others lose their tokens."""
    rng = np.random.default_rng(1)
    N, d, kv, slots = 16, 64, 2, 95
    lens = np.array([90, 5000, 70], np.int32)
    table, blocks = wide.tables(rng, np.array([90, 90, 70]), N, 6)
    codec = _codec(N, d, 2 * kv)
    cache = rng.integers(0, 256, (blocks, codec.fp4_block_bytes), dtype=np.uint8) if fp4 else rng.integers(0, 1 << 16, (blocks, 2 * kv, N, d), dtype=np.uint16)
    weights, positions = rng.random((3, kv, slots)).astype(np.float32), rng.integers(0, 99, (3, kv, slots)).astype(np.int32)
    seen, keep = lens.copy(), np.full(3, 40, np.int32)
    ct, wt, pt, lt = dev(cache if fp4 else cache.view(np.float16)), dev(weights), dev(positions), dev(lens)
    codec.evict(ct, dev(table), lt, dev(keep), 4, wt, pt, dev(seen), lt, torch.empty(kvc.evict_workspace(3, kv, slots), dtype=torch.uint8, device=DEV))
    parts = ref.parts(cache, N, d, 2 * kv) if fp4 else [cache]
    new, status = ref.evict([x[:, a:a + kv] for x in parts for a in (0, kv)], N, table, lens, keep, 4, weights, positions, seen)
    assert status == 4 and codec.stats()["status"] == kvc.ST_BAD_INDEX
    assert new.tolist() == [40, 5000, 40] == lt.tolist()
    assert np.array_equal(ct.cpu().numpy().view(cache.dtype), cache) and np.array_equal(wt.cpu().numpy(), weights) and np.array_equal(pt.cpu().numpy(), positions)
