"""Forked sequences over a cache in 4 bits: the blocks that an eviction writes are copied as bytes, as copy_blocks copies FP16 blocks, and the parent keeps what it has."""
import numpy as np
import pytest
import torch

import fp4_reference as ref
import wide_reference as wide
from gpu_util import DEV
from paper_2512_11920_amd import kvc
from wide_reference import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,keep", [(16, 40), (5, 33)])
def test_a_fork_is_evicted_and_its_parent_is_not(N, keep):
    d, kv, heads, n = 64, 2, 6, 75
    rng = np.random.default_rng(N)
    codec = kvc.Codec(N, d, 2 * kv)
    codec.alloc_pool(1, 4096, DEV)
    each, shared = -(-n // N), -(-keep // N)  # blocks of the sequence; those that hold slots below the budget
    cache = torch.zeros((each + shared + 2, codec.fp4_block_bytes), dtype=torch.uint8, device=DEV)
    ids = rng.permutation(len(cache)).astype(np.int32)
    parent = ids[:each]
    child = np.concatenate([ids[each:each + shared], parent[shared:]])  # (blocks behind the budget are read alone, and stay shared)
    table, lens = dev(np.stack([parent, child])), dev(np.array([n, n], np.int32))
    x = dev(rng.standard_normal((1, n, 2 * kv, d)).astype(np.float16))
    codec.append_fp4(cache, table[:1], lens[:1], x[:, :, :kv], x[:, :, kv:])
    before = cache.clone()
    src, dst = dev(parent[:shared]), dev(child[:shared])
    with pytest.raises(AssertionError):
        codec.copy_blocks(cache, src, dst)  # (FP16 caches alone)
    cache[dst] = cache[src]
    assert torch.equal(cache[dst], before[src])

    slots = each * N
    weights = rng.random((1, kv, slots)).astype(np.float32)
    positions = np.broadcast_to(np.arange(slots, dtype=np.int32), weights.shape).copy()
    w, p = dev(weights), dev(positions)
    codec.evict(cache, table[1:], lens[1:], dev(np.array([keep], np.int32)), 7, w, p, dev(np.array([n], np.int32)), lens[1:], torch.empty(kvc.evict_workspace(1, kv, slots), dtype=torch.uint8, device=DEV))
    assert lens.tolist() == [n, keep] and codec.stats()["status"] == 0
    assert torch.equal(cache[dev(parent)], before[dev(parent)])
    # both are attended over: the parent's tokens, and the fork's that stayed, each head its own
    q = dev(rng.standard_normal((2, 1, heads, d)).astype(np.float16))
    out = torch.empty((2, 1, heads, d), dtype=torch.float16, device=DEV)
    codec.attend_fp4(out, q, cache, table, lens, torch.empty(kvc.attend_fp4_workspace(2, 1, heads, kv, d), dtype=torch.uint8, device=DEV))
    rows = ref.values(*ref.pack(x.cpu().numpy()))[0]  # [token][head][d]
    kept = p.cpu().numpy()[0, :, :keep]
    for s, tokens in enumerate(([np.arange(n)] * kv, kept)):
        for h in range(kv):
            assert sorted(tokens[h]) == ref.stays(weights[0, h], positions[0, h], n, n, n if s == 0 else keep, 7)
            k, v = rows[tokens[h], h], rows[tokens[h], kv + h]
            # a cache of this head's tokens alone, in 64 bits
            pages = np.stack([k, v], 0)[None]
            want, _, bound, _ = wide_attend(q[s:s + 1, :, h * 3:h * 3 + 3], pages, len(k), d)
            assert ((out[s:s + 1, :, h * 3:h * 3 + 3].double() - want).abs() <= bound).all()


def wide_attend(q, pages, n, d):
    at = wide.Pages(pages.astype(np.float16), n, d, 2)
    return wide.attend(q, at, at, 1, 1, np.zeros((1, 1), np.int32), np.array([n], np.int32), d ** -0.5)
