"""The statements for large calls (wide_reference) against the ones for small calls (paged_reference, fp4_reference)."""
import numpy as np
import pytest
import torch

import fp4_reference as ref
import paged_reference as paged
import wide_reference as wide

LENS = np.array([0, 70, 3, 33, 129], np.int32)


@pytest.fixture(autouse=True)
def _on_the_cpu(monkeypatch):
    monkeypatch.setattr(wide, "DEV", "cpu")


def _case(fp4, N=5, d=32, kv=2, group=3, nq=4):
    rng = np.random.default_rng(fp4)
    table, blocks = wide.tables(rng, LENS, N, 27)
    cache = (wide.cache_fp4 if fp4 else wide.cache_fp16)(rng, table, LENS, N, d, 2 * kv, blocks)
    table[1, 3], table[4, 2] = -1, blocks
    with np.errstate(invalid="ignore"):
        pages = ref.values(*ref.parts(cache, N, d, 2 * kv)) if fp4 else cache.astype(np.float64)
    return rng, table, cache, pages, rng.standard_normal((len(LENS), nq, kv * group, d)).astype(np.float16)


@pytest.mark.parametrize("fp4", [False, True])
def test_attention(fp4):
    _, table, cache, pages, q = _case(fp4)
    at = wide.Pages(cache, 5, 32, 4)
    got = wide.attend(torch.from_numpy(q), at, at, 2, 2, table, LENS, 0.3)
    want = paged.attend(q, pages, pages, 2, 2, 5, table, LENS, 0.3)
    # (sums of 64 bits in another order: a score is off by 32 * 2^-53 * 0.3 * sum |q k|, the sum below 32 * 4 * 4, which is 6e-13 on either side, and so is its weight; values are below 4)
    for g, w in zip(got, want):
        assert np.allclose(g.numpy(), w, rtol=1e-11, atol=1e-11)


@pytest.mark.parametrize("fp4", [False, True])
def test_weights(fp4):
    rng, table, cache, pages, q = _case(fp4)
    lse = (np.log(np.maximum(LENS, 1))[:, None, None] + rng.uniform(0, 3, q.shape[:3])).astype(np.float32)
    lse[1, 2, 1] = -np.inf
    weights, positions = rng.random((len(LENS), 2, 130)).astype(np.float32), rng.integers(0, 99, (len(LENS), 2, 130)).astype(np.int32)
    seen = LENS + 7
    got = wide.weigh(weights, positions, seen, torch.from_numpy(q), wide.Pages(cache, 5, 32, 4), 2, table, LENS, torch.from_numpy(lse), -0.2)
    want = ref.weigh(weights, positions, seen, q, pages, 2, 5, table, LENS, lse, -0.2)
    inside = np.broadcast_to(np.arange(130) < LENS[:, None, None], weights.shape)
    for g, w in zip(got, want):
        assert np.allclose(g[inside], w[inside], rtol=1e-11, atol=1e-300)
    assert np.array_equal(got[1], want[1])


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("keep,recent", [(0, 0), (40, 9), (60, 100), (500, 2)])
def test_eviction(kind, keep, recent):
    rng, table, cache, _, _ = _case(False)
    table[1, 3], table[4, 2] = 0, 1
    weights = rng.integers(0, 4, (len(LENS), 2, 130)).astype(np.float32) if kind else rng.random((len(LENS), 2, 130)).astype(np.float32)
    weights[rng.random(weights.shape) < 0.1] = np.nan
    positions, seen = rng.permuted(np.broadcast_to(np.arange(130, dtype=np.int32), weights.shape), axis=2), LENS + 3
    results = []
    for f in (wide.evict, lambda *a: ref.evict(*a)[0]):
        rows, w, p = cache.copy().view(np.uint16), weights.copy(), positions.copy()
        results.append((f([rows[:, :2], rows[:, 2:]], 5, table, LENS, np.full(len(LENS), keep), recent, w, p, seen), rows, w.view(np.uint32), p))
    for a, b in zip(*results):
        assert np.array_equal(a, b)
