"""NaN and infinite scores in kvc_attend: what the formula makes of them comes out, whichever kernels a call takes and however its work
is divided.  Tolerances are the reference's own bound (paged_reference.attend); where it is NaN the output has to be."""
import numpy as np
import pytest

import paged_reference as ref
from test_gpu_attend import _run, _setup, _want, _wider

import torch  # noqa: F401  (before the library, which shares its runtime)

pytestmark = pytest.mark.gpu

#: (head dimension, heads of K and V, query heads each, queries, lengths, prefixes, groups, tokens that the own and the prefix table have room for).
#: By which kernels: a workgroup for every unit; waves with units of their own; units that many waves share, joined by one and by several threads a row;
#: with prefixes, both parts in one launch, apart and divided; and in launches of their own.
WAYS = {
    "direct": (64, 2, 2, 3, [1, 31, 33, 64, 65, 257, 300, 450], (), (0,), 0, 0),
    "direct_two_tiles": (96, 1, 8, 4, [5, 32, 97, 200, 500], (), (0,), 0, 0),
    "alone": (64, 2, 2, 2, [1, 2, 20, 31, 32], (), (0,), 2000, 0),
    "shared": (128, 2, 4, 2, [3000, 33, 64, 700, 1], (), (0,), 0, 0),
    "shared_two_tiles": (128, 1, 8, 4, [2000, 33, 65], (), (0,), 0, 0),
    "shared_wide": (256, 1, 2, 2, [1500, 40, 65], (), (0,), 0, 0),
    "one_thread_a_row": (128, 8, 8, 1, [40, 700, 33] * 22, (), (0,), 0, 0),
    "prefix": (128, 2, 4, 1, [5, 31, 33, 64, 700, 0], (333, 700), (0, 2, 5), 0, 0),
    "prefix_divided": (64, 2, 4, 2, [5, 31, 33, 64, 700, 0], (333, 1500), (0, 2, 5), 0, 900000),
    "prefix_by_itself": (160, 2, 4, 1, [5, 31, 33, 64, 700, 0], (333, 700), (0, 2, 5), 0, 0),
}


def _case(way, seed, q_scale=1.0):
    d, kv, group, q, lens, prefix, first, room, proom = WAYS[way]
    c = _setup(np.random.default_rng([seed, d, len(lens)]), 16, d, kv, group, q, lens, prefix=prefix, first=first, q_scale=q_scale)
    if room:
        c["table"] = _wider(c["table"], room // 16)
    if proom:
        c["prefix_table"] = _wider(c["prefix_table"], proom // 16)
    return c


def _row(c, s, t):
    """Where key and value rows of token t of sequence s are; s < 0: of prefix -1 - s."""
    return (c["table"][s] if s >= 0 else c["prefix_table"][-1 - s])[t // c["N"]], t % c["N"]


def _check(c, out, lse, rows=slice(None)):
    """out and lse of the sequences `rows` against the formula.  Tokens whose score is -infinity have weight zero exactly: the bound is that of the other
    tokens (what rounding does to -infinity has no number)."""
    with np.errstate(invalid="ignore"):
        want, wl, _, _ = _want(c)
        with pytest.MonkeyPatch.context() as m:
            m.setattr(ref, "tokens_of", lambda *a, all_of=ref.tokens_of: (lambda t, k, v, keep: (t[keep], k[keep], v[keep]))(*(x := all_of(*a)), ~np.isneginf(x[1]).any(1)))
            _, _, bound, lb = _want(c)
        out, lse, want, wl, bound, lb = (x[rows] for x in (out, lse, want, wl, bound, lb))
        bad = np.argwhere(np.isnan(out) != np.isnan(want))
        assert not len(bad), ("NaN", len(bad), bad[:5])
        assert (np.isnan(lse) == np.isnan(wl)).all(), np.argwhere(np.isnan(lse) != np.isnan(wl))[:5]
        fine = np.isfinite(want)
        assert np.array_equal(out[~fine], want[~fine], equal_nan=True)
        assert (np.abs(out - want)[fine] <= bound[fine]).all()
        assert np.array_equal(lse[~np.isfinite(wl)], wl[~np.isfinite(wl)], equal_nan=True)
        seen = np.isfinite(wl)
        assert (np.abs(lse - wl)[seen] <= lb[seen]).all()
    return want


@pytest.mark.parametrize("way", WAYS)
def test_a_query_with_a_nan(way):
    """All its scores are NaN, and so are its output and its sum; a query that sees no token has neither scores nor NaN."""
    c = _case(way, 1)
    rng = np.random.default_rng(2)
    S, q = c["qkv"].shape[:2]
    for s in range(S):
        c["qkv"][s, rng.integers(0, q), rng.integers(0, c["heads"]), rng.integers(0, c["d"])] = np.nan
    c["lens"][-1] = 0 if len(c["lens"]) > 5 else c["lens"][-1]
    _, out, lse = _run(c)
    want = _check(c, out, lse)
    assert np.isnan(want).any() and np.isfinite(want).any()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("where", ["last", "first", "tile", "all"])
def test_keys_that_are_nan(way, where):
    """One token (alone in the last tile of some sequences), a whole tile, whole sequences and whole prefixes."""
    c = _case(way, 3)
    rows = [(s, int(n)) for s, n in enumerate(c["lens"])] + [(-1 - g, int(n)) for g, n in enumerate(c["prefix_lens"])]
    for i, (s, n) in enumerate(rows):
        if i % 2 and len(rows) > 3 or n == 0:
            continue
        for t in {"last": [n - 1], "first": [0], "tile": range((n - 1) // 32 * 32, n), "all": range(n)}[where]:
            b, r = _row(c, s, t)
            c["k"][b, :c["kv"], r, 3 if where != "all" else slice(None)] = np.nan
    _, out, lse = _run(c)
    want = _check(c, out, lse)
    assert np.isnan(want).any()


@pytest.mark.parametrize("way", WAYS)
def test_infinite_keys_among_the_last_tokens(way):
    """They reach the queries that see them and no others: a score that is +infinity makes the row NaN, one that is -infinity has no weight."""
    c = _case(way, 4)
    q = c["qkv"].shape[1]
    c["qkv"][:, :, :, 0] = np.abs(c["qkv"][:, :, :, 0]) + np.float16(0.1)
    for s, n in enumerate(c["lens"]):
        for back in range(1, min(q, int(n)) + 1):
            b, r = _row(c, s, int(n) - back)
            c["k"][b, :c["kv"], r, 0] = [np.inf, -np.inf, np.nan][(s + back) % 3]
    # (a row whose only tokens have no weight is the next test's)
    _, out, lse = _run(c)
    want = _check(c, out, lse, [s for s, n in enumerate(c["lens"]) if n > q])
    assert np.isnan(want).any() and np.isfinite(want).any()


@pytest.mark.parametrize("way", WAYS)
def test_infinite_values_of_tokens_without_weight(way):
    """Whole tiles have scores of -infinity, weight zero, and one of their values is infinite: zero times infinity, also where a piece of the work has no other token.
    (NaN as a rule; in the tile in which the last queries' views end, infinite.)"""
    c = _case(way, 5)
    kv = c["kv"]
    c["qkv"][:, :, :, 0] = np.abs(c["qkv"][:, :, :, 0]) + np.float16(0.1)
    hit = 0
    for s, n in enumerate(c["lens"]):
        if n < 65:
            continue
        for t in range((int(n) // 32 - 1) * 32, int(n) // 32 * 32 - 8):
            b, r = _row(c, s, t)
            c["k"][b, :kv, r, 0] = -np.inf
            if t % 32 == 5:
                c["k"][b, kv:, r, 7] = np.inf
                hit += 1
    _, out, lse = _run(c)
    with np.errstate(invalid="ignore"):
        nan = np.isnan(_want(c)[0])
    for s, n in enumerate(c["lens"]):
        if c["qkv"].shape[1] > 1 and int(n) // 32 * 32 + c["qkv"].shape[1] - 1 > n:  # (the tile with those values is that one)
            assert not np.isfinite(out[s][nan[s]]).any()
            out[s][nan[s]] = np.nan
    want = _check(c, out, lse)
    assert np.isnan(want).any() == (hit > 0)


@pytest.mark.parametrize("way", WAYS)
def test_rows_of_scores_of_minus_infinity(way):
    """No token of theirs has any weight: out = 0 and lse = -infinity, as where there is no token."""
    c = _case(way, 6)
    kv = c["kv"]
    c["qkv"][:, :, :, 0] = np.abs(c["qkv"][:, :, :, 0]) + np.float16(0.1)
    for s, n in enumerate(c["lens"]):
        for t in range(int(n)):
            b, r = _row(c, s, t)
            c["k"][b, :kv, r, 0] = -np.inf
    seen = _case(way, 6)
    seen["qkv"] = c["qkv"]
    seen["lens"] = np.zeros_like(c["lens"])  # what is left: the prefixes
    _, out, lse = _run(c)
    want, wl, bound, lb = _want(seen)
    assert np.isfinite(out).all() and (np.abs(out - want) <= bound).all()
    none = np.isneginf(wl)
    assert np.isneginf(lse[none]).all() and (out[none] == 0).all()
    assert (np.abs(lse[~none] - wl[~none]) <= lb[~none]).all()


def test_the_reference_makes_nan_of_them():
    """(What the other tests lean on.)"""
    c = _case("direct", 7)
    c["qkv"][0, :, 0] = np.nan
    with np.errstate(invalid="ignore"):
        want, wl, _, _ = ref.attend(c["qkv"][:, :, :c["heads"]], c["k"], c["k"], c["kv"], c["kv"], c["N"], c["table"], c["lens"], 1.0)
    assert np.isnan(want[0, -1, 0]).all() and np.isnan(wl[0, -1, 0]) and np.isfinite(want[1:]).all()
