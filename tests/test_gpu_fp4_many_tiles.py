"""attend_fp4 and weigh where a worker has several tiles, sequences and units, as in a serving step of many long sequences: against statements in 64 bits, within bounds that are derived there
(paged_reference, fp4_reference).  Each test asserts how many tiles a worker has."""
import numpy as np
import pytest
import torch

import fp4_reference as ref
import wide_reference as wide
from gpu_util import DEV
from paper_2512_11920_amd import kvc
from wide_reference import dev

pytestmark = pytest.mark.gpu


def _lens(rng, S, most, empty=True):
    lens = rng.integers(1, most + 1, S).astype(np.int32)
    lens[0], lens[-1] = most, 1
    if empty:
        lens[[1, S // 2]] = 0
    return lens


def _codec(N, d, ppb, token_major=False):
    c = kvc.Codec(N, d, ppb)
    c.alloc_pool(1, 4096, DEV)
    if token_major:
        c.set_cache_layout(N * ppb * d, d, ppb * d)
    return c


# ------------------------------------------------------------------------------------------------ attention


def _workers(S, nq, H, kv, d):
    """-> units (KV heads and their tiles of rows), ranges of the sequences' tiles that workers of a unit share; as the workspace has room for."""
    rows = H // kv * nq
    of_tile = 16 if rows <= 16 or d > 192 else 32
    units = kv * -(-rows // of_tile)
    wide_rows = d * of_tile // 16
    ranges = max(1, (3 if wide_rows <= 32 else 2 if wide_rows <= 128 else 1) * 1024 // units)
    slots = S * nq * H + (2 * ranges * units * of_tile if ranges > 1 else 0)
    round_256 = lambda n: -(-n // 256) * 256
    assert kvc.attend_fp4_workspace(S, nq, H, kv, d) == round_256(4 * S + 4) + round_256(8) + round_256(8 * slots) + 4 * d * slots
    return units, ranges


def _attend_case(seed, N, d, kv, group, nq, lens, holes=False, separate=False):
    rng = np.random.default_rng(seed)
    lens = np.array(lens, np.int32)
    table, blocks = wide.tables(rng, lens, N, -(-int(lens.max()) // N) + 1)
    ppb = kv if separate else 2 * kv
    caches = [wide.cache_fp4(rng, table, lens, N, d, ppb, blocks) for _ in range(1 + separate)]
    if holes:
        table[rng.random(table.shape) < 0.1] = -1
    return dict(N=N, d=d, kv=kv, ppb=ppb, lens=lens, table=table, caches=caches, q=rng.standard_normal((len(lens), nq, kv * group, d), dtype=np.float32).astype(np.float16), separate=separate)


def _run(c, dirty=0xFF):
    codec = _codec(c["N"], c["d"], c["ppb"])
    S, nq, H, d = c["q"].shape
    q = dev(np.concatenate([c["q"], np.full((S, nq, 2, d), np.nan, np.float16)], 2))
    out, lse = torch.full((S, nq, H + 1, d), 7.0, dtype=torch.float16, device=DEV), torch.full((S, nq, H), 5.0, device=DEV)
    work = torch.full((kvc.attend_fp4_workspace(S, nq, H, c["kv"], d),), dirty, dtype=torch.uint8, device=DEV)
    caches = [dev(x) for x in c["caches"]]
    codec.attend_fp4(out[:, :, :H], q[:, :, :H], caches[0], dev(c["table"]), dev(c["lens"]), work, v_cache=caches[1] if c["separate"] else None, lse=lse)
    torch.cuda.synchronize()
    assert codec.stats()["status"] == 0 and (out[:, :, H] == 7).all()
    return out[:, :, :H], lse


def _check(c):
    out, lse = _run(c)
    k = wide.Pages(c["caches"][0], c["N"], c["d"], c["ppb"])
    v = wide.Pages(c["caches"][1], c["N"], c["d"], c["ppb"]) if c["separate"] else k
    want, want_lse, bound, lse_bound = wide.attend(dev(c["q"]), k, v, 0 if c["separate"] else c["kv"], c["kv"], c["table"], c["lens"], c["d"] ** -0.5)
    off = (out.double() - want).abs()
    assert torch.isfinite(out).all() and (off <= bound).all(), float((off / bound.clamp_min(1e-30)).nan_to_num(9e9).max())
    seen = torch.isfinite(want_lse)
    assert torch.equal(torch.isneginf(lse), ~seen) and (out[~seen] == 0).all()
    assert ((lse.double() - want_lse).abs()[seen] <= lse_bound[seen]).all()


def _share(c):
    """Units, ranges, and tiles of a range; divided calls alone."""
    S, nq, H, d = c["q"].shape
    units, ranges = _workers(S, nq, H, c["kv"], d)
    assert units * S > 512 or c["table"].shape[1] * c["N"] > 8192
    tiles = -(-c["lens"].astype(np.int64) // 32)
    return units, ranges, -(-int(tiles.sum()) // ranges), tiles


# N, d, KV heads, heads of a group, queries, sequences, longest
MANY = [(16, 32, 64, 1, 1, 14, 2500), (5, 32, 64, 1, 1, 14, 2500), (8, 64, 40, 2, 3, 18, 1500), (16, 128, 32, 8, 1, 24, 1400), (7, 128, 32, 5, 3, 24, 1400), (16, 96, 24, 1, 1, 30, 1700),
        (16, 128, 8, 8, 5, 40, 1100), (5, 128, 8, 8, 5, 40, 1100), (24, 96, 24, 1, 40, 15, 900), (3, 64, 10, 7, 6, 40, 1000), (7, 192, 16, 5, 8, 20, 1000), (16, 160, 12, 6, 3, 45, 1500),
        (16, 256, 32, 4, 12, 7, 900), (9, 224, 20, 3, 2, 30, 1100), (16, 32, 30, 4, 9, 20, 900)]


@pytest.mark.parametrize("N,d,kv,group,nq,S,most", MANY)
@pytest.mark.parametrize("holes", [False, True])
def test_attention_by_workers_of_many_tiles(N, d, kv, group, nq, S, most, holes):
    rng = np.random.default_rng(N * d + kv)
    c = _attend_case(d + N, N, d, kv, group, nq, _lens(rng, S, most), holes=holes, separate=holes)
    units, ranges, share, tiles = _share(c)
    assert ranges > 1 and share >= 4 and tiles.max() > 2 * share  # (a sequence of several workers, one in the middle of it)
    begins = np.concatenate([[0], np.cumsum(tiles)])
    assert any(b % share and (b + n) // share == b // share for b, n in zip(begins, tiles) if n)  # (and one that a worker has whole, behind another's)
    _check(c)


def test_attention_over_many_short_sequences():
    """More sequences than threads add up lengths, and many of them to a worker."""
    lens = np.random.default_rng(0).integers(0, 200, 300)
    lens[40:60] = 0
    c = _attend_case(1, 16, 32, 32, 1, 1, lens)
    _, ranges, share, _ = _share(c)
    assert ranges == 96 and share >= 8
    _check(c)


@pytest.mark.parametrize("N,d,kv,group,nq,ranges", [(16, 32, 16, 8, 260, 1), (5, 32, 16, 8, 260, 1), (16, 64, 16, 8, 256, 2), (8, 96, 40, 8, 64, 1), (5, 192, 64, 8, 64, 1), (16, 128, 16, 8, 100, 2),
                                                    (16, 256, 64, 4, 70, 1)])
def test_attention_of_many_rows(N, d, kv, group, nq, ranges):
    """Chunks of prompts: many tiles of rows, and few ranges, or one, which leaves nothing to join; sequences of fewer tokens than queries among them."""
    c = _attend_case(d + nq, N, d, kv, group, nq, [0, 300, 33, 500, 64])
    assert _share(c)[1] == ranges
    _check(c)


@pytest.mark.parametrize("N,d,kv,group,nq,S,most", [(16, 128, 8, 8, 5, 40, 1100), (5, 64, 40, 2, 3, 18, 1500), (16, 32, 16, 8, 260, 5, 300)])
def test_a_value_that_is_nan_among_the_last_tokens_of_long_sequences(N, d, kv, group, nq, S, most):
    """It reaches the queries that see its token, and no other, sequence or head."""
    rng = np.random.default_rng(3)
    c = _attend_case(4, N, d, kv, group, nq, _lens(rng, S, most))
    _share(c)
    values = ref.parts(c["caches"][0], N, d, c["ppb"])[1][:, kv:]
    s = int(np.argsort(c["lens"])[-2])
    t, h = int(c["lens"][s]) - 2, kv - 1  # the last two queries see it
    before = _run(c)[0]
    values[c["table"][s, t // N], h, t % N, 0] = 255
    after = _run(c)[0]
    want = before.clone()
    want[s, nq - 2:, h * group:, :32] = torch.nan
    assert torch.isnan(after[s, nq - 2:, h * group:, :32]).all()
    # (elsewhere, the same weights and other sums in 32 bits of the same products: rows that see so much are done by themselves)
    assert torch.equal(torch.isnan(after), torch.isnan(want)) and ((after.float() - want.float()).abs().nan_to_num(0.0) <= 2.0 ** -10 * before.abs().max().float()).all()


def test_the_same_call_gives_the_same_bits():
    c = _attend_case(5, 16, 128, 8, 8, 5, _lens(np.random.default_rng(5), 40, 1100))
    assert _share(c)[2] >= 4
    a = _run(c, 0)
    for dirty in (0xFF, 0x3C):
        for x, y in zip(a, _run(c, dirty)):
            assert torch.equal(x, y)


# ------------------------------------------------------------------------------------------------ weights


def _weigh_case(seed, N, d, kv, group, nq, lens, fp4, holes, token_major):
    rng = np.random.default_rng(seed)
    lens = np.array(lens, np.int32)
    table, blocks = wide.tables(rng, lens, N, -(-int(lens.max()) // N) + 1)
    cache = (wide.cache_fp4 if fp4 else wide.cache_fp16)(rng, table, lens, N, d, kv, blocks)
    if holes:
        table[rng.random(table.shape) < 0.1] = -1
    S, H, slots = len(lens), kv * group, table.shape[1] * N + 3
    return dict(N=N, d=d, kv=kv, lens=lens, table=table, cache=cache, fp4=fp4, token_major=token_major, q=rng.standard_normal((S, nq, H, d), dtype=np.float32).astype(np.float16),
                lse=(np.log(np.maximum(lens, 1))[:, None, None] + rng.uniform(0, 3, (S, nq, H))).astype(np.float32), weights=np.exp(2 * rng.standard_normal((S, kv, slots))).astype(np.float32),
                positions=rng.integers(-5, 1000, (S, kv, slots)).astype(np.int32), seen=(lens + rng.integers(0, 500, S)).astype(np.int32))


def _check_weigh(c, apart):
    codec = _codec(c["N"], c["d"], c["kv"], c["token_major"])
    S, nq, H, d = c["q"].shape
    q = dev(np.concatenate([c["q"], np.full((S, nq, 2, d), np.nan, np.float16)], 2))
    weights, positions, lse = dev(c["weights"]), dev(c["positions"]), dev(c["lse"])
    out = torch.full_like(weights, -3.0) if apart else weights
    cache = dev(c["cache"].transpose(0, 2, 1, 3) if c["token_major"] else c["cache"])
    codec.weigh(weights, positions, dev(c["seen"]), q[:, :, :H], cache, dev(c["table"]), dev(c["lens"]), lse, weights_out=out if apart else None)
    torch.cuda.synchronize()
    want, want_positions, bound = wide.weigh(c["weights"], c["positions"], c["seen"], dev(c["q"]), wide.Pages(c["cache"], c["N"], d, c["kv"]), c["kv"], c["table"], c["lens"], lse, d ** -0.5)
    got = out.cpu().numpy()
    inside = np.broadcast_to(np.arange(got.shape[2]) < c["lens"][:, None, None], got.shape)
    off = np.abs(got - want)[inside]
    assert (off <= bound[inside]).all(), float((off / np.maximum(bound[inside], 1e-38)).max())
    assert np.array_equal(got[~inside], np.full_like(got, -3.0)[~inside] if apart else c["weights"][~inside])
    assert np.array_equal(positions.cpu().numpy(), want_positions) and codec.stats()["status"] == 0
    if apart:
        assert np.array_equal(weights.cpu().numpy(), c["weights"])


@pytest.mark.parametrize("group,nq", [(1, 1), (2, 8), (3, 7), (8, 8)])
@pytest.mark.parametrize("N,d,most", [(16, 32, 1800), (5, 64, 1800), (16, 128, 1500), (8, 96, 1500), (3, 192, 1500), (16, 256, 1500)])
@pytest.mark.parametrize("fp4", [False, True])
def test_weights_by_waves_of_many_tiles(N, d, most, group, nq, fp4):
    """Up to 64 rows: three waves on a SIMD share the tiles of all sequences and heads."""
    kv, lens = 64, _lens(np.random.default_rng(d), 10, most)
    tiles = -(-lens // 32)
    share = -(-int(tiles.sum()) * kv // (3 * 1024))
    assert share >= 4 and tiles.max() > share and (tiles % share).any()
    c = _weigh_case(d + nq, N, d, kv, group, nq, lens, fp4, holes=nq > 1, token_major=not fp4 and N == 16)
    _check_weigh(c, apart=nq != 7)


@pytest.mark.parametrize("N,d,most", [(16, 32, 1500), (5, 64, 1500), (16, 128, 1300), (16, 256, 900)])
@pytest.mark.parametrize("fp4", [False, True])
def test_weights_of_many_queries_by_workgroups_of_many_chunks(N, d, most, fp4):
    """80 rows: 768 workgroups share the chunks of 64 tokens of all sequences and heads."""
    kv, lens = 64, _lens(np.random.default_rng(d + 1), 9, most)
    assert int((-(-lens // 64)).sum()) * kv > 3 * 768
    c = _weigh_case(d, N, d, kv, 2, 40, lens, fp4, holes=N == 5, token_major=False)
    _check_weigh(c, apart=fp4)


@pytest.mark.parametrize("nq", [1, 40])
def test_weights_of_many_short_sequences(nq):
    lens = np.random.default_rng(1).integers(0, 200, 600)
    lens[100:120] = 0
    _check_weigh(_weigh_case(7, 16, 32, 16, 2, nq, lens, True, holes=False, token_major=False), apart=True)
