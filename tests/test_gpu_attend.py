"""kvc_attend against the formula in 64 bits: page shapes, heads, lengths, prefixes, blocks that are not there, and what memory holds
where no token is.  Tolerances are the reference's own bound (paged_reference.attend)."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from gpu_util import DEV
from paper_2512_11920_amd import kvc

pytestmark = pytest.mark.gpu
POISON = np.array([np.nan, np.inf, -np.inf, 65504.0, -65504.0], np.float16)


def _say(m):
    print(m, flush=True)


def _setup(rng, N, d, kv, group, q, lens, prefix=(), first=(0,), separate=False, token_major=False, holes=0.0, room=1, q_scale=1.0, blocks=None):
    """Inputs on the host.  Every row that no token owns holds NaN, infinities and FP16's extremes."""
    S, lens = len(lens), np.asarray(lens, np.int32)
    each = [-(-int(n) // N) for n in lens] + [-(-int(n) // N) for n in prefix]
    total = sum(each) + 2
    ppb = kv if separate else 2 * kv

    def cache():
        return POISON[rng.integers(0, len(POISON), (total, ppb, N, d))]

    k, v = cache(), cache() if separate else None
    perm, at, rows = rng.permutation(total), 0, []
    width, pwidth = max([0] + each[:S]) + room, max([1] + each[S:])
    for i, (n, length) in enumerate(zip(each, list(lens) + list(prefix))):
        row = np.full(width if i < S else pwidth, -1, np.int32)
        row[:n] = perm[at:at + n]
        at += n
        for j in range(n):
            here = min(N, int(length) - j * N)
            if rng.random() < holes:
                row[j] = -1  # (its block keeps the poison)
                continue
            scale = np.exp(0.5 * rng.standard_normal((ppb, 1, d)))
            k[row[j], :, :here] = (rng.standard_normal((ppb, here, d)) * scale).astype(np.float16)
            if separate:
                v[row[j], :, :here] = rng.standard_normal((ppb, here, d)).astype(np.float16)
        rows.append(row)
    heads = kv * group
    qkv = (q_scale * rng.standard_normal((S, q, heads + 2 * kv, d))).astype(np.float16)
    return dict(N=N, d=d, kv=kv, ppb=ppb, k=k, v=v, table=np.array(rows[:S], np.int32).reshape(S, width), lens=lens, qkv=qkv, heads=heads,
                prefix_table=np.array(rows[S:], np.int32).reshape(len(prefix), pwidth), prefix_lens=np.array(prefix, np.int32), prefix_first=np.array(first, np.int32),
                token_major=token_major)


def _dev_cache(x, c):
    t = torch.from_numpy(x).to(DEV)
    return t.transpose(1, 2).contiguous() if c["token_major"] else t


def _run(c, lse=True, scale=None):
    """-> codec, out, lse of a call, with the queries as a slice of a wider tensor."""
    N, d, kv, ppb = c["N"], c["d"], c["kv"], c["ppb"]
    codec = kvc.Codec(N, d, ppb)
    if c["token_major"]:
        codec.set_cache_layout(N * ppb * d, d, ppb * d)
    k, v = _dev_cache(c["k"], c), None if c["v"] is None else _dev_cache(c["v"], c)
    q = torch.from_numpy(c["qkv"]).to(DEV)[:, :, :c["heads"]]
    S, nq, H, _ = q.shape
    out = torch.full((S, nq, H, d), 7.0, dtype=torch.float16, device=DEV)
    sums = torch.full((S, nq, H), 7.0, device=DEV) if lse else None
    n_prefix = len(c["prefix_lens"])
    work = torch.full((kvc.attend_workspace(S, nq, H, kv, d, n_prefix),), 255, dtype=torch.uint8, device=DEV)
    kw = {}
    if n_prefix:
        kw = {k_: torch.from_numpy(c[k_]).to(DEV) for k_ in ("prefix_table", "prefix_lens", "prefix_first")}
    codec.attend(out, q, k, torch.from_numpy(c["table"]).to(DEV), torch.from_numpy(c["lens"]).to(DEV), work, v_cache=v, lse=sums, scale=scale, **kw)
    torch.cuda.synchronize()
    return codec, out.cpu().numpy().astype(np.float64), None if sums is None else sums.cpu().numpy().astype(np.float64)


def _want(c, scale=None):
    q = c["qkv"][:, :, :c["heads"]]
    v = c["k"] if c["v"] is None else c["v"]
    return ref.attend(q, c["k"], v, c["kv"] if c["v"] is None else 0, c["kv"], c["N"], c["table"], c["lens"], c["d"] ** -0.5 if scale is None else scale,
                      c["prefix_table"], c["prefix_lens"], c["prefix_first"])


def _compare(c, out, lse, scale=None):
    want, wl, bound, lb = _want(c, scale)
    off = np.abs(out - want)
    assert np.isfinite(out).all()
    assert (off <= bound).all(), (np.argwhere(off > bound)[:5], off.max(), (off / bound).max())
    if lse is not None:
        none = np.isneginf(wl)
        assert np.isneginf(lse[none]).all() and (out[none] == 0).all()
        assert (np.abs(lse[~none] - wl[~none]) <= lb[~none]).all(), np.abs(lse[~none] - wl[~none]).max()


EDGES = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129]


@pytest.mark.parametrize("d", range(32, 257, 32))
def test_every_head_dimension(d):
    rng = np.random.default_rng(d)
    c = _setup(rng, 16, d, 2, 3, 2, EDGES, prefix=[70, 5], first=[1, 6, 9])
    codec, out, lse = _run(c)
    _compare(c, out, lse)
    assert codec.stats()["status"] == 0 if codec.pool is not None else True


@pytest.mark.parametrize("N", [1, 3, 8, 16, 24, 31, 32, 64])
@pytest.mark.parametrize("token_major", [False, True])
def test_every_block_size(N, token_major):
    rng = np.random.default_rng(N)
    _say(f"[case] N {N} token_major {token_major}")
    c = _setup(rng, N, 64, 3, 2, 1, EDGES, prefix=[97, 64], first=[0, 4, 14], token_major=token_major, holes=0.1)
    _, out, lse = _run(c)
    _compare(c, out, lse)


@pytest.mark.parametrize("kv,group,q", [(1, 1, 1), (4, 1, 1), (2, 16, 1), (1, 17, 1), (2, 8, 4), (1, 5, 13), (1, 64, 1), (1, 33, 3)])
@pytest.mark.parametrize("separate", [False, True])
def test_heads_and_several_queries(kv, group, q, separate):
    """Up to several tiles of rows; sequences shorter than their queries, whose first queries see no token or the prefix alone."""
    rng = np.random.default_rng(kv * 100 + group * 10 + q)
    c = _setup(rng, 16, 64, kv, group, q, [0, 1, 3, 12, 40, 100], prefix=[50], first=[2, 5], separate=separate)
    _, out, lse = _run(c)
    _compare(c, out, lse)


@pytest.mark.parametrize("lens,prefix,first", [([5000], (), (0,)), ([1], (3000,), (0, 1)), ([0, 0, 0], (700,), (0, 3)), ([0, 0], (0,), (0, 2)), ([3, 0, 2500, 1], (1500, 33), (0, 1, 3)),
                                               ([9] * 70, (400,), (0, 70)), ([40] * 33, (100, 200, 300), (0, 1, 20, 33)), ([1, 2, 3], (10, 20, 30), (0, 0, 2, 2))])
def test_lengths_and_groups(lens, prefix, first):
    rng = np.random.default_rng(len(lens))
    c = _setup(rng, 16, 128, 2, 4, 1, lens, prefix=prefix, first=first)
    _, out, lse = _run(c)
    _compare(c, out, lse)


def _wider(table, width):
    """The same table with room for longer rows: which kernels a call takes goes by the room, as lengths are on the device."""
    return np.concatenate([table, np.full((len(table), width - table.shape[1]), -1, np.int32)], axis=1)


@pytest.mark.parametrize("d,N", [(32, 16), (64, 5), (96, 24), (128, 16), (128, 31), (160, 8), (192, 16), (224, 3), (256, 16)])
@pytest.mark.parametrize("rows", [(1, 1), (8, 4)])
def test_short_sequences_in_wide_tables(d, N, rows):
    """Without a prefix: in one launch, and divided over waves and joined."""
    rng = np.random.default_rng(d + N)
    group, q = rows
    lens = EDGES + [200, 300]
    c = _setup(rng, N, d, 2, group, q, lens, holes=0.05)
    _, out, lse = _run(c)
    _compare(c, out, lse)
    c["table"] = _wider(c["table"], 40000 // N)
    _, out, lse = _run(c)
    _compare(c, out, lse)


@pytest.mark.parametrize("d,N", [(32, 16), (64, 24), (96, 8), (128, 16), (128, 7), (160, 16), (256, 5)])
@pytest.mark.parametrize("rows", [(3, 1), (8, 3)])
def test_prefixes_in_wide_tables(d, N, rows):
    """Where the tables have room for long prefixes, every workgroup has a part of both; rows of one tile and of several."""
    rng = np.random.default_rng(d * 3 + N)
    group, q = rows
    lens = [0, 5, 31, 64, 100, 333, 7, 7, 7, 7, 12, 90]
    c = _setup(rng, N, d, 2, group, q, lens, prefix=(500, 1, 64, 33), first=(0, 2, 7, 8, 12), holes=0.05)
    _, out, lse = _run(c)
    _compare(c, out, lse)
    c["prefix_table"] = _wider(c["prefix_table"], 900000 // N)
    _, out, lse = _run(c)
    _compare(c, out, lse)


@pytest.mark.parametrize("d,seqs,group,q,prefix,first", [
    (160, 400, 8, 4, (160,), (0, 400)),             # 100 tiles of rows: even shares of one unit each would take 300 workers, longer ones 200
    (64, 400, 8, 4, (160,), (0, 400)),
    (160, 280, 16, 8, (70,), (0, 280)),             # more units than workers
    (32, 90, 4, 1, (300, 31, 0, 500), (0, 20, 21, 40, 88)),
    (64, 40, 2, 1, tuple(range(20, 56)), tuple(range(37)))])  # more prefixes than lanes look at
def test_division_of_prefixes(d, seqs, group, q, prefix, first):
    rng = np.random.default_rng([20, d, seqs])
    c = _setup(rng, 16, d, 1, group, q, rng.integers(0, 9, seqs), prefix=prefix, first=first)
    _, out, lse = _run(c)
    _compare(c, out, lse)


def test_many_short_sequences():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 40, 700)
    c = _setup(rng, 8, 32, 1, 2, 1, lens, prefix=(20, 60, 1, 90), first=(3, 100, 101, 400, 650))
    _, out, lse = _run(c)
    _compare(c, out, lse)


def test_prefix_rows_beyond_one_tile():
    """A group whose rows fill several tiles of any size, and end inside one."""
    rng = np.random.default_rng(6)
    c = _setup(rng, 16, 128, 1, 8, 1, [7] * 75, prefix=(333,), first=(0, 75))
    _, out, lse = _run(c)
    _compare(c, out, lse)


def test_blocks_that_are_not_there():
    """Whole tables of missing blocks leave rows empty; missing blocks inside a sequence are passed over."""
    rng = np.random.default_rng(7)
    c = _setup(rng, 16, 96, 2, 2, 3, [100, 100, 100, 64], prefix=(90, 40), first=(0, 1, 3), holes=0.4)
    c["table"][0] = -1
    c["table"][3] = -1
    c["prefix_table"][0] = -1
    _, out, lse = _run(c)
    _compare(c, out, lse)
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all() and np.isneginf(lse[3]).all()


@pytest.mark.parametrize("own,prefix", [(0, 3), (3, 0), (0, 0)])
def test_tables_of_no_blocks(own, prefix):
    """Sequences without tokens of their own behind a prefix, a prefix of no blocks, and both: tables of width zero."""
    rng = np.random.default_rng(19)
    c = _setup(rng, 16, 64, 2, 2, 1, [16 * own] * 3, prefix=(16 * prefix,), first=(0, 2), room=0)
    c["table"], c["prefix_table"] = c["table"][:, :own], c["prefix_table"][:, :prefix]
    _, out, lse = _run(c)
    _compare(c, out, lse)
    assert (out[2] == 0).all() == (own == 0)


def test_large_scores_leave_one_token():
    """Scores far apart: weights underflow to one token's, running maxima rise late."""
    rng = np.random.default_rng(8)
    c = _setup(rng, 16, 64, 2, 2, 1, [130, 1000, 64], prefix=(200,), first=(0, 2), q_scale=60.0)
    _, out, lse = _run(c)
    _compare(c, out, lse)


def test_scores_that_rise_with_every_token():
    rng = np.random.default_rng(9)
    c = _setup(rng, 16, 64, 1, 1, 1, [640])
    k = c["k"]
    for t in range(640):
        k[c["table"][0, t // 16], 0, t % 16] = np.float16(0.02 * t)
    c["qkv"][0, 0, 0] = 1.0
    _, out, lse = _run(c)
    _compare(c, out, lse)


def test_infinities_in_seen_tokens_come_through():
    rng = np.random.default_rng(10)
    c = _setup(rng, 16, 64, 1, 2, 1, [40, 40, 40])
    c["k"][c["table"][1, 1], 0, 3, 5] = np.inf   # a score of +-inf or NaN, as the formula has it
    c["k"][c["table"][2, 0], 1, 2, 7] = np.inf   # a value
    _, out, _ = _run(c)
    want = _want({**c, "k": c["k"][:, :, :, :]})[0]
    assert np.isfinite(out[0]).all()
    assert np.isinf(out[2, 0, :, 7]).all() and np.isfinite(np.delete(out[2, 0], 7, axis=1)).all()
    assert (np.isnan(out[1, 0]) == np.isnan(want[1, 0])).all()


@pytest.mark.parametrize("d,kv,group,q,N,prefix", [(64, 2, 2, 3, 16, ()), (128, 1, 8, 1, 16, (70,)), (128, 1, 4, 4, 6, (70,)), (96, 2, 4, 9, 8, ()), (192, 1, 8, 4, 16, (33,)), (256, 1, 2, 2, 8, ())])
def test_infinite_values_reach_only_the_queries_that_see_them(d, kv, group, q, N, prefix):
    """Of the last tokens, the earlier queries see fewer; and where the sequence is shorter than the queries are many, the first see none."""
    rng = np.random.default_rng([17, d, q])
    lens = [1, 2, 31, 32, 33, 64, 65, 100, 700]
    c = _setup(rng, N, d, kv, group, q, lens, prefix=prefix, first=(0, 5) if prefix else (0,))
    for s, n in enumerate(lens):
        for back in range(1, min(q, n) + 1):
            t = n - back
            at = c["table"][s, t // N], slice(kv, 2 * kv), t % N
            bad = rng.integers(0, d, 3)
            c["k"][at][:, bad] = np.array([np.inf, -np.inf, np.nan], np.float16)
    _, out, lse = _run(c)
    with np.errstate(invalid="ignore"):
        want, wl, bound, lb = _want(c)
    fine = np.isfinite(want)
    assert (np.isnan(out) == np.isnan(want)).all()
    assert (out[~fine & ~np.isnan(want)] == want[~fine & ~np.isnan(want)]).all()
    assert (np.abs(out - want)[fine] <= bound[fine]).all()
    none = np.isneginf(wl)
    assert np.isneginf(lse[none]).all() and (np.abs(lse[~none] - wl[~none]) <= lb[~none]).all()


@pytest.mark.parametrize("scale", [0.0, -0.2, 1e-30])
@pytest.mark.parametrize("d,q,N", [(64, 1, 16), (128, 3, 6), (192, 2, 16)])
def test_scales_of_zero_and_below(scale, d, q, N):
    rng = np.random.default_rng([18, d])
    c = _setup(rng, N, d, 2, 4, q, [50, 20, 0, 333, 1], prefix=(40, 97, 600), first=(0, 2, 4, 5), holes=0.3)
    _, out, lse = _run(c, scale=scale)
    _compare(c, out, lse, scale)


def test_bad_entries_are_passed_over_and_reported():
    rng = np.random.default_rng(11)
    c = _setup(rng, 16, 64, 2, 2, 1, [50, 50], prefix=(40,), first=(0, 2))
    c["table"][0, 1] = 10**6
    c["prefix_table"][0, 0] = len(c["k"])
    codec, out, lse = _run(c)
    _compare(c, out, lse)
    codec.alloc_pool(1, 4096, DEV)  # (stats wants a pool; the status is cleared with it)
    codec2, _, _ = _run_with_pool(c)
    assert codec2.stats()["status"] == kvc.ST_BAD_INDEX
    # a length beyond its table's row is cut to it
    c = _setup(rng, 16, 64, 1, 1, 1, [32, 32], room=0)
    c["lens"] = np.array([32, 200], np.int32)
    codec2, out, _ = _run_with_pool(c)
    assert codec2.stats()["status"] == kvc.ST_BAD_INDEX
    c["lens"] = np.array([32, 32], np.int32)
    want, _, bound, _ = _want(c)
    assert (np.abs(out - want) <= bound).all()


def test_groups_out_of_order_are_reported_and_not_seen():
    rng = np.random.default_rng(16)
    for first in ([0, 3, 1, 4], [4, 0, 4, 0], [2, 1, 0, -5]):
        c = _setup(rng, 16, 64, 2, 2, 1, [50, 20, 0, 33], prefix=(40, 70, 10), first=first)
        codec, out, _ = _run_with_pool(c)
        assert codec.stats()["status"] == kvc.ST_BAD_INDEX, first
        c["prefix_lens"] = np.zeros(0, np.int32)
        want, _, bound, _ = _want(c)
        assert (np.abs(out - want) <= bound).all(), first
    # ends beyond the batch are cut to it
    c = _setup(rng, 16, 64, 2, 2, 1, [50, 20, 0, 33], prefix=(40, 70), first=[-3, 2, 9])
    codec, out, _ = _run_with_pool(c)
    want, _, bound, _ = _want(c)
    assert (np.abs(out - want) <= bound).all() and codec.stats()["status"] == 0


def _run_with_pool(c):
    N, d, ppb = c["N"], c["d"], c["ppb"]
    codec = kvc.Codec(N, d, ppb)
    codec.alloc_pool(1, 4096, DEV)
    S, nq, H = c["qkv"].shape[0], c["qkv"].shape[1], c["heads"]
    q = torch.from_numpy(c["qkv"]).to(DEV)[:, :, :H]
    out = torch.empty((S, nq, H, d), dtype=torch.float16, device=DEV)
    n_prefix = len(c["prefix_lens"])
    work = torch.empty(kvc.attend_workspace(S, nq, H, c["kv"], d, n_prefix), dtype=torch.uint8, device=DEV)
    kw = {k_: torch.from_numpy(c[k_]).to(DEV) for k_ in ("prefix_table", "prefix_lens", "prefix_first")} if n_prefix else {}
    codec.attend(out, q, _dev_cache(c["k"], c), torch.from_numpy(c["table"]).to(DEV), torch.from_numpy(c["lens"]).to(DEV), work, **kw)
    torch.cuda.synchronize()
    return codec, out.cpu().numpy().astype(np.float64), None


def test_blocks_beyond_32_bit_offsets():
    """A cache of more than 2^32 elements, of which the last blocks are used."""
    N, d, kv, blocks = 16, 128, 8, (1 << 32) // (16 * 16 * 128) + 40
    rng = np.random.default_rng(12)
    cache = torch.empty((blocks, 2 * kv, N, d), dtype=torch.float16, device=DEV)
    small = _setup(rng, N, d, kv, 2, 1, [50, 33], prefix=(47,), first=(0, 2))
    n = len(small["k"])
    base = blocks - n
    cache[base:] = torch.from_numpy(small["k"]).to(DEV)
    table = np.where(small["table"] >= 0, small["table"] + base, -1).astype(np.int32)
    ptable = np.where(small["prefix_table"] >= 0, small["prefix_table"] + base, -1).astype(np.int32)
    codec = kvc.Codec(N, d, 2 * kv)
    q = torch.from_numpy(small["qkv"]).to(DEV)[:, :, :small["heads"]]
    out = torch.empty(q.shape, dtype=torch.float16, device=DEV)
    work = torch.empty(kvc.attend_workspace(2, 1, small["heads"], kv, d, 1), dtype=torch.uint8, device=DEV)
    codec.attend(out, q, cache, torch.from_numpy(table).to(DEV), torch.from_numpy(small["lens"]).to(DEV), work, prefix_table=torch.from_numpy(ptable).to(DEV),
                 prefix_lens=torch.from_numpy(small["prefix_lens"]).to(DEV), prefix_first=torch.from_numpy(small["prefix_first"]).to(DEV))
    _compare(small, out.cpu().numpy().astype(np.float64), None)
    # a token appended there and a block copied there land there too
    k = torch.randn((2, 1, kv, d), device=DEV).half()
    codec.append(cache, torch.from_numpy(table).to(DEV), torch.from_numpy(small["lens"]).to(DEV), k, -k)
    assert torch.equal(cache[int(table[0, 49 // N]), :kv, 49 % N], k[0, 0]) and torch.equal(cache[int(table[1, 32 // N]), kv:, 32 % N], -k[1, 0])
    codec.copy_blocks(cache, torch.tensor([blocks - 1], dtype=torch.int32, device=DEV), torch.tensor([3], dtype=torch.int32, device=DEV))
    assert torch.equal(cache[3].view(torch.int16), cache[blocks - 1].view(torch.int16))


def test_strided_output_and_another_stream():
    rng = np.random.default_rng(13)
    c = _setup(rng, 16, 64, 2, 2, 2, [70, 20, 5], prefix=(30,), first=(0, 2))
    side = torch.cuda.Stream()
    codec = kvc.Codec(16, 64, 4)
    q = torch.from_numpy(c["qkv"]).to(DEV)[:, :, :4]
    wide = torch.full((3, 4, 2, 96), 9.0, dtype=torch.float16, device=DEV)
    out = wide.transpose(1, 2)[..., 8:72]  # [sequence][token][head][channel] inside [sequence][head][token][96]
    work = torch.empty(kvc.attend_workspace(3, 2, 4, 2, 64, 1), dtype=torch.uint8, device=DEV)
    args = [torch.from_numpy(c[k_]).to(DEV) for k_ in ("table", "lens", "prefix_table", "prefix_lens", "prefix_first")]
    k = torch.from_numpy(c["k"]).to(DEV)
    torch.cuda.synchronize()
    codec.attend(out, q, k, args[0], args[1], work, prefix_table=args[2], prefix_lens=args[3], prefix_first=args[4], stream=side)
    side.synchronize()
    _compare(c, out.cpu().numpy().astype(np.float64), None)
    assert (wide[..., :8] == 9).all() and (wide[..., 72:] == 9).all()


def test_a_captured_step_replays():
    """append and attend of a decode step in a HIP graph, replayed with changing lengths, tables and tokens, each replay against the eager call."""
    rng = np.random.default_rng(14)
    c = _setup(rng, 16, 128, 2, 4, 1, [300, 40, 7, 0], prefix=(500,), first=(0, 3))
    codec = kvc.Codec(16, 128, 4)
    k = torch.from_numpy(np.nan_to_num(c["k"].astype(np.float32), nan=0, posinf=1, neginf=-1).clip(-4, 4).astype(np.float16)).to(DEV)
    eager_k = k.clone()
    dev = {k_: torch.from_numpy(c[k_]).to(DEV) for k_ in ("table", "lens", "prefix_table", "prefix_lens", "prefix_first")}
    qkv = torch.from_numpy(c["qkv"]).to(DEV)
    out, want = torch.empty((4, 1, 8, 128), dtype=torch.float16, device=DEV), torch.empty((4, 1, 8, 128), dtype=torch.float16, device=DEV)
    work, work2 = (torch.empty(kvc.attend_workspace(4, 1, 8, 2, 128, 1), dtype=torch.uint8, device=DEV) for _ in range(2))

    def step(cache, o, w, stream=None):
        codec.append(cache, dev["table"], dev["lens"], qkv[:, :, 8:10], qkv[:, :, 10:], stream=stream)
        codec.attend(o, qkv[:, :, :8], cache, dev["table"], dev["lens"], w, prefix_table=dev["prefix_table"], prefix_lens=dev["prefix_lens"],
                     prefix_first=dev["prefix_first"], stream=stream)

    step(k.clone(), want, work2)
    torch.cuda.synchronize()
    cap, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(cap):
        graph.capture_begin()
        step(k, out, work, cap)
        graph.capture_end()
    for rep in range(4):
        dev["lens"].copy_(torch.tensor([300 - 60 * rep, 33 + rep, 7, rep % 2], dtype=torch.int32, device=DEV))
        dev["prefix_lens"].fill_(500 - 99 * rep)
        dev["prefix_first"].copy_(torch.tensor([rep % 2, 3], dtype=torch.int32, device=DEV))
        qkv.copy_(torch.randn_like(qkv))
        torch.cuda.synchronize()
        graph.replay()
        step(eager_k, want, work2)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), want.view(torch.int16)) and torch.equal(k.view(torch.int16), eager_k.view(torch.int16)), rep


def test_the_same_call_gives_the_same_bits():
    rng = np.random.default_rng(15)
    c = _setup(rng, 16, 128, 2, 8, 1, rng.integers(1, 900, 20), prefix=(1500, 40), first=(0, 15, 18))
    outs = [_run(c)[1] for _ in range(3)]
    assert np.array_equal(outs[0], outs[1]) and np.array_equal(outs[0], outs[2])


def test_refusals():
    codec = kvc.Codec(16, 64, 4)
    cache = torch.zeros((6, 4, 16, 64), dtype=torch.float16, device=DEV)
    q = torch.zeros((2, 1, 4, 64), dtype=torch.float16, device=DEV)
    table, lens = torch.zeros((2, 3), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    work = torch.empty(kvc.attend_workspace(2, 1, 4, 2, 64, 1), dtype=torch.uint8, device=DEV)
    good = dict(out=torch.empty_like(q), q=q, cache=cache, block_table=table, lens=lens, work=work)
    codec.attend(**good)
    one = torch.zeros(1, dtype=torch.int32, device=DEV)
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(q=q[0]), dict(out=torch.empty((2, 1, 8, 64), dtype=torch.float16, device=DEV)), dict(block_table=table.long()),
                dict(block_table=table[:1]), dict(lens=lens[:1]), dict(lens=lens.float()), dict(work=work.view(torch.int8)), dict(cache=cache.float()), dict(cache=cache.transpose(1, 2)),
                dict(v_cache=cache[:3]), dict(prefix_table=table), dict(prefix_table=table, prefix_lens=one, prefix_first=torch.zeros(2, dtype=torch.int32, device=DEV)),
                dict(prefix_table=table[:1], prefix_lens=one, prefix_first=one), dict(lse=torch.empty(3, device=DEV)),
                dict(out=torch.empty((2, 1, 4, 64), dtype=torch.float16, device=DEV).transpose(2, 3)), dict(out=q[:1].expand(2, 1, 4, 64))):
        with pytest.raises(AssertionError):
            codec.attend(**{**good, **bad})
    for bad in (dict(work=work[:0]), dict(work=torch.empty(work.numel() + 16, dtype=torch.uint8, device=DEV)[8:]), dict(v_cache=cache),  # 4 heads each, 4 query heads: fine, see below
                dict(q=torch.zeros((2, 1, 4, 68), dtype=torch.float16, device=DEV)[..., :64]), dict(q=torch.zeros((2, 1, 3, 64), dtype=torch.float16, device=DEV),
                                                                                                  out=torch.empty((2, 1, 3, 64), dtype=torch.float16, device=DEV))):
        if "v_cache" in bad:
            codec.attend(**{**good, **bad, "work": torch.empty(kvc.attend_workspace(2, 1, 4, 4, 64), dtype=torch.uint8, device=DEV)})
            continue
        with pytest.raises(kvc.KvcError):
            codec.attend(**{**good, **bad})
    for scale in (float("nan"), float("inf"), 3e38):
        with pytest.raises(kvc.KvcError):
            codec.attend(**{**good, "scale": scale})
    for sizes in ((1, 1, 5, 2, 64), (1, 0, 4, 2, 64), (1, 1, 4, 2, 60), (-1, 1, 4, 2, 64), (1, 1, 4, 0, 64)):
        with pytest.raises(kvc.KvcError):
            kvc.attend_workspace(*sizes)
    # nothing to do
    codec.attend(torch.empty((0, 1, 4, 64), dtype=torch.float16, device=DEV), torch.empty((0, 1, 4, 64), dtype=torch.float16, device=DEV), cache,
                 torch.zeros((0, 3), dtype=torch.int32, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV), work)
