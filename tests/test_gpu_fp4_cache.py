"""append_fp4, unpack_fp4 and attend_fp4 against plain statements in 64 bits: rows and blocks bit for bit, attention within the bound that paged_reference.attend derives for FP16 values,
which is what a cache in 4 bits holds."""
import numpy as np
import pytest
import torch

import fp4_reference as ref
import paged_reference as paged
from gpu_util import DEV
from paper_2512_11920_amd import kvc

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _codec(N, d, ppb):
    c = kvc.Codec(N, d, ppb)
    c.alloc_pool(1, 4096, DEV)
    return c


def _table(rng, lens, N, width, spare=3):
    each = [-(-int(n) // N) for n in lens]
    perm = rng.permutation(sum(each) + spare).astype(np.int32)
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for s, n in enumerate(each):
        table[s, :n] = perm[at:at + n]
        at += n
    return table, sum(each) + spare


def _rows(rng, shape):
    """Rows as caches have them, and beside them groups of every magnitude, of zeros, and some that are not finite."""
    x = rng.standard_normal(shape).astype(np.float32) * np.exp(rng.standard_normal((*shape[:-1], 1))).astype(np.float32)
    kind = rng.random((*shape[:-1], shape[-1] // 32))
    f = np.where(kind < 0.1, 2.0 ** rng.uniform(-26, 17, kind.shape), 1.0) * (kind > 0.05)
    with np.errstate(over="ignore"):  # (beyond FP16: infinities)
        return (x * np.repeat(f, 32, -1)).astype(np.float16)


def test_conversions_are_those_of_the_definition():
    """Every FP16 value beside every largest magnitude's binade: codes and exponents; and every code with every exponent."""
    N, d = 16, 256
    every = np.arange(1 << 16, dtype=np.uint16).view(np.float16)
    tops = [m * 2.0 ** k for k in range(-24, 16) for m in (1.0, 1.25, 1.5, 1.75, 1.75 + 2.0 ** -10, 2.0 - 2.0 ** -10)]
    tops = sorted({float(np.float16(t)) for t in tops if 0 < t <= 65504})
    rng = np.random.default_rng(0)
    groups = []
    for top in tops:
        fits = every[np.abs(every.astype(np.float64)) <= top]
        groups.append(np.concatenate([[np.float16(top)], rng.choice(fits, 31 + 32 * 3)])[:128].astype(np.float16).reshape(4, 32))
        groups[-1][1:, 0] = np.float16(-top)
    groups += [np.concatenate([[np.float16(x)], every[31 * i:31 * i + 31]]).reshape(1, 32) for i in range(0, 2114, 40) for x in (65504.0, 1.0, 2.0 ** -14)]
    x = np.concatenate(groups)
    x = np.concatenate([x, np.zeros((-len(x) % (d // 32 * N), 32), np.float16)]).reshape(-1, 1, 1, d)
    x = x.reshape(1, -1, 1, d)
    n = x.shape[1]
    codec = _codec(N, d, 2)
    cache = torch.full((n // N, codec.fp4_block_bytes), 0xEE, dtype=torch.uint8, device=DEV)
    codec.append_fp4(cache, _dev(np.arange(n // N, dtype=np.int32)[None]), _dev(np.array([n], np.int32)), _dev(x), _dev(-x))
    want = np.full((n // N, codec.fp4_block_bytes), 0xEE, np.uint8)
    ref.append(want, 2, 0, N, np.arange(n // N, dtype=np.int32)[None], np.array([n]), x)
    ref.append(want, 2, 1, N, np.arange(n // N, dtype=np.int32)[None], np.array([n]), -x)
    assert np.array_equal(cache.cpu().numpy(), want)
    # all codes under all exponents that FP16 values give, and NaN
    want = rng.integers(0, 256, (9, codec.fp4_block_bytes)).astype(np.uint8)
    codes, exps = ref.parts(want, N, d, 2)
    exps.reshape(-1)  # (a copy: exps is strided)
    for i, e in enumerate(list(range(101, 141)) + [0, 255]):
        exps[i % 9, i // 9 % 2, (i // 18) % N, :] = e
    exps[:] = np.where((exps >= 101) & (exps <= 140) | (exps == 0) | (exps == 255), exps, 101 + exps % 40)
    out = torch.empty((9, 2, N, d), dtype=torch.float16, device=DEV)
    codec.unpack_fp4(out, _dev(want))
    got, value = out.cpu().numpy(), ref.values(codes, exps)
    with np.errstate(over="ignore"):
        value = value.astype(np.float16)  # (codes of 6 * 2^14 and more, which no append writes, are infinite)
    nan = np.isnan(value)
    assert np.array_equal(np.isnan(got), nan) and np.array_equal(got.view(np.uint16)[~nan], value.view(np.uint16)[~nan])


@pytest.mark.parametrize("N,d,kv,new", [(16, 64, 4, 1), (16, 128, 8, 3), (1, 32, 1, 5), (7, 96, 3, 20), (32, 128, 2, 70), (8, 256, 5, 2), (16, 224, 16, 1), (5, 160, 2, 9), (11, 192, 1, 30)])
@pytest.mark.parametrize("separate", [False, True])
def test_append(N, d, kv, new, separate):
    rng = np.random.default_rng(N * d + kv)
    S, ppb, width = 9, kv if separate else 2 * kv, 6 + -(-new // N)
    lens = np.array([0, 1, new, N, N + 1, 2 * N, 3 * N - 1, new + 1, 5 * N], np.int32)
    blocks = S * width
    table = rng.permutation(blocks).astype(np.int32).reshape(S, width)
    table[4, 0] = -1          # a block that is not there
    table[6, 2] = blocks      # and one that cannot be
    codec = _codec(N, d, ppb)
    codec.set_cache_layout(ppb * N * (d + 8), N * (d + 8), d + 8)  # (which is FP16's, and not looked at)
    k, v = (rng.integers(0, 256, (blocks, codec.fp4_block_bytes)).astype(np.uint8) for _ in range(2))
    qkv = _rows(rng, (S, new, 3 + 2 * kv, d))
    kt, vt, x = _dev(k), _dev(v), _dev(qkv)
    codec.append_fp4(kt, _dev(table), _dev(lens), x[:, :, 3:3 + kv], x[:, :, 3 + kv:], v_cache=vt if separate else None)
    ref.append(k, ppb, 0, N, table, lens, qkv[:, :, 3:3 + kv])
    ref.append(v if separate else k, ppb, 0 if separate else kv, N, table, lens, qkv[:, :, 3 + kv:])
    assert np.array_equal(kt.cpu().numpy(), k) and np.array_equal(vt.cpu().numpy(), v)
    hit = lens[6] - new <= 2 * N + N - 1 and lens[6] > 2 * N
    assert codec.stats()["status"] == (kvc.ST_BAD_INDEX if hit else 0)


def test_tokens_behind_the_table_are_reported():
    codec = _codec(16, 64, 2)
    cache = torch.zeros((4, codec.fp4_block_bytes), dtype=torch.uint8, device=DEV)
    x = torch.ones((1, 3, 1, 64), dtype=torch.float16, device=DEV)
    codec.append_fp4(cache, _dev(np.array([[1, 2]], np.int32)), _dev(np.array([34], np.int32)), x, x)  # (token 31 has a place)
    assert codec.stats()["status"] == kvc.ST_BAD_INDEX
    want = np.zeros((4, codec.fp4_block_bytes), np.uint8)
    for page in (0, 1):
        ref.append(want, 2, page, 16, np.array([[1, 2]]), [34], np.ones((1, 3, 1, 64), np.float16))
    assert np.array_equal(cache.cpu().numpy(), want) and want.any()


@pytest.mark.parametrize("N,d,ppb", [(16, 64, 8), (16, 128, 16), (5, 32, 1), (24, 96, 12), (1, 256, 3), (7, 160, 2), (128, 32, 5)])
@pytest.mark.parametrize("layout", ["dense", "token_major", "padded"])
def test_unpack(N, d, ppb, layout):
    rng = np.random.default_rng(N + d)
    row, page, block = {"dense": (d, N * d, ppb * N * d), "token_major": (ppb * d, d, N * ppb * d), "padded": (d + 8, N * (d + 8) + 16, ppb * (N * (d + 8) + 16) + 32)}[layout]
    codec = _codec(N, d, ppb)
    codec.set_cache_layout(block, page, row)
    cache = rng.integers(0, 256, (9, codec.fp4_block_bytes)).astype(np.uint8)
    codes, exps = ref.parts(cache, N, d, ppb)
    exps[:] = 101 + exps % 40
    want = rng.integers(0, 1 << 16, 7 * block).astype(np.uint16)
    out = _dev(want.view(np.float16))
    src, dst = np.array([0, 8, -1, 3, 3, 9, 5, 1], np.int32), np.array([1, 0, 2, -1, 6, 3, 7, 4], np.int32)
    codec.unpack_fp4(out, _dev(cache), _dev(src), _dev(dst))
    with np.errstate(over="ignore"):
        value = ref.values(codes, exps).astype(np.float16).view(np.uint16)
    at = np.arange(ppb)[:, None, None] * page + np.arange(N)[None, :, None] * row + np.arange(d)[None, None]
    for s, t in zip(src, dst):
        if 0 <= s < 9 and 0 <= t < 7:
            want[t * block + at] = value[s]
    assert np.array_equal(out.cpu().numpy().view(np.uint16), want)
    assert codec.stats()["status"] == kvc.ST_BAD_INDEX


# ------------------------------------------------------------------------------------------------ attention


def _case(seed, N, d, kv, group, nq, lens, separate=False, width=None, holes=False):
    """A cache in which every byte that no token owns is random: codes of any kind under exponents of any kind, NaN among them."""
    rng = np.random.default_rng(seed)
    lens = np.array(lens, np.int32)
    width = max(1, -(-int(lens.max(initial=0)) // N)) + 1 if width is None else width
    table, blocks = _table(rng, lens, N, width)
    ppb = kv if separate else 2 * kv
    caches = [rng.integers(0, 256, (blocks, ppb * ref.page_bytes(N, d))).astype(np.uint8) for _ in range(1 + separate)]
    for c in caches:
        ref.parts(c, N, d, ppb)[1][rng.random((blocks, ppb, N, d // 32)) < 0.3] = 255
    most = int(lens.max(initial=0))
    k, v = (rng.standard_normal((len(lens), most, kv, d)).astype(np.float32) * np.exp(0.5 * rng.standard_normal((kv, d))) for _ in range(2))
    for s, n in enumerate(lens):
        ref.append(caches[0], ppb, 0, N, table[s:s + 1], [n], k[s:s + 1, :n].astype(np.float16))
        ref.append(caches[-1], ppb, 0 if separate else kv, N, table[s:s + 1], [n], v[s:s + 1, :n].astype(np.float16))
    if holes:
        table[rng.random(table.shape) < 0.2] = -1
    q = rng.standard_normal((len(lens), nq, kv * group, d)).astype(np.float16)
    return dict(N=N, d=d, kv=kv, ppb=ppb, lens=lens, table=table, caches=caches, q=q, separate=separate)


def _values(c):
    with np.errstate(over="ignore"):
        pages = [ref.values(*ref.parts(x, c["N"], c["d"], c["ppb"])).astype(np.float16) for x in c["caches"]]
    return pages[0], pages[-1], 0 if c["separate"] else c["kv"]


def _run(c, scale=None, stream=None, strided=False, dirty=0xAA):
    codec = _codec(c["N"], c["d"], c["ppb"])
    S, nq, H, d = c["q"].shape
    wide = _dev(np.concatenate([c["q"], np.full((S, nq, 3, d), np.nan, np.float16)], 2)) if strided else _dev(c["q"])
    out = torch.full((S, nq, H + 1, d) if strided else (S, nq, H, d), 7.0, dtype=torch.float16, device=DEV)
    lse = torch.full((S, nq, H), 5.0, device=DEV)
    work = torch.full((kvc.attend_fp4_workspace(S, nq, H, c["kv"], d),), dirty, dtype=torch.uint8, device=DEV)
    caches = [_dev(x) for x in c["caches"]]
    args = (out[:, :, :H], wide[:, :, :H], caches[0], _dev(c["table"]), _dev(c["lens"]), work)
    torch.cuda.synchronize()
    codec.attend_fp4(*args, v_cache=caches[1] if c["separate"] else None, scale=scale, lse=lse, stream=stream)
    torch.cuda.synchronize()
    if strided:
        assert (out[:, :, H] == 7).all()
    return out[:, :, :H].cpu().numpy(), lse.cpu().numpy(), codec.stats()["status"]


def _check(c, scale=None, status=0, **kw):
    out, lse, st = _run(c, scale, **kw)
    k, v, first = _values(c)
    with np.errstate(invalid="ignore"):
        want, want_lse, bound, lse_bound = paged.attend(c["q"], k, v, first, c["kv"], c["N"], c["table"], c["lens"], c["d"] ** -0.5 if scale is None else scale)
    assert np.isfinite(out).all()
    assert (np.abs(out - want) <= bound).all(), float((np.abs(out - want) / np.maximum(bound, 1e-30)).max())
    seen = np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(lse), ~seen) and (out[~seen] == 0).all()
    assert (np.abs(lse[seen] - want_lse[seen]) <= lse_bound[seen]).all()
    assert st == status
    return out


@pytest.mark.parametrize("d", range(32, 257, 32))
@pytest.mark.parametrize("N", [16, 8, 5, 1])
@pytest.mark.parametrize("kv,group,nq", [(2, 1, 1), (1, 8, 2), (2, 5, 4), (1, 7, 5)])
def test_attention_of_short_tables(d, N, kv, group, nq):
    """One launch: tables of up to 512 tokens."""
    if N * d > 4096:
        N = 4096 // d
    _check(_case(d + N, N, d, kv, group, nq, [0, 1, 2, N, 31, 32, 33, 100, 255, 256]))


@pytest.mark.parametrize("d", range(32, 257, 32))
@pytest.mark.parametrize("N", [16, 8, 3])
@pytest.mark.parametrize("kv,group,nq", [(2, 1, 1), (1, 8, 1), (2, 5, 5)])
def test_attention_of_wide_tables(d, N, kv, group, nq):
    """Divided among workers and joined, ragged, with empty sequences, missing blocks and strides."""
    if N * d > 4096:
        N = 4096 // d
    _check(_case(d + N, N, d, kv, group, nq, [0, 700, 1, 0, 33, 512, 1037, 5], separate=d % 64 == 0, width=-(-1100 // N), holes=nq > 1), strided=True)


@pytest.mark.parametrize("d", [32, 96, 128])
@pytest.mark.parametrize("N", [16, 5])
@pytest.mark.parametrize("group,nq", [(1, 1), (4, 3)])
def test_attention_of_middling_tables(d, N, group, nq):
    """One launch, several tiles to a wave."""
    _check(_case(d + N, N, d, 2, group, nq, [0, 900, 257, 512, 3, 1000, 511, 769], width=1020 // N, holes=nq > 1))


def test_one_launch_of_long_sequences():
    """256 units of up to 4,096 tokens."""
    c = _case(20, 16, 32, 64, 1, 1, [4000, 100, 0, 2100])
    _check(c)


def test_one_long_sequence():
    _check(_case(1, 16, 128, 1, 8, 1, [20011]))


def test_more_sequences_than_workers():
    _check(_case(2, 16, 32, 1, 1, 1, list(np.random.default_rng(0).integers(0, 40, 700)), width=33))


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.5])
def test_scales(scale):
    for width in (None, 70):
        _check(_case(3, 16, 64, 2, 3, 2, [77, 300, 3], width=width), scale=scale)


@pytest.mark.parametrize("N", [16, 5])
@pytest.mark.parametrize("width", [None, 70])
def test_rows_with_a_score_beyond_32_bits_are_nan(width, N):
    """Whether the tile has a mask or not; rows that stay within 32 bits have the value of their largest score, as all others are far below it."""
    c = _case(11, N, 64, 2, 6, 1, [96, 128, 40], width=width)
    scale = 8e36
    out, lse, _ = _run(c, scale)
    k, v, first = _values(c)
    seen = []
    for s, n in enumerate(c["lens"]):
        rows = [(c["table"][s, t // N], t % N) for t in range(n)]
        for h in range(c["q"].shape[2]):
            x = np.array([k[b, h // 6, r].astype(np.float64) @ c["q"][s, 0, h].astype(np.float64) for b, r in rows]) * scale / np.log(2)
            top, best = x.max(), x.argmax()
            assert abs(top / 2.0 ** 128 - 1) > 1e-4 and np.sort(x)[-2] < top * (1 - 1e-4)  # (sums are off by 64 * 2^-24 of their magnitudes' at most, here 1.5e-5 of the largest score)
            seen.append(top > 2.0 ** 128)
            if seen[-1]:
                assert np.isnan(out[s, 0, h]).all() and np.isnan(lse[s, 0, h])
            else:
                b, r = rows[best]
                assert np.array_equal(out[s, 0, h], v[b, first + h // 6, r])
    assert any(seen) and not all(seen)


def test_lengths_beyond_the_table_and_blocks_beyond_the_cache():
    for width in (None, 70):
        c = _case(4, 16, 96, 2, 2, 2, [40, 90, 64], width=width)
        c["table"][1, 2] = len(c["caches"][0])
        _check(c, status=kvc.ST_BAD_INDEX)
        c = _case(5, 16, 96, 2, 2, 1, [40, 90, 64])
        c["lens"] = c["lens"].copy()
        c["table"] = np.ascontiguousarray(c["table"][:, :5])
        c["lens"][1] = 81
        _check(c, status=kvc.ST_BAD_INDEX)
    c = _case(6, 16, 64, 1, 1, 1, [40, 30])
    c["lens"] = np.array([-3, 30], np.int32)
    _check(c)


@pytest.mark.parametrize("width", [None, 70])
@pytest.mark.parametrize("nq", [1, 4])
@pytest.mark.parametrize("N", [16, 5])
@pytest.mark.parametrize("group", [2, 8])
def test_groups_that_are_nan_reach_only_the_queries_that_see_them(width, nq, N, group):
    """A NaN group of keys makes the rows that see it NaN, one of values its channels of them; among the last tokens, of some queries and not of others."""
    c = _case(7, N, 64, 1, group, nq, [60, 100, 33], width=width)
    k, v = ref.parts(c["caches"][0], N, 64, 2), ref.parts(c["caches"][0], N, 64, 2)
    t = 99
    v[1][c["table"][1, t // N], 1, t % N, 1] = 255
    k[1][c["table"][2, 32 // N], 0, 32 % N, 0] = 255
    out, lse, _ = _run(c)
    assert np.isfinite(out[0]).all()
    assert np.isnan(out[1, nq - 1][:, 32:]).all() and np.isfinite(out[1, nq - 1][:, :32]).all() and np.isfinite(lse[1]).all()
    assert np.isnan(out[2, nq - 1]).all() and np.isnan(lse[2, nq - 1]).all()
    assert np.isfinite(out[1:, :nq - 1]).all()
    b = c["table"][1, 0]
    v[1][b, 1, 0, 0] = 255
    assert np.isnan(_run(c)[0][1][:, :, :32]).all()


def test_the_same_call_gives_the_same_bits_whatever_the_workspace_holds():
    c = _case(8, 16, 128, 2, 4, 2, [900, 3, 1500, 40])
    a = _run(c)[0]
    for dirty in (0, 0xFF):
        assert np.array_equal(_run(c, dirty=dirty)[0].view(np.uint16), a.view(np.uint16))


def test_as_attention_over_the_unpacked_cache():
    """The same products in the same order of tokens: out differs by what the order of channels does to sums in 32 bits, so within both bounds."""
    c = _case(9, 16, 128, 2, 4, 1, [900, 3, 1500, 40])
    out = _check(c)
    codec = _codec(16, 128, 4)
    fp16 = torch.empty((len(c["caches"][0]), 4, 16, 128), dtype=torch.float16, device=DEV)
    codec.unpack_fp4(fp16, _dev(c["caches"][0]))
    other = torch.empty(c["q"].shape, dtype=torch.float16, device=DEV)
    work = torch.empty(kvc.attend_workspace(4, 1, 8, 2, 128), dtype=torch.uint8, device=DEV)
    codec.attend(other, _dev(c["q"]), fp16, _dev(c["table"]), _dev(c["lens"]), work)
    k, v, first = _values(c)
    bound = paged.attend(c["q"], k, v, first, 2, 16, c["table"], c["lens"], 128 ** -0.5)[2]
    assert (np.abs(out.astype(np.float64) - other.cpu().numpy()) <= 2 * bound).all()


def test_offsets_past_32_bits():
    """Blocks at the end of a cache of 5 GB."""
    N, d, kv = 16, 128, 8
    codec = _codec(N, d, 2 * kv)
    blocks = 5 * 10**9 // codec.fp4_block_bytes
    cache = torch.zeros((blocks, codec.fp4_block_bytes), dtype=torch.uint8, device=DEV)
    c = _case(10, N, d, kv, 2, 2, [70, 33])
    small = c["table"].copy()
    c["table"][c["table"] >= 0] += blocks - len(c["caches"][0])
    cache[blocks - len(c["caches"][0]):] = _dev(c["caches"][0])
    x = _rows(np.random.default_rng(1), (2, 2, 2 * kv, d))
    x[~np.isfinite(x)] = 1
    xt = _dev(x)
    lens = _dev(c["lens"])
    codec.append_fp4(cache, _dev(c["table"]), lens, xt[:, :, :kv], xt[:, :, kv:])
    ref.append(c["caches"][0], 2 * kv, 0, N, small, c["lens"], x[:, :, :kv])
    ref.append(c["caches"][0], 2 * kv, kv, N, small, c["lens"], x[:, :, kv:])
    assert np.array_equal(cache[blocks - len(c["caches"][0]):].cpu().numpy(), c["caches"][0])
    out = torch.empty(c["q"].shape, dtype=torch.float16, device=DEV)
    work = torch.empty(kvc.attend_fp4_workspace(2, 2, 2 * kv, kv, d), dtype=torch.uint8, device=DEV)
    codec.attend_fp4(out, _dev(c["q"]), cache, _dev(c["table"]), lens, work)
    c["table"] = small
    want = _run(c)[0]
    assert np.array_equal(out.cpu().numpy().view(np.uint16), want.view(np.uint16))
    fp16 = torch.empty((2, 2 * kv, N, d), dtype=torch.float16, device=DEV)
    codec.unpack_fp4(fp16, cache, _dev(np.array([blocks - 1, blocks - 2], np.int32)))
    with np.errstate(over="ignore"):
        value = ref.values(*ref.parts(c["caches"][0], N, d, 2 * kv)).astype(np.float16)[[-1, -2]]
    assert np.array_equal(fp16.cpu().numpy(), value, equal_nan=True)


def test_another_stream_and_nothing_to_do():
    s = torch.cuda.Stream()
    _check(_case(11, 16, 64, 2, 2, 1, [50, 1200]), stream=s)
    codec = _codec(16, 64, 4)
    cache = torch.zeros((1, codec.fp4_block_bytes), dtype=torch.uint8, device=DEV)
    none = torch.empty((0, 1, 4, 64), dtype=torch.float16, device=DEV)
    ids = torch.empty(0, dtype=torch.int32, device=DEV)
    codec.attend_fp4(none, none, cache, ids.view(0, 1), ids, torch.empty(kvc.attend_fp4_workspace(0, 1, 4, 2, 64), dtype=torch.uint8, device=DEV))
    codec.append_fp4(cache, ids.view(0, 1), ids, none[:, :, :2], none[:, :, 2:])
    codec.unpack_fp4(torch.empty((0, 4, 16, 64), dtype=torch.float16, device=DEV), cache, ids)


@pytest.mark.parametrize("what", ["dtype", "span", "heads", "shape", "table", "lens", "work", "v_cache", "strides"])
def test_the_binding_refuses(what):
    codec = _codec(16, 64, 4)
    cache = torch.zeros((3, codec.fp4_block_bytes), dtype=torch.uint8, device=DEV)
    q = torch.zeros((2, 1, 4, 64), dtype=torch.float16, device=DEV)
    table, lens = torch.zeros((2, 2), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    a = dict(out=torch.empty_like(q), q=q, cache=cache, block_table=table, lens=lens, work=torch.empty(kvc.attend_fp4_workspace(2, 1, 4, 2, 64), dtype=torch.uint8, device=DEV))
    codec.attend_fp4(**a)
    bad = {"dtype": dict(cache=cache.view(torch.int8)), "span": dict(cache=cache.cpu()), "heads": dict(q=q[:, :, :3], out=a["out"][:, :, :3]), "shape": dict(q=q[:1]), "table": dict(block_table=table[:1]),
           "lens": dict(lens=lens.long()), "work": dict(work=a["work"][:512]), "v_cache": dict(v_cache=cache[:2]), "strides": dict(q=torch.zeros((2, 1, 4, 68), dtype=torch.float16, device=DEV)[..., :64])}[what]
    with pytest.raises((AssertionError, kvc.KvcError)):
        codec.attend_fp4(**dict(a, **bad))
