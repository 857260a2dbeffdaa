"""The conversions of a cache in 4 bits, exhaustively: every finite FP16 value into it, every code with every exponent byte that append writes out of it, wherever the byte lies among its neighbours."""
import numpy as np
import pytest
import torch

import fp4_reference as ref
from gpu_util import DEV
from paper_2512_11920_amd import kvc
from wide_reference import dev

pytestmark = pytest.mark.gpu

WRITTEN = [0, *range(101, 141), 255]  # exponent bytes that append writes


def _codec(N, d, ppb):
    c = kvc.Codec(N, d, ppb)
    c.alloc_pool(1, 4096, DEV)
    return c


def test_append_of_every_fp16_value():
    """All 63,488 finite bit patterns, 31 to a group, in groups whose largest magnitude is of their own binade, and of up to four binades more, at either end of the binade and beside its 1.75."""
    N, d = 16, 256
    every = np.arange(1 << 16, dtype=np.uint16)
    every = every[every & 0x7FFF < 0x7C00]
    every = every[np.argsort(every & 0x7FFF, kind="stable")]
    few = every.reshape(2048, 31)
    top = (few & 0x7FFF).max(1).astype(np.int64)
    groups = []
    for binades in range(5):
        for mantissa in (None, 0x000, 0x2FF, 0x300, 0x301, 0x3FF):  # (None: the largest's own; 0x300: 1.75)
            lead = (top & 0x7C00) + (binades << 10) + mantissa if mantissa is not None else (top.astype(np.uint16).view(np.float16).astype(np.float64) * 2.0 ** binades).clip(0, 65504).astype(np.float16).view(np.uint16)
            lead = np.clip(lead, top, 0x7BFF).astype(np.uint16)
            sign = np.where(np.arange(len(lead)) % 2, 0x8000, 0).astype(np.uint16)
            groups.append(np.concatenate([few[:, :13], (lead | sign)[:, None], few[:, 13:]], 1))
    x = np.concatenate(groups)
    x = np.concatenate([x, np.zeros((-len(x) % (d // 32 * N), 32), np.uint16)]).view(np.float16).reshape(1, -1, 1, d)
    assert set(np.unique(x.view(np.uint16))) == set(every.tolist())
    blocks = x.shape[1] // N
    codec = _codec(N, d, 2)
    cache = torch.full((blocks, codec.fp4_block_bytes), 0xEE, dtype=torch.uint8, device=DEV)
    table, lens = np.arange(blocks, dtype=np.int32)[None], np.array([x.shape[1]], np.int32)
    codec.append_fp4(cache, dev(table), dev(lens), dev(x), dev(-x))
    got = ref.parts(cache.cpu().numpy(), N, d, 2)
    rows = x.reshape(blocks, N, d)
    for page, r in enumerate((rows, -rows)):
        codes, exps = ref.pack(r)
        assert np.array_equal(got[0][:, page], codes) and np.array_equal(got[1][:, page], exps)


def test_unpack_of_every_code_and_exponent():
    N, d = 16, 256
    rng = np.random.default_rng(0)
    cache = rng.integers(0, 256, (40, 2 * ref.page_bytes(N, d)), dtype=np.uint8)
    codes, exps = ref.parts(cache, N, d, 2)
    exps[:] = np.array(WRITTEN, np.uint8)[np.arange(exps.size) % len(WRITTEN)].reshape(exps.shape)
    both = {(int(c), int(e)) for e in WRITTEN for c in np.unique(np.concatenate([(codes & 15)[np.repeat(exps == e, 16, -1)], (codes >> 4)[np.repeat(exps == e, 16, -1)]]))}
    assert len(both) == 16 * len(WRITTEN)
    out = torch.empty((40, 2, N, d), dtype=torch.float16, device=DEV)
    _codec(N, d, 2).unpack_fp4(out, dev(cache))
    with np.errstate(over="ignore"):
        want = ref.values(codes, exps).astype(np.float16)
    got = out.cpu().numpy()
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan) and np.array_equal(got.view(np.uint16)[~nan], want.view(np.uint16)[~nan])


def _blocks(rng, N, d, S):
    """S caches' blocks of a K and a V page, all bytes random."""
    cache = rng.integers(0, 256, (S, 2 * ref.page_bytes(N, d)), dtype=np.uint8)
    return cache, *ref.parts(cache, N, d, 2)


def _attend(N, d, out, q, cache, table, lens, at_once, lse=None):
    """So many sequences to a call: few of short tables take one launch, where there are registers for it, others two."""
    codec, args = _codec(N, d, 2), [dev(x) for x in (q, table, lens)]
    cache, (S, _, H, _) = dev(cache), q.shape
    for s in range(0, S, at_once):
        n = min(at_once, S - s)
        part = [x[s:s + n] for x in args]
        codec.attend_fp4(out[s:s + n], part[0], cache, part[1], part[2], torch.empty(kvc.attend_fp4_workspace(n, 1, H, 1, d), dtype=torch.uint8, device=DEV), scale=1.0, lse=None if lse is None else lse[s:s + n])
    assert codec.stats()["status"] == 0


def _turns(N, groups):
    """Token of interest, and the exponent of each of its groups, so that every token meets every exponent in every group."""
    return [(j, [WRITTEN[(i + g) % len(WRITTEN)] for g in range(groups)]) for j in range(N) for i in range(len(WRITTEN))]


SHAPES = [(16, 32), (16, 64), (16, 96), (16, 128), (16, 224), (16, 256), (8, 192), (5, 224), (3, 256), (7, 64), (1, 160)]


@pytest.mark.parametrize("N,d", SHAPES)
@pytest.mark.parametrize("wide", [False, True])
def test_attention_reads_every_value(N, d, wide):
    """Sequence by sequence, the last token's score is 2,048 above the others', whose weights are zero: the output is its value, exactly.  Exponent bytes beside it are any that are finite, and
    behind it, where no token is, any."""
    rng = np.random.default_rng(N * d + wide)
    turns = _turns(N, d // 32)
    S = len(turns)
    cache, codes, exps = _blocks(rng, N, d, S)
    exps[:, 0] = 127
    codes[:, 0] = 0
    for s, (j, e) in enumerate(turns):
        exps[s, 1, :j] = rng.integers(0, 141, (j, d // 32))
        exps[s, 1, j] = e
        codes[s, 1, j] = rng.permuted(np.tile(np.arange(16, dtype=np.uint8) * 17, d // 32).reshape(d // 32, 16), axis=1).reshape(-1)  # (each code in either half of a byte)
        exps[s, 0, :, 0] = 127 + 8
        codes[s, 0, :j, 0], codes[s, 0, j, 0] = 0x0E, 0x06  # -4, 4
    q = np.zeros((S, 1, 1, d), np.float16)
    q[..., 0] = 1
    lens = np.array([j + 1 for j, _ in turns], np.int32)
    table = np.full((S, 9000 // N if wide else 1), -1, np.int32)
    table[:, 0] = np.arange(S)
    out = torch.empty((S, 1, 1, d), dtype=torch.float16, device=DEV)
    _attend(N, d, out, q, cache, table, lens, S if wide else 300)
    at = np.arange(S), 1, lens - 1
    want = ref.values(codes[at], exps[at]).astype(np.float16)
    got = out.cpu().numpy()[:, 0, 0]
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan) and nan.any()
    assert np.array_equal(got[~nan], want[~nan])  # (zeros of either sign alike, as sums have none of their own)


@pytest.mark.parametrize("N,d", SHAPES[1:])
@pytest.mark.parametrize("many", [False, True])
def test_scores_of_every_value(N, d, many):
    """16 or 80 heads, each with a channel of its own: lse is the last token's score, 64 and its key's channel times a power of two that makes it 2^-12 to 6, as the other tokens' weights are below
    2^-149; and the token gets a weight of one from each.  Exponent bytes beside the token are any that are finite, behind it any."""
    rng = np.random.default_rng(N * d + many)
    groups = d // 32
    turns = _turns(N, groups)
    S, H = len(turns), 80 if many else 16
    cache, codes, exps = _blocks(rng, N, d, S)
    codes[:, 0] = 0
    q = np.zeros((S, 1, H, d), np.float16)
    q[..., 0] = 1
    channel = np.empty((S, H), np.int64)
    for s, (j, e) in enumerate(turns):
        exps[s, 0, :j] = rng.integers(0, 141, (j, groups))
        exps[s, 0, j] = e
        exps[s, 0, :, 0] = 127 + 4
        codes[s, 0, :j, 0], codes[s, 0, j, 0] = 0x0E, 0x06
        codes[s, 0, j, 16:] = rng.permuted(np.tile(np.arange(16, dtype=np.uint8) * 17, groups - 1).reshape(groups - 1, 16), axis=1).reshape(-1)
        # a head's channel: all channels of the groups in turn; NaN's exponent is left to a head of its own
        channel[s] = 32 + (np.arange(H) + 16 * s) % (d - 32)
        of = exps[s, 0, j, channel[s] // 32].astype(int)
        q[s, 0, np.arange(H), channel[s]] = 2.0 ** np.clip(127 - of, -14, 15)
    nan_groups = exps[np.arange(S), 0, [j for j, _ in turns]] == 255
    nan_groups[:, 0] = False
    lens = np.array([j + 1 for j, _ in turns], np.int32)
    table = np.arange(S, dtype=np.int32)[:, None].copy()
    codec = _codec(N, d, 2)
    out, lse = torch.empty((S, 1, H, d), dtype=torch.float16, device=DEV), torch.empty((S, 1, H), device=DEV)
    _attend(N, d, out, q, cache, table, lens, S if many else 300, lse)
    got = lse.cpu().numpy()[:, 0].astype(np.float64)
    at = np.arange(S), 0, lens - 1
    # (as unpack gives it: halves and wholes of 2^-26 and the like, which append does not write as its inputs are multiples of 2^-24, are no FP16 numbers)
    key = ref.values(codes[at], exps[at]).astype(np.float16).astype(np.float64)
    want = 64 + np.take_along_axis(key, channel, 1) * np.take_along_axis(q[:, 0].astype(np.float64), channel[:, :, None], 2)[..., 0]
    none = nan_groups.any(1)  # (a NaN anywhere in a key makes its scores NaN)
    assert np.isnan(got[none]).all() and none.any()
    # eight products of 32 channels are added, a rounding each; the score is scaled by log2(e), which is rounded, relative to it the logarithm of 2^10 is made, and both are added and come back by
    # ln(2), which is rounded: 14 * 2^-24 of the score; and 2^-20 for that logarithm.  (Half of 2^-12 is 2^-13, and 14 * 2^-24 * 70 is 2^-14: every code is told from the next.)
    assert (np.abs(got - want)[~none] <= 14 * 2.0 ** -24 * np.abs(want)[~none] + 2.0 ** -20).all()
    # a weight is e^(score - lse): the score as above, 9 roundings, lse rounded to 32 bits, and by log2(e), which is rounded, and the difference: 14 at most; 2^-20 for the power; H numbers are added
    sums = np.where(none[:, None], 0.0, want).astype(np.float32)[:, None]
    weights, positions = torch.zeros((S, 1, N), device=DEV), torch.zeros((S, 1, N), dtype=torch.int32, device=DEV)
    codec.weigh(weights, positions, dev(lens), dev(q), dev(cache), dev(table), dev(lens), dev(sums), scale=1.0)
    w = weights.cpu().numpy()[np.arange(S), 0, lens - 1].astype(np.float64)
    assert np.isnan(w[none]).all()
    off = 14 * 2.0 ** -24 * np.abs(want).max(1)[~none] + 2.0 ** -20 + H * 2.0 ** -24
    assert (np.abs(w[~none] / H - 1) <= off * (1 + off)).all()
