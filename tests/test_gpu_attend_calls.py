"""kvc_attend as programs call it: chunks of prompts, tables with entries behind the last token, the status word after calls in order, and infinite values
among the last tokens of short sequences.  Tolerances are the reference's own bound (paged_reference.attend)."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from paper_2512_11920_amd import kvc
from test_gpu_attend import EDGES, _compare, _dev_cache, _run, _run_with_pool, _setup, _want, _wider

pytestmark = pytest.mark.gpu


def _garbage(c, rng):
    """Entries behind a row's last token are whatever memory held, also where the tables have room: they are no block numbers."""
    N = c["N"]
    for name, lens in (("table", c["lens"]), ("prefix_table", c["prefix_lens"])):
        table = _wider(c[name], c[name].shape[1] + 3)
        for row, n in zip(table, lens):
            behind = slice(-(-int(n) // N), None)
            row[behind] = rng.integers(-2**31, 2**31 - 1, len(row[behind]))
        c[name] = table


@pytest.mark.parametrize("d", range(32, 257, 32))
@pytest.mark.parametrize("N,prefix,first", [(16, (70, 5), (1, 6, 9)), (16, (), (0,)), (7, (70, 5), (1, 6, 9)), (7, (), (0,))])
def test_status_stays_clear(d, N, prefix, first):
    rng = np.random.default_rng([30, d, N, len(prefix)])
    c = _setup(rng, N, d, 2, 3, 2, EDGES, prefix=prefix, first=first, holes=0.05)
    _garbage(c, rng)
    codec, out, _ = _run_with_pool(c)
    _compare(c, out, None)
    assert codec.stats()["status"] == 0
    c["table"] = _wider(c["table"], 40000 // N)  # (by the kernels for long sequences too)
    codec, out, _ = _run_with_pool(c)
    _compare(c, out, None)
    assert codec.stats()["status"] == 0


@pytest.mark.parametrize("d,kv,group,q,lens,prefix,first", [
    (128, 1, 8, 128, [128, 300], (), (0,)),               # a first chunk, and a later one
    (128, 2, 2, 512, [512], (), (0,)),
    (64, 1, 4, 200, [200, 777, 201], (333,), (0, 2)),     # behind a system prompt
    (96, 2, 1, 333, [400, 100, 333], (), (0,)),           # (one sequence is shorter than its queries)
    (256, 1, 1, 150, [150, 1000], (64,), (1, 2)),
    (32, 2, 3, 65, [65, 70, 4000], (), (0,)),
    (160, 1, 2, 130, [140, 0, 131], (90, 40), (0, 1, 3))])
def test_chunks_of_prompts(d, kv, group, q, lens, prefix, first):
    rng = np.random.default_rng([31, d, q])
    c = _setup(rng, 16, d, kv, group, q, lens, prefix=prefix, first=first, holes=0.03)
    _, out, lse = _run(c)
    _compare(c, out, lse)


def test_chunks_add_up_to_the_whole_prompt():
    """A prompt's rows come out the same, within the bound, whichever chunk computed them."""
    rng = np.random.default_rng(32)
    n = 300
    c = _setup(rng, 16, 64, 2, 2, n, [n])
    want, _, bound, _ = _want(c)
    for chunk in (300, 128, 64, 17, 1):
        got = np.zeros_like(want)
        for at in range(0, n, chunk):
            m = min(chunk, n - at)
            part = dict(c, qkv=c["qkv"][:, at:at + m], lens=np.array([at + m], np.int32))
            got[:, at:at + m] = _run(part, lse=False)[1]
        assert (np.abs(got - want) <= bound).all(), chunk


@pytest.mark.parametrize("d,kv,group,q,N", [(64, 2, 2, 3, 16), (128, 1, 8, 2, 16), (128, 2, 4, 4, 6), (96, 2, 4, 9, 8), (224, 1, 2, 4, 16), (32, 1, 1, 2, 31)])
@pytest.mark.parametrize("what", ["values", "keys"])
def test_infinite_rows_of_short_sequences_reach_only_the_queries_that_see_them(d, kv, group, q, N, what):
    """Where every sequence is short, a call is one launch with limits of its own for each tile."""
    rng = np.random.default_rng([33, d, q])
    lens = [1, 2, 31, 32, 33, 64, 65, 100, 257, 440]
    c = _setup(rng, N, d, kv, group, q, lens)
    assert c["table"].shape[1] * N <= 512
    for s, n in enumerate(lens):
        for back in range(1, min(q, n) + 1):
            t = n - back
            block = c["k"][c["table"][s, t // N]]
            if what == "values":
                block[kv:, t % N][:, rng.integers(0, d, 3)] = np.array([np.inf, -np.inf, np.nan], np.float16)
            else:
                block[:kv, t % N, 0] = np.nan
    _, out, lse = _run(c)
    with np.errstate(invalid="ignore"):
        want, wl, bound, lb = _want(c)
    fine = np.isfinite(want)
    assert (~fine).any() and fine.any()
    assert np.array_equal(out[~fine], want[~fine], equal_nan=True) and (np.abs(out - want)[fine] <= bound[fine]).all()
    known = np.isfinite(wl)
    assert np.array_equal(lse[~known], wl[~known], equal_nan=True) and (np.abs(lse - wl)[known] <= lb[known]).all()


def test_the_same_inputs_give_the_same_bits_whatever_lay_in_the_workspace():
    """Every shape of work, three times over, with other bytes left in the workspace and the output."""
    rng = np.random.default_rng(34)
    for N, d, kv, group, q, lens, prefix, first in ((16, 128, 8, 8, 1, rng.integers(1, 500, 64), (4096,), (0, 64)), (24, 96, 6, 3, 4, rng.integers(7, 901, 45), (333, 800, 2222), (0, 5, 20, 45)),
                                                    (16, 128, 4, 1, 1, rng.integers(1024, 2048, 8), (), (0,)), (16, 64, 4, 1, 1, [256], (), (0,)), (16, 160, 2, 8, 4, [900, 12, 77], (640,), (0, 2)),
                                                    (16, 128, 2, 8, 4, [3000, 50], (), (0,))):
        c = _setup(rng, N, d, kv, group, q, lens, prefix=prefix, first=first)
        codec, S, H = kvc.Codec(N, d, 2 * kv), len(lens), c["heads"]
        k = _dev_cache(c["k"], c)
        dev = {n: torch.from_numpy(c[n]).to(DEV) for n in ("table", "lens", "qkv", "prefix_table", "prefix_lens", "prefix_first")}
        kw = {n: dev[n] for n in ("prefix_table", "prefix_lens", "prefix_first")} if len(prefix) else {}
        got = []
        for fill in (0, 255, 0x3C):
            work = torch.full((kvc.attend_workspace(S, q, H, kv, d, len(prefix)),), fill, dtype=torch.uint8, device=DEV)
            out, lse = torch.full((S, q, H, d), float(fill), dtype=torch.float16, device=DEV), torch.full((S, q, H), float(fill), device=DEV)
            codec.attend(out, dev["qkv"][:, :, :H], k, dev["table"], dev["lens"], work, lse=lse, **kw)
            got.append((out.view(torch.int16), lse.view(torch.int32)))
        assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other)), (N, d)
