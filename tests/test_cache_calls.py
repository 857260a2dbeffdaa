"""What the decode-step calls refuse before they launch anything, found without a GPU (tests/cache_calls.py)."""
import pytest

from cache_calls import HOST, SEEN_LOWER, UNREACHABLE, answers
from paper_2512_11920_amd import kvc

MB = 1 << 20
#: buffers of a compaction, and their bytes: a pool that one workgroup compacts, and a larger one
SIZES = [dict(pool=64 * 1024, desc=16 * 100, pool_out=32 * 1024, desc_out=16 * 100, used=8), dict(pool=8 * MB, desc=16 * 5000, pool_out=8 * MB, desc_out=16 * 5000, used=8)]


def _compaction(sizes, **at):
    sizes = dict(sizes, work=kvc.compact_workspace(sizes["pool"]))
    where = {name: (i + 1) << 30 for i, name in enumerate(sizes)}
    return sizes, dict(where, op="compact", pool_bytes=sizes["pool"], out_bytes=sizes["pool_out"], pages=sizes["desc"] // 16, **at)


@pytest.mark.parametrize("sizes", SIZES)
def test_compaction_refuses_buffers_that_overlap(sizes):
    """None of what it writes may lie in what it reads, or in something else that it writes."""
    sizes, good = _compaction(sizes)
    written = ("pool_out", "desc_out", "used", "work")
    pairs = [(a, b) for a in written for b in sizes if a != b and not (b in written and b < a)]
    calls, want = [good], [kvc.OK]
    for a, b in pairs:
        align = 256 if "work" in (a, b) else 16
        for at, code in ((good[b], kvc.ERR_ARG), (good[b] + (sizes[b] - 1) // align * align, kvc.ERR_ARG), (good[b] - (sizes[a] - 1) // align * align, kvc.ERR_ARG),
                         (good[b] + -(-sizes[b] // align) * align, kvc.OK), (good[b] - -(-sizes[a] // align) * align, kvc.OK)):
            calls.append(dict(good, **{a: at}))
            want.append(code)
    calls.append(dict(good, out_bytes=(1 << 64) - 16, pool_out=good["pool"] - 256))  # (its end has no address)
    want.append(kvc.ERR_ARG)
    got = answers(calls)
    assert [g[0] for g in got] == want, [(c, g, w) for c, g, w in zip(calls, got, want) if g[0] != w]
    assert all((n > 0) == (code == kvc.OK) for code, n, _, _ in got)


@pytest.mark.parametrize("sizes", SIZES)
def test_compaction_writes_where_the_device_sees_pinned_memory(sizes):
    """As kvc_bind_pool takes pools: pinned memory by the device's address, other host memory not at all."""
    _, good = _compaction(sizes)
    pinned = dict(good, pool_out=HOST + (7 << 30), desc_out=HOST + (8 << 30))
    both = dict(pinned, pool=HOST + (9 << 30), desc=HOST + (10 << 30))
    got = answers([good, pinned, both])
    assert [(g[0], g[2], g[3]) for g in got] == [(kvc.OK, good["pool_out"], good["desc_out"])] + [(kvc.OK, pinned["pool_out"] - SEEN_LOWER, pinned["desc_out"] - SEEN_LOWER)] * 2
    refused = [dict(good, pool_out=UNREACHABLE), dict(good, desc_out=UNREACHABLE),
               dict(both, pool_out=both["pool"] - SEEN_LOWER), dict(pinned, used=pinned["pool_out"] - SEEN_LOWER)]  # (the device sees them in one place)
    assert [g[:2] for g in answers(refused)] == [(kvc.ERR_ARG, 0)] * len(refused)


@pytest.mark.parametrize("d", [32, 96, 128, 256])
@pytest.mark.parametrize("n_q,group", [(1, 1), (3, 8)])
def test_attention_has_a_workspace_for_the_sizes_that_it_takes(d, n_q, group):
    """Query rows up to what one launch joins: 2^24 - 1 workgroups of 2048 / d (rounded down) rows.  Beyond it the call is refused, and has no workspace."""
    most = ((1 << 24) - 1) * (2048 // d) // (n_q * group)
    calls, works = [], []
    for n_seq in (most, most + 1):
        work = kvc.load().kvc_attend_workspace(n_seq, n_q, group, 1, d, 0)
        works.append(work > 0)
        calls.append(dict(op="attend", N=16, d=d, ppb=2, n_seq=n_seq, n_q=n_q, n_heads=group, n_kv_heads=1, max_blocks=1, n_cache_blocks=1, scale=1.0, d_q=MB, d_out=MB, d_k_cache=MB,
                          d_block_table=MB, d_lens=MB, d_work=MB, work_bytes=work or 1 << 60))
    assert works == [True, False]
    assert [g[0] for g in answers(calls)] == [kvc.OK, kvc.ERR_ARG]
