"""What the calls on small caches refuse before they launch anything, and their workspaces, found without a GPU (tests/fp4_calls.py)."""
import ctypes as C

import pytest

import fp4_reference as ref
from fp4_calls import answers
from paper_2512_11920_amd import kvc

MB = 1 << 20
BIG = 1 << 40  # (addresses that nobody looks at)


def _append(**k):
    return dict(dict(op="append_fp4", d_k_cache=MB, n_cache_blocks=8, d_block_table=MB, d_lens=MB, d_k_new=MB, d_v_new=MB, k_strides=[8, 8, 8], v_strides=[8, 8, 8], max_blocks=4, n_seq=2, n_new=1,
                     n_kv_heads=1), **k)


def _attend(**k):
    return dict(dict(op="attend_fp4", d_q=MB, d_out=MB, q_strides=[8, 8, 8], out_strides=[8, 8, 8], d_k_cache=MB, n_cache_blocks=8, d_block_table=MB, d_lens=MB, max_blocks=100, n_seq=2, n_q=1,
                     n_heads=4, n_kv_heads=1, scale=0.1, d_work=MB, work_bytes=BIG), **k)


def _weigh(**k):
    return dict(dict(op="weigh", d_q=MB, q_strides=[8, 8, 8], d_k_cache=MB, n_cache_blocks=8, d_block_table=MB, d_lens=MB, d_lse=MB, d_weights=2 * MB, d_weights_out=2 * MB, d_positions=3 * MB, d_seen=MB,
                     max_blocks=4, n_seq=2, n_q=1, n_heads=4, n_kv_heads=1, width=64, fp4=0, scale=0.1), **k)


def _evict(**k):
    return dict(dict(op="evict", d_k_cache=MB, n_cache_blocks=8, d_block_table=MB, d_lens=MB, d_keep=MB, d_seen=MB, d_new_lens=MB, d_weights=2 * MB, d_weights_out=2 * MB, d_positions=3 * MB,
                     d_positions_out=3 * MB, max_blocks=4, n_seq=2, n_kv_heads=1, width=64, recent=3, fp4=0, d_work=MB, work_bytes=BIG), **k)


def _unpack(out=MB, n_out=8, cache=MB, n_cache=8, src=MB, dst=MB, n=3):
    return dict(op="unpack_fp4", args=[out, n_out, cache, n_cache, src, dst, n])


GOOD = [_append(), _append(n_seq=0, d_k_cache=0), _append(n_new=0, d_lens=0), _append(max_blocks=0, d_block_table=0), _attend(), _attend(n_seq=0, d_q=0), _attend(max_blocks=0, d_block_table=0),
        _attend(n_cache_blocks=0), _weigh(), _weigh(fp4=1), _weigh(n_seq=0, d_q=0), _weigh(width=0, d_weights=0, d_weights_out=0, d_positions=0), _weigh(ppb=1), _weigh(d_weights_out=2 * MB + 512), _evict(),
        _evict(fp4=1), _evict(n_seq=0, d_k_cache=0), _evict(width=0, d_weights=0, d_weights_out=0, d_positions=0, d_positions_out=0), _evict(d_weights_out=2 * MB + 512, d_positions_out=3 * MB - 512),
        _evict(ppb=1, d_v_cache=MB), _unpack(), _unpack(n=0, out=0), _unpack(src=0, dst=0, n=8)]
BAD = [
    *[_append(**{f: 0}) for f in ("d_k_cache", "d_block_table", "d_lens", "d_k_new", "d_v_new")], *[_append(**{f: MB + 8}) for f in ("d_k_cache", "d_v_cache", "d_k_new", "d_v_new")],
    _append(n_seq=-1), _append(n_new=-1), _append(max_blocks=-1), _append(n_cache_blocks=-1), _append(n_kv_heads=2), _append(n_kv_heads=0), _append(k_strides=[4, 8, 8]), _append(v_strides=[8, -8, 8]),
    _append(n_seq=1 << 20, n_new=1 << 4), _append(n_kv_heads=2, d_v_cache=MB, ppb=3),
    *[_attend(**{f: 0}) for f in ("d_q", "d_out", "d_k_cache", "d_block_table", "d_lens", "d_work", "n_q", "n_kv_heads", "n_heads")],
    *[_attend(**{f: MB + 8}) for f in ("d_q", "d_out", "d_k_cache", "d_v_cache", "d_work")], _attend(n_prefix=1), _attend(n_prefix=-1), _attend(n_heads=3, n_kv_heads=2, ppb=4), _attend(q_strides=[8, 8, 4]),
    _attend(out_strides=[-8, 8, 8]), _attend(scale=float("inf")), _attend(scale=float("nan")), _attend(scale=3e38), _attend(work_bytes=0), _attend(max_blocks=1 << 27), _attend(max_blocks=1 << 26, n_seq=100),
    _attend(n_seq=1 << 30, n_q=4), _attend(max_blocks=-1), _attend(n_cache_blocks=-1), _attend(n_seq=-1),
    *[_weigh(**{f: 0}) for f in ("d_q", "d_k_cache", "d_block_table", "d_lens", "d_lse", "d_weights", "d_weights_out", "d_positions", "d_seen", "n_q", "n_kv_heads")], _weigh(d_q=MB + 8),
    _weigh(d_k_cache=MB + 8), _weigh(ppb=3), _weigh(n_heads=3, n_kv_heads=2, ppb=4), _weigh(q_strides=[8, 8, 9]), _weigh(scale=float("inf")), _weigh(width=-1), _weigh(max_blocks=1 << 27),
    _weigh(max_blocks=1 << 26, n_seq=100), _weigh(d_weights_out=2 * MB + 256), _weigh(d_positions=2 * MB), _weigh(d_positions=2 * MB - 256), _weigh(d_weights_out=3 * MB + 4), _weigh(width=(1 << 31) - 1),
    *[_evict(**{f: 0}) for f in ("d_k_cache", "d_block_table", "d_lens", "d_keep", "d_seen", "d_new_lens", "d_weights", "d_weights_out", "d_positions", "d_positions_out", "d_work", "n_kv_heads")],
    _evict(d_k_cache=MB + 8), _evict(d_v_cache=MB + 8, ppb=1), _evict(d_work=MB + 128), _evict(work_bytes=511), _evict(recent=-1), _evict(width=-1), _evict(n_seq=-1), _evict(n_kv_heads=2),
    _evict(d_weights_out=2 * MB + 256), _evict(d_positions_out=3 * MB + 256), _evict(d_positions=2 * MB, d_positions_out=2 * MB), _evict(d_positions_out=2 * MB), _evict(d_weights_out=3 * MB),
    _evict(width=1 << 30, n_seq=8), _evict(n_seq=1 << 22, width=2), _evict(max_blocks=1 << 27),
    _unpack(out=0), _unpack(cache=0), _unpack(out=MB + 8), _unpack(cache=MB + 8), _unpack(n=-1), _unpack(n_out=-1), _unpack(n_cache=-1), _unpack(src=0, n=9), _unpack(dst=0, n=9), _unpack(n=1 << 24),
]


def test_calls_that_are_taken_and_calls_that_are_refused():
    got = answers(GOOD + BAD)
    launches = {"append_fp4": 1, "attend_fp4": 2, "weigh": 1, "evict": 2, "unpack_fp4": 1}
    for c, (code, n) in zip(GOOD, got):
        empty = c.get("n_seq", 1) == 0 or c.get("n_new", 1) == 0 or c.get("args", [1])[-1] == 0
        want = 1 if c["op"] == "attend_fp4" and c["max_blocks"] == 0 else launches[c["op"]]  # (short tables take one)
        assert code == kvc.OK and n == (0 if empty else want), (c, code, n)
    for c, (code, n) in zip(BAD, got[len(GOOD):]):
        assert code == kvc.ERR_ARG and n == 0, (c, code, n)


def test_calls_of_few_tokens_and_units_take_one_launch():
    """A workgroup for every unit: up to 512 units of tables of 512 tokens, and longer ones where heads are narrow and units are many enough."""
    calls = [(_attend(max_blocks=64), 1), (_attend(max_blocks=65), 2), (_attend(max_blocks=65, n_seq=32), 1), (_attend(max_blocks=128, n_seq=512), 1), (_attend(max_blocks=32, n_seq=513), 2),
             (_attend(max_blocks=512, n_seq=256), 1), (_attend(max_blocks=512, n_seq=128), 2), (_attend(max_blocks=512, n_seq=257), 2), (_attend(max_blocks=513, n_seq=256), 2),
             (_attend(max_blocks=32, n_heads=20), 1), (_attend(max_blocks=33, n_heads=20), 2), (_attend(max_blocks=32, d=224), 1), (_attend(max_blocks=33, d=224), 2), (_attend(max_blocks=1, d=256), 2)]
    assert answers([dict(c) for c, _ in calls]) == [(kvc.OK, n) for _, n in calls]


def test_calls_without_a_context_are_refused():
    lib = kvc.load()
    for name, record in (("append_fp4", kvc.Append), ("attend_fp4", kvc.Attend), ("weigh", kvc.Weigh), ("evict", kvc.Evict)):
        assert getattr(lib, "kvc_" + name)(None, C.byref(record()), None) == kvc.ERR_ARG
    assert lib.kvc_unpack_fp4(None, None, 0, None, 0, None, None, 0, None) == kvc.ERR_ARG


def test_argument_records_are_laid_out_as_in_c():
    assert C.sizeof(kvc.Weigh) == 8 + 24 + 9 * 8 + 8 * 4
    assert C.sizeof(kvc.Evict) == 12 * 8 + 6 * 4 + 16


@pytest.mark.parametrize("N,d,ppb", [(16, 128, 16), (16, 64, 8), (1, 32, 1), (24, 96, 12), (7, 224, 3), (128, 32, 2)])
def test_block_bytes(N, d, ppb):
    assert kvc.load().kvc_fp4_block_bytes(N, d, ppb) == ppb * ref.page_bytes(N, d)


@pytest.mark.parametrize("shape", [(0, 64, 1), (16, 48, 1), (16, 0, 1), (16, 288, 1), (64, 128, 1), (16, 64, 0)])
def test_shapes_that_no_codec_has_have_no_block(shape):
    assert kvc.load().kvc_fp4_block_bytes(*shape) == 0


@pytest.mark.parametrize("sizes", [(-1, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 4, 3, 64), (1, 1, 2, 4, 64), (1, 1, 4, 0, 64), (1, 1, 4, 2, 48), (1, 1, 4, 2, 288), (2**31 - 1, 2, 1, 1, 64)])
def test_attention_of_impossible_sizes_has_no_workspace(sizes):
    with pytest.raises(kvc.KvcError):
        kvc.attend_fp4_workspace(*sizes)


@pytest.mark.parametrize("sizes", [(-1, 1, 4), (1, 0, 4), (1, 1, -1), (2**20, 2**10, 4096)])
def test_eviction_of_impossible_sizes_has_no_workspace(sizes):
    with pytest.raises(kvc.KvcError):
        kvc.evict_workspace(*sizes)


@pytest.mark.parametrize("n_seq,kv,width", [(0, 1, 0), (1, 1, 1), (7, 3, 129), (64, 8, 8208)])
def test_eviction_workspace_holds_all_moves(n_seq, kv, width):
    assert kvc.evict_workspace(n_seq, kv, width) >= n_seq * kv * (2 * (width // 2) + 1) * 4 + 4 * n_seq
