"""The largest sizes that the calls on small caches take, found without a GPU (tests/fp4_calls.py)."""
import pytest

from fp4_calls import answers
from paper_2512_11920_amd import kvc

MB = 1 << 20


def _evict(n_seq, n_kv_heads, width):
    return dict(op="evict", ppb=2 * n_kv_heads, d_k_cache=MB, n_cache_blocks=8, d_block_table=MB, d_lens=MB, d_keep=MB, d_seen=MB, d_new_lens=MB, d_weights=1 << 44, d_weights_out=1 << 44, d_positions=2 << 44,
                d_positions_out=2 << 44, max_blocks=4, n_seq=n_seq, n_kv_heads=n_kv_heads, width=width, recent=3, fp4=0, d_work=MB, work_bytes=1 << 50)


@pytest.mark.parametrize("sizes", [(1 << 22, 1, 2), (1 << 20, 4, 0), ((1 << 22) - 1, 1, 2), (1, 1, (1 << 31) - 1), (1, 1, (1 << 31) - 256), (1, 1, (1 << 31) - 257), (1, 1, 0), (3, 5, 1 << 20)])
def test_a_workspace_for_every_eviction_that_is_taken_and_for_no_other(sizes):
    code = answers([_evict(*sizes)])[0][0]
    has = bool(kvc.load().kvc_evict_workspace(*sizes))
    assert (code, has) in ((kvc.OK, True), (kvc.ERR_ARG, False))


@pytest.mark.parametrize("d,most", [(32, 1 << 28), (256, 1 << 25)])
def test_append_counts_the_pieces_of_a_tokens_rows_in_31_bits(d, most):
    """2 * KV heads * d / 8 pieces of 16 bytes: of as many as 2^31 the count would be zero, and the call nothing."""
    call = dict(op="append_fp4", d=d, d_k_cache=MB, d_v_cache=2 * MB, n_cache_blocks=8, d_block_table=MB, d_lens=MB, d_k_new=MB, d_v_new=MB, k_strides=[8, 8, 0], v_strides=[8, 8, 0], max_blocks=4, n_seq=2,
                n_new=1)
    calls = [dict(call, ppb=n, n_kv_heads=n) for n in (most - 1, most, 2 * most)]
    assert answers(calls) == [(kvc.OK, 1), (kvc.ERR_ARG, 0), (kvc.ERR_ARG, 0)]
