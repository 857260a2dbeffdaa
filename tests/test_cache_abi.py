"""The decode-step calls' host-side checks, which answer before any device work; and their workspaces' sizes."""
import ctypes as C

import pytest

from paper_2512_11920_amd import kvc


def test_calls_without_a_context_are_refused():
    lib = kvc.load()
    a, t = kvc.Append(), kvc.Attend()
    assert lib.kvc_append(None, C.byref(a), None) == kvc.ERR_ARG
    assert lib.kvc_attend(None, C.byref(t), None) == kvc.ERR_ARG
    assert lib.kvc_copy_blocks(None, None, 0, None, None, 0, 0, 0, None) == kvc.ERR_ARG
    assert lib.kvc_fork_blocks(None, None, None, 0, 0, 0, None) == kvc.ERR_ARG
    assert lib.kvc_free_blocks(None, None, 0, 0, 0, None) == kvc.ERR_ARG
    assert lib.kvc_compact_pool(None, None, 0, None, None, None, 0, None) == kvc.ERR_ARG
    assert lib.kvc_adopt_pool(None, None, 0, None, 0, None, None) == kvc.ERR_ARG


def test_argument_records_are_laid_out_as_in_c():
    assert C.sizeof(kvc.Append) == 7 * 8 + 2 * 24 + 16
    assert C.sizeof(kvc.Attend) == 3 * 8 + 2 * 24 + 3 * 8 + 5 * 8 + 7 * 4 + 4 + 16


@pytest.mark.parametrize("sizes", [(-1, 1, 4, 2, 64, 0), (1, 0, 4, 2, 64, 0), (1, 1, 4, 3, 64, 0), (1, 1, 2, 4, 64, 0), (1, 1, 4, 0, 64, 0), (1, 1, 4, 2, 0, 0), (1, 1, 4, 2, 48, 0),
                                   (1, 1, 4, 2, 288, 0), (1, 1, 4, 2, 64, -1), (2**31 - 1, 2, 1, 1, 64, 0), (2**16, 2**8, 2**8, 1, 64, 0)])
def test_attention_of_impossible_sizes_has_no_workspace(sizes):
    assert kvc.load().kvc_attend_workspace(*sizes) == 0
    with pytest.raises(kvc.KvcError):
        kvc.attend_workspace(*sizes)


@pytest.mark.parametrize("d", range(32, 257, 32))
@pytest.mark.parametrize("n_seq,n_q,heads,kv,prefixes", [(0, 1, 1, 1, 0), (1, 1, 1, 1, 0), (7, 3, 12, 4, 0), (64, 1, 64, 8, 3)])
def test_attention_workspace_holds_every_rows_sums(d, n_seq, n_q, heads, kv, prefixes):
    """A row's sums (32 bits, d of them), its maximum and its sum of weights, for each of the two parts."""
    rows = n_seq * n_q * heads * (2 if prefixes else 1)
    n = kvc.attend_workspace(n_seq, n_q, heads, kv, d, prefixes)
    assert n % 4 == 0 and rows * (4 * d + 8) <= n
    assert kvc.attend_workspace(n_seq + 1, n_q, heads, kv, d, prefixes) >= n


@pytest.mark.parametrize("pool_bytes", [16, 4096, 2**20, 2**20 + 16, 10**9, 2**33])
def test_compaction_workspace_holds_the_bitmap_and_its_sums(pool_bytes):
    groups = -(-pool_bytes // 2**20)
    assert kvc.compact_workspace(pool_bytes) >= groups * (1024 * 10 + 8)
    assert kvc.compact_workspace(pool_bytes) <= pool_bytes / 90 + 11 * 1024
