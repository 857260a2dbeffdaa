"""compact_pool on tables whose payloads overlap in every way: offsets dealt to pages of other sizes than they were made for."""
import numpy as np
import pytest

import paged_reference as ref
from test_gpu_cache_ops import _check_compact, _compact, _dev
from paper_2512_11920_amd import kvc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages,units,sizes", [(64, 4096, [63, 64, 65]), (500, 4097, [1, 2, 5]), (200, 70000, [0, 1, 128, 256, 512]), (3000, 300001, [3, 64, 100, 300])])
def test_offsets_of_other_pages(pages, units, sizes):
    rng = np.random.default_rng([40, pages])
    desc = np.zeros(pages, kvc.DESC_DTYPE)
    desc["n16"] = rng.choice(sizes, pages)
    off = np.minimum(np.cumsum(desc["n16"].astype(np.int64) + rng.integers(0, 30, pages)) - desc["n16"], units)
    desc["off"] = 16 * off[rng.permutation(pages)]
    desc["mode"] = rng.choice([0, 1, 2, 3, 4, 5, 0xFF], pages)
    desc["scale"] = rng.random(pages)
    codec = kvc.Codec(16, 128, 1)
    codec.bind_pool(_dev(rng.integers(0, 256, 16 * units).astype(np.uint8)), _dev(desc.view(np.uint8)))
    held = ref.compact(desc, codec.pool.cpu().numpy(), 16 * units)[1]
    for room in (16 * units, max(16, held), max(16, held // 32 * 16)):
        codec.restore_pool(0)  # (clears the status)
        out, desc_out, used = _compact(codec, room)
        assert codec.stats()["status"] == _check_compact(codec, out, desc_out, used)
