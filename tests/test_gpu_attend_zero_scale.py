"""A scale of zero makes zeros of finite products and NaN of infinite ones, in a sequence's own tokens and in a prefix's alike."""
import numpy as np
import pytest

from test_gpu_attend_nan import _case, _row
from test_gpu_attend import _run, _want

import torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("way", ["direct", "shared", "prefix", "prefix_divided", "prefix_by_itself"])
@pytest.mark.parametrize("what", ["key", "query"])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_infinite_products(way, what, value):
    c = _case(way, 8)
    c["qkv"][:, :, :, 0] = np.abs(c["qkv"][:, :, :, 0]) + np.float16(0.1)
    if what == "query":
        c["qkv"][0, :, 1, 5] = value
    else:
        for s, n in [(0, c["lens"][0])] + [(-1 - g, n) for g, n in enumerate(c["prefix_lens"][:1])]:
            b, r = _row(c, s, int(n) - 1)
            c["k"][b, :c["kv"], r, 0] = value
    _, out, lse = _run(c, scale=0.0)
    with np.errstate(invalid="ignore"):
        want, wl, bound, _ = _want(c, 0.0)
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(np.isnan(lse), np.isnan(wl))
    assert np.isnan(want).any() and np.isfinite(want).any()
    fine = np.isfinite(want)
    assert (np.abs(out - want)[fine] <= bound[fine]).all()
