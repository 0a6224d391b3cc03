"""Pins of the 4-bit cache format's oracle (oracle/paged.py): no GPU."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import paged
from paper_2608_24204_gb300 import build, ops


def nearest(x, unit, grid):
    """The place of the nearest grid value to x / unit in exact arithmetic, the even one of two that are as near."""
    x, unit = Fraction(float(x)), Fraction(float(unit))
    far = [abs(x - Fraction(float(v)) * unit) for v in grid]
    best = min(far)
    at = [i for i, f in enumerate(far) if f == best]
    return at[0] if len(at) == 1 else next(i for i in at if i % 2 == 0)


@pytest.mark.parametrize("round_to", [None, 8])
def test_codes_and_block_scales_are_the_nearest_in_exact_arithmetic(round_to):
    rng = np.random.default_rng(1)
    x = rng.normal(size=(12, 32)).astype(np.float32)
    if round_to:                                               # few bits: quotients on the middles
        m, e = np.frexp(x)
        x = np.ldexp(np.round(m * 16) / 16, e).astype(np.float32)
    x[0], x[1, :16] = 0, 0
    x[2, 5] = 1.75
    codes, each, scales = paged.quantise_e2m1(x)
    positive = paged.E4M3[:127]
    for i in range(len(x)):
        top = np.abs(x[i]).max()
        assert scales[i] == np.float32(np.float64(top) / 2688)
        for j in range(2):
            block = np.abs(x[i, 16 * j:16 * j + 16])
            b = nearest(block.max(), 6 * np.float64(scales[i]), positive) if top else 0
            assert each[i, j] == b
            for p in range(16):
                c = codes[i, 16 * j + p]
                want = nearest(block[p], positive[b] * np.float64(scales[i]), paged.E2M1[:8]) if b else 0
                assert (c & 7) == want and (c >> 3) == (np.signbit(x[i, 16 * j + p]) and top > 0)


def test_values_stay_within_the_formats_step():
    x = np.random.default_rng(2).normal(size=(200, 128)).astype(np.float32)
    codes, each, scales = paged.quantise_e2m1(x)
    v = paged.e2m1_values(codes, each, scales)
    block = np.abs(x).reshape(200, 8, 16).max(-1)
    # half a step of e2m1's largest binade is 1 of 6, and a block scale that was rounded down by 2^-4 cuts the largest
    assert np.all(np.abs(v - x).reshape(200, 8, 16).max(-1) <= block * (1 / 6 + 2.0 ** -4))
    assert np.abs(v - x).mean() < 0.1


def test_special_heads():
    x = np.ones((4, 32), np.float32)
    x[0, 3], x[1, 9], x[2] = np.inf, np.nan, 1e-33
    codes, each, scales = paged.quantise_e2m1(x)
    assert np.isnan(scales[:2]).all() and scales[2] == 0 and not codes[:3].any() and not each[:3].any()
    assert np.all(codes[3] == 7) and np.all(paged.E4M3[each[3]] == 448)


def test_pages_of_the_format():
    build.build()
    rng = np.random.default_rng(3)
    parts = (rng.integers(0, 16, (48, 2, 3, 64)).astype(np.uint8), rng.integers(0, 127, (48, 2, 3, 4)).astype(np.uint8),
             rng.normal(size=(48, 2, 3)).astype(np.float32))
    data = paged.pack_e2m1(*parts)
    assert len(data) == 3 * ops.wici_kv_page_bytes(ops.WICI_KV_E2M1, 3, 64) == 3 * 2 * 3 * 16 * (32 + 4 + 4)
    assert ops.wici_kv_page_bytes(ops.WICI_KV_E2M1, 1, 128) == 2 * 16 * (64 + 8 + 4)
    for a, b in zip(paged.unpack_e2m1(data, 3, 64), parts):
        np.testing.assert_array_equal(a, b)
    # slot 17, V, head 2, element 5: the upper half of byte 2 of its row
    block = data.reshape(3, 2, 3, -1)[1, 1, 2]
    assert block[1 * 32 + 2] >> 4 == parts[0][17, 1, 2, 5] and block[16 * 32 + 1 * 4] == parts[1][17, 1, 2, 0]
