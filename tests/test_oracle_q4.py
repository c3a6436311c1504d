"""The 4-bit format's oracle against its definition by brute force, and the bounds its documentation gives."""
import numpy as np
import pytest

import synthetic as syn
from oracle import q4


def test_scales_ascend_and_products_are_bf16_values():
    s = q4.scale_value(np.arange(q4.SCALES))
    assert s[0] == 2.0 ** -38 and s[-1] == 7.0 * 2.0 ** 22 and (np.diff(s) > 0).all()
    p = (s[:, None] * np.arange(-8, 8)).astype(np.float32)
    assert (p.astype(np.float64) == s[:, None] * np.arange(-8, 8)).all()
    assert (syn.round_bf16(p) == p).all()
    assert np.isnan(q4.scale_value(np.arange(252, 256))).all()


@pytest.mark.parametrize("size", [2.0 ** -45, 1e-9, 0.3, 1.0, 700.0, 1e9])
def test_encode_is_the_least_scale_and_the_nearest_code(size):
    rng = np.random.default_rng(1)
    a = syn.round_bf16((rng.normal(0, size, (40, 64))).astype(np.float32)).astype(np.float64)
    codes, b = q4.encode(a)
    s = q4.scale_value(np.arange(q4.SCALES))
    for i in range(40):
        for g in range(2):
            x = a[i, 32 * g:32 * g + 32]
            fits = [k for k in range(q4.SCALES) if 7 * s[k] >= np.abs(x).max()]
            k = fits[0] if fits else q4.SCALES - 1
            assert b[i, g] == k
            for c in range(32):
                off = [abs(x[c] - v * s[k]) for v in range(-7, 8)]
                v = int(codes[i, 32 * g + c]) - 8
                assert off[v + 7] == min(off)
                if off.count(min(off)) > 1:
                    assert v % 2 == 0
                if fits:
                    assert min(off) <= s[k] / 2
    assert (q4.unpack(q4.pack(codes)) == codes).all()


def test_a_group_without_numbers_is_marked_and_alone():
    a = np.ones((3, 64))
    a[0, 5], a[1, 40] = np.nan, -np.inf
    codes, b = q4.encode(a)
    assert (b == [[255, b[2, 0]], [b[2, 0], 255], [b[2, 0], b[2, 0]]]).all()
    v = q4.decode(codes, b)
    assert np.isnan(v[0, :32]).all() and np.isnan(v[1, 32:]).all()
    assert (q4.encode(np.zeros((1, 32)))[0] == 8).all()
    assert np.abs(v[2] - 1).max() <= q4.scale_value(b[2, 0]) / 2
