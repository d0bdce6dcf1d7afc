"""Pins of the 4-bit rows' oracle: rounding by every border, the power of two by its definition, the packing."""

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged4_case import pack4, unpack4


def test_rounding_at_every_border():
    """Between neighbours the border goes to the even code; next to it the nearer value."""
    for i in range(7):
        border = (ref.E2M1[i] + ref.E2M1[i + 1]) / 2
        even = i if i % 2 == 0 else i + 1
        for sign in (1, -1):
            got = ref.e2m1_codes(sign * np.array([border, border - 2.0 ** -20, border + 2.0 ** -20]))
            assert got.tolist() == [c + (8 if sign < 0 else 0) for c in (even, i, i + 1)]
    assert ref.e2m1_codes(ref.E2M1).tolist() == list(range(8)) and ref.e2m1_codes([-0.0]).tolist() == [8]


def test_exponents_by_definition():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 2, 64)) * 2.0 ** rng.integers(-140, 120, (40, 2, 1))
    x[0] = 0
    x[1, 0, :32], x[1, 1, 40] = 6.0, np.nan
    x[2, 0, 5], x[2, 1, :] = np.inf, 3.3e38
    codes, e = ref.quantise4_ref(x)
    assert e[0].tolist() == [[-100] * 2] * 2 and e[1, 0, 0] == 0 and e[1, 1, 1] == 128 and e[2, 0, 0] == 128
    m = np.abs(x.reshape(40, 2, 2, 32)).max(-1)
    ok = e != 128
    assert np.all((m <= 6 * 2.0 ** e.astype(float))[ok]) and np.all(((m > 6 * 2.0 ** (e - 1.0)) | (e == -100))[ok])
    held = ref.held4_ref(codes, e)
    assert np.isnan(held[1, 1, 32:]).all() and np.isfinite(held[1, 1, :32]).all()
    # A value is off by at most half of the widest step below 6, and by half a step of its own.
    g, h = (np.asarray(a).reshape(40, 2, 2, 32)[ok] for a in (x, held))
    s = 2.0 ** e[ok][:, None].astype(float)
    step = np.where(np.abs(g) < 2 * s, 0.5, np.where(np.abs(g) < 4 * s, 1.0, 2.0)) * s
    assert np.all(np.abs(g - h) <= step / 2)


@pytest.mark.parametrize("d", [64, 128])
def test_packing(d):
    codes = np.random.default_rng(1).integers(0, 16, (5, d))
    byte = pack4(codes)
    assert byte.dtype is torch.uint8 and byte.shape == (5, d // 2)
    assert int(byte[0, 0]) == codes[0, 0] | codes[0, 1] << 4
    assert np.array_equal(unpack4(byte.numpy()), codes)


def test_how_far_a_held_element_is_off():
    """At most 1/5 of itself, 1/12 of the largest of its 32, or 2^-102 (a quarter of the least power of two)."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((200, 64)) * 2.0 ** rng.integers(-130, 120, (200, 1))
    x[:40] = np.linspace(-6, 6, 40 * 64).reshape(40, 64)
    x[:, 0] = np.abs(x).max(-1)
    off = np.abs(ref.held4_ref(*ref.quantise4_ref(x)) - x)
    most = np.repeat(np.abs(x.reshape(200, 2, 32)).max(-1), 32, -1)
    assert np.all(off <= np.maximum(np.maximum(np.abs(x) / 5, most / 12), 2.0 ** -102) * (1 + 2.0 ** -50))
