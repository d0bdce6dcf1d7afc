"""pd_qk_norm_rope against float64: types, head counts, strided rows of a fused projection, in place, far and negative
positions, single rows and many, rows of zeros and non-finite ones."""

import numpy as np
import pytest
import torch

import oracle.paged as ref
from paged_case import HALF_STEP, h64
from paper_2606_10537_amd import _lib
from paper_2606_10537_amd._lib import PD_BF16, PD_FP32

pytestmark = pytest.mark.gpu
TYPES = {PD_BF16: torch.bfloat16, PD_FP32: torch.float32}


def check(x, w, eps, pos, base, got, dtype):
    """Tolerance, in units of |y_i| + |y_{i+d/2}|, y the normalised row: the fp32 sum of d squares, its root and
    reciprocal and three products take at most 16 roundings of 2^-24, the rotation's products two more; the reduced
    angle, at most half a turn, is rounded to fp32 (2^-25 turns, 2 pi 2^-25 rad), and sine and cosine are good to two
    units in the last place: together below 2^-19.  Then one rounding to the output type."""
    x = h64(x)
    y = ref.qk_norm_rope_ref(x, None if w is None else h64(w), eps, None, 0)
    want = ref.qk_norm_rope_ref(x, None if w is None else h64(w), eps, None if pos is None else h64(pos), base)
    size = np.abs(y)
    if base:
        size = size + np.abs(np.roll(y, y.shape[-1] // 2, -1))
    tol = 2.0 ** -19 * size + HALF_STEP[dtype] * np.abs(want) + 1e-38
    err = np.abs(h64(got) - want)
    assert np.all(err <= tol), (np.argwhere(~(err <= tol))[:4], err.max())


def rows(T, hq, hkv, d, dtype, seed, extra=0, sigma=1.5):
    g = torch.Generator().manual_seed(seed)
    fused = (torch.randn(T, hq + hkv + extra, d, generator=g) * sigma).to(TYPES[dtype]).cuda()
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(TYPES[dtype]).cuda() for _ in range(2)]
    pos = torch.randint(0, 131072, (T,), generator=g, dtype=torch.int32).cuda()
    return fused, w, pos


@pytest.mark.parametrize("dtype", [PD_BF16, PD_FP32])
@pytest.mark.parametrize("T,hq,hkv,d,extra", [(1, 28, 4, 128, 4), (1, 1, 1, 64, 0), (3, 7, 1, 128, 1), (17, 12, 4, 64, 4),
                                              (77, 5, 5, 128, 0), (1031, 32, 8, 64, 8), (2500, 9, 3, 128, 3)])
def test_fused_rows(gpu_lib, dtype, T, hq, hkv, d, extra):
    print(f"[norm] {dtype} {T} rows, {hq}/{hkv} heads of {d}", flush=True)
    fused, w, pos = rows(T, hq, hkv, d, dtype, T + hq, extra)
    q, k = fused[:, :hq], fused[:, hq:hq + hkv]
    before = fused.clone()
    qo = torch.empty(T, hq, d, dtype=fused.dtype, device="cuda")
    ko = torch.empty(T, hkv, d, dtype=fused.dtype, device="cuda")
    _lib.pd_qk_norm_rope(q, k, w[0], w[1], 1e-6, pos, 5e5, qo, ko)
    assert torch.equal(fused, before)
    check(q, w[0], 1e-6, pos, 5e5, qo, dtype)
    check(k, w[1], 1e-6, pos, 5e5, ko, dtype)
    # In place, in the rows of the projection: the same bits, and the rest of the rows untouched.
    _lib.pd_qk_norm_rope(q, k, w[0], w[1], 1e-6, pos, 5e5, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert torch.equal(fused[:, hq + hkv:], before[:, hq + hkv:])


@pytest.mark.parametrize("dtype", [PD_BF16, PD_FP32])
def test_parts(gpu_lib, dtype):
    """Norm alone, rotation alone, one of the two weights, queries alone, no rows."""
    fused, w, pos = rows(9, 6, 2, 64, dtype, 5)
    q, k = fused[:, :6], fused[:, 6:]
    out = lambda x: torch.full(x.shape, 3.0, dtype=x.dtype, device="cuda")  # noqa: E731
    qo, ko = out(q), out(k)
    _lib.pd_qk_norm_rope(q, k, w[0], w[1], 0.5, None, 0.0, qo, ko)
    check(q, w[0], 0.5, None, 0, qo, dtype)
    check(k, w[1], 0.5, None, 0, ko, dtype)
    _lib.pd_qk_norm_rope(q, k, None, None, 0.0, pos, 1e4, qo, ko)
    check(q, None, 0, pos, 1e4, qo, dtype)
    check(k, None, 0, pos, 1e4, ko, dtype)
    _lib.pd_qk_norm_rope(q, k, None, w[1], 1e-5, pos, 1e4, qo, ko)
    check(q, None, 0, pos, 1e4, qo, dtype)
    check(k, w[1], 1e-5, pos, 1e4, ko, dtype)
    _lib.pd_qk_norm_rope(q, k, None, None, 0.0, None, 0.0, qo, ko)
    assert torch.equal(qo, q) and torch.equal(ko, k)
    qo2 = out(q)
    _lib.pd_qk_norm_rope(q, None, w[0], None, 1e-6, pos, 1e4, qo2, None)
    check(q, w[0], 1e-6, pos, 1e4, qo2, dtype)
    _lib.pd_qk_norm_rope(q[:0], k[:0], w[0], w[1], 1e-6, pos[:0], 1e4, qo[:0], ko[:0])


def test_far_positions(gpu_lib):
    """Positions of a million and more, negative ones and the ends of int32: the angle is reduced in double."""
    fused, _, _ = rows(8, 2, 2, 128, PD_FP32, 6)
    pos = torch.tensor([0, 1, -1, 131071, 1 << 20, 123456789, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32, device="cuda")
    qo, ko = torch.empty(8, 2, 128, device="cuda"), torch.empty(8, 2, 128, device="cuda")
    _lib.pd_qk_norm_rope(fused[:, :2], fused[:, 2:], None, None, 0.0, pos, 1e6, qo, ko)
    check(fused[:, :2], None, 0, pos, 1e6, qo, PD_FP32)


def test_norms_beyond_the_range_of_their_squares(gpu_lib):
    """2^60 squared times 64 still fits fp32, 2^100 squared does not: zeros."""
    x = torch.ones(2, 3, 64, device="cuda")
    x[0] *= 2.0 ** 60
    x[1] *= 2.0 ** 100
    w, out = torch.full((64,), 1.5, device="cuda"), torch.full_like(x, 7.0)
    _lib.pd_qk_norm_rope(x, None, w, None, 1e-6, None, 0.0, out, None)
    assert torch.all((out[0] - 1.5).abs() <= 1.5 * 4 * 2.0 ** -24) and torch.all(out[1] == 0)   # root, division, two products


def test_zero_and_nonfinite_rows(gpu_lib):
    """A row of zeros stays zeros with eps > 0; a non-finite head spoils itself alone."""
    fused, w, pos = rows(6, 4, 2, 64, PD_BF16, 7)
    clean = fused.clone()
    fused[1, 2] = 0
    fused[3, 0, 5] = float("inf")
    fused[4, 5, 9] = float("nan")
    outs = []
    for x in (clean, fused):
        qo, ko = torch.empty(6, 4, 64, dtype=x.dtype, device="cuda"), torch.empty(6, 2, 64, dtype=x.dtype, device="cuda")
        _lib.pd_qk_norm_rope(x[:, :4], x[:, 4:], w[0], w[1], 1e-6, pos, 1e4, qo, ko)
        outs.append(torch.cat([qo, ko], 1))
    a, b = outs
    assert torch.all(b[1, 2] == 0) and torch.isnan(b[3, 0]).any() and torch.isnan(b[4, 5]).all()
    same = torch.ones(6, 6, dtype=torch.bool)
    same[1, 2] = same[3, 0] = same[4, 5] = False
    assert torch.equal(a[same], b[same])


@pytest.mark.parametrize("d", [64, 128])
def test_sines_and_cosines_keep_their_leading_bits_near_zero(gpu_lib, d):
    """Rows (1, .., 1, 0, .., 0) turn into the cosines and sines themselves.  Each is good to two units in the last place
    (2 * 2^-23 of itself) and three roundings, at the angle itself, not at the nearest fp32 one: the angle in double
    is off by at most 8 * 2^-53 of 131072 / 2 pi turns, 2^-33 rad, and so is the oracle's."""
    T = 4096
    pos = (torch.arange(T, dtype=torch.int32, device="cuda") * 32 + 7)
    x = torch.cat([torch.ones(T, 1, d // 2, device="cuda"), torch.zeros(T, 1, d // 2, device="cuda")], -1)
    out = torch.empty_like(x)
    _lib.pd_qk_norm_rope(x, None, None, None, 0.0, pos, 5e5, out, None)
    want = ref.qk_norm_rope_ref(h64(x), None, 0, h64(pos), 5e5)
    err = np.abs(h64(out) - want)
    assert np.all(err <= (2 * 2.0 ** -23 + 3 * 2.0 ** -24) * np.abs(want) + 2.0 ** -32), err.max()


def test_norms_without_eps_at_the_lower_end_of_their_squares(gpu_lib):
    """eps = 0: a mean square of 2^-126 is still there, one that vanishes in fp32 divides by zero."""
    x = torch.ones(3, 1, 64, device="cuda")
    x[0] *= 2.0 ** -63
    x[1] *= 2.0 ** -80
    x[2] = 0
    w, out = torch.full((64,), 1.5, device="cuda"), torch.full_like(x, 7.0)
    _lib.pd_qk_norm_rope(x, None, w, None, 0.0, None, 0.0, out, None)
    assert torch.all((out[0] - 1.5).abs() <= 1.5 * 4 * 2.0 ** -24)        # root, division, two products
    assert torch.all(torch.isinf(out[1])) and torch.all(torch.isnan(out[2]))
    _lib.pd_qk_norm_rope(x, None, w, None, 1e-12, None, 0.0, out, None)   # with eps all are finite
    assert torch.isfinite(out).all() and torch.all(out[2] == 0)
