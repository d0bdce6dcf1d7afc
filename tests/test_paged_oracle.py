"""Pins of the paged-cache oracle: rotations as complex products, E4M3 rounding against torch's conversion, the power
of two by its definition, page choice by enumeration, attention against a dense masked softmax."""

import itertools
import math

import numpy as np
import pytest
import torch

import oracle.paged as ref


def test_norm_and_rotation_worked_example():
    """d = 4, base 100: the pairs (0, 2) and (1, 3) turn by pos and pos / 10; [3, 0, 4, 0] has mean square 25/4."""
    x = np.array([[[3.0, 0.0, 4.0, 0.0]]])
    y = ref.qk_norm_rope_ref(x, np.array([2.0, 1.0, 1.0, 1.0]), 0.0, [2], 100.0)[0, 0]
    a, b = 3 / 2.5 * 2, 4 / 2.5
    np.testing.assert_allclose(y, [a * math.cos(2) - b * math.sin(2), 0, b * math.cos(2) + a * math.sin(2), 0], atol=1e-15)
    assert np.array_equal(ref.qk_norm_rope_ref(x, None, 1.0, None, 0), x)


def test_rotation_is_a_complex_product_and_keeps_relative_positions():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 16))
    pos = np.array([0, 1, 7, -4, 131071])
    y = ref.qk_norm_rope_ref(x, None, 0, pos, 1e4)
    f = 1e4 ** (-2 * np.arange(8) / 16)
    z = (x[..., :8] + 1j * x[..., 8:]) * np.exp(1j * pos[:, None, None] * f)
    np.testing.assert_allclose(y, np.concatenate([z.real, z.imag], -1), atol=1e-9)
    q, k = rng.standard_normal((2, 1, 1, 16))
    dots = [float((ref.qk_norm_rope_ref(q, None, 0, [p + 3], 1e4) * ref.qk_norm_rope_ref(k, None, 0, [p], 1e4)).sum())
            for p in (0, 50, 1000)]
    assert max(dots) - min(dots) < 1e-9


def test_e4m3_rounding_matches_torch():
    rng = np.random.default_rng(2)
    x = np.concatenate([rng.uniform(-448, 448, 20000), 2.0 ** rng.uniform(-14, 8, 20000), ref.E4M3[:127],
                        (ref.E4M3[:126] + ref.E4M3[1:127]) / 2, [0.0, -0.0, 448.0, -448.0]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.e4m3_round(x), want)
    assert np.isnan(ref.e4m3_round([np.nan]))[0]


def test_exponent_is_the_least_that_fits():
    rows = np.array([[448.0, 1], [448.5, 0], [449.0, -1e-3], [224.0, 3], [0, 0], [1e-40, 0], [3e38, 1], [np.inf, 2.0], [np.nan, -7.0]])
    val, e = ref.quantise_ref(rows)
    assert e.tolist() == [0, 1, 1, -1, -100, -100, 120, -7, -6]
    for r in range(7):
        if -100 < e[r] < 120:
            assert np.abs(rows[r]).max() <= 448 * 2.0 ** e[r] and np.abs(rows[r]).max() > 448 * 2.0 ** (e[r] - 1)
    assert np.isnan(val[7, 0]) and np.isnan(val[8, 0]) and val[7, 1] * 2.0 ** e[7] == 2.0


def test_page_choice_by_enumeration():
    rng = np.random.default_rng(3)
    for n, k, first, last in itertools.product((1, 2, 5, 6), (1, 2, 4), (0, 1), (0, 2)):
        score = rng.integers(-2, 3, n).astype(float)
        got = ref.select_ref(score, k, first, last)
        forced = [j for j in range(n) if j < first or j >= n - last]
        best = None
        for s in itertools.combinations(range(n), min(k, n)):
            v = (sum(j in forced for j in s), sum(score[j] for j in s if j not in forced), [-j for j in s])
            # fewest forced pages missing, then the largest sum, then the lowest pages
            if len(forced) >= k:
                v = (v[0], 0, v[2])
            if best is None or v > best[0]:
                best = (v, list(s))
        assert got == best[1], (score, k, first, last, got, best)
    assert ref.select_ref(np.array([1.0, np.nan, 9.0, np.inf]), 2, 0, 0) == [1, 3]


def test_scores_bound_every_key():
    rng = np.random.default_rng(4)
    keys = rng.standard_normal((6, 20, 8))
    q = rng.standard_normal((3, 8))
    s = ref.page_scores_ref(q, keys.min(1), keys.max(1))
    assert np.all(s >= np.einsum("rd,pkd->prk", q, keys).max((1, 2)))
    one = keys[:, :1]
    np.testing.assert_allclose(ref.page_scores_ref(q, one.min(1), one.max(1)), (one[:, 0] @ q.T).max(1))


@pytest.mark.parametrize("causal", [0, 1])
def test_attention_against_dense_masked_softmax(causal):
    rng = np.random.default_rng(5)
    q, k, v = (rng.standard_normal(s) for s in ((4, 8), (7, 8), (7, 8)))
    ends = [4, 5, 6, 7] if causal else [7] * 4
    o, lse, mass, _ = ref.attn_ref(q, k, v, ends, 0.3)
    mask = torch.arange(7)[None] < torch.tensor(ends)[:, None]
    tq, tk, tv = (torch.from_numpy(a)[None] for a in (q, k, v))
    want = torch.nn.functional.scaled_dot_product_attention(tq, tk, tv, attn_mask=mask, scale=0.3)[0].numpy()
    np.testing.assert_allclose(o, want, atol=1e-13)
    s = torch.from_numpy(0.3 * q @ k.T).masked_fill(~mask, -math.inf)
    np.testing.assert_allclose(lse, torch.logsumexp(s, -1).numpy(), atol=1e-13)
    assert np.all(mass >= np.abs(o) - 1e-13)
    o, lse, _, _ = ref.attn_ref(q, k, v, [0, -3, 1, 2], 0.3)
    assert np.all(o[:2] == 0) and np.all(lse[:2] == -np.inf)
    np.testing.assert_allclose(o[2], v[0])
