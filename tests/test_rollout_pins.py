"""Pins of the oracle of 4-bit floats, the layer for a few tokens and Muon:
values worked out by hand and properties that the definitions imply."""
import numpy as np
import pytest

import oracle.foremoe_rollout as R


@pytest.mark.parametrize("y,place", [(0.0, 0), (0.25, 0), (0.26, 1), (0.75, 2), (0.74, 1), (1.25, 2), (1.3, 3),
                                     (1.75, 4), (2.5, 4), (2.6, 5), (3.5, 6), (3.4, 5), (5.0, 6), (5.1, 7), (6.9, 7)])
def test_round_to_the_grid(y, place):
    assert R.mx_round(np.array([y, -y]))[0].tolist() == [place, place]
    assert R.mx_round(np.array([-y]))[1][0]


@pytest.mark.parametrize("amax,e", [(6.0, 0), (6.99, 0), (7.0, 1), (3.4, -1), (3.5, 0), (0.0, -127), (2.0 ** -140, -127),
                                    (7 * 2.0 ** -127, -126), (7 * 2.0 ** 124, 125), (3.4e38, 125), (1.0, -2)])
def test_exponent(amax, e):
    assert R.mx_exponent(np.array([amax]))[0] == e


def test_codes_by_hand():
    x = np.zeros(34)
    x[:6] = [1.0, -2.0, 3.0, 6.0, -0.2, 0.4]  # scale 1
    x[32:] = [14.0, -1.0]                     # 14 = 7 * 2: scale 4, 3.5 is a tie to 4; -0.25 a tie to 0
    codes, scales = R.mxfp4_quantize(x)
    assert scales.tolist() == [127, 129] and codes.shape == (32,)
    assert codes[:3].tolist() == [2 | 12 << 4, 5 | 7 << 4, 8 | 1 << 4]
    assert codes[16] == (6 | 8 << 4) and not codes[17:].any()
    v = R.mxfp4_values(codes, scales, 34)
    assert v[:6].tolist() == [1.0, -2.0, 3.0, 6.0, 0.0, 0.5] and v[32:].tolist() == [16.0, 0.0]


def test_values_of_values_are_themselves():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 96)) * np.exp(rng.standard_normal((40, 1)) * 20)
    v = R.mxfp4_values(*R.mxfp4_quantize(x))
    assert np.array_equal(R.mxfp4_values(*R.mxfp4_quantize(v)), v)
    # off by half of the largest step at most
    top = np.abs(x).reshape(40, 3, 32).max(-1).repeat(32, -1)
    assert np.all(np.abs(v - x) <= top / 7 * 2)


def test_a_block_that_is_not_finite():
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(64)
        x[3] = bad
        codes, scales = R.mxfp4_quantize(x)
        assert scales.tolist() == [255, 125] and not codes[:16].any()
        assert np.isnan(R.mxfp4_values(codes, scales)[:32]).all()


def test_few_tokens_is_the_sum_over_places():
    rng = np.random.default_rng(1)
    x, gu, dn = rng.standard_normal((2, 5)), rng.standard_normal((3, 8, 5)), rng.standard_normal((3, 5, 4))
    ids, gates = np.array([[0, 2, 2], [7, -1, 1]]), np.array([[0.5, 0.25, 0.25], [np.nan, np.nan, 2.0]])
    one = lambda t, e: dn[e] @ (R.silu(gu[e, :4] @ x[t]) * (gu[e, 4:] @ x[t]))  # noqa: E731
    y = R.few_tokens(x, ids, gates, gu, dn)
    np.testing.assert_allclose(y[0], 0.5 * one(0, 0) + 0.5 * one(0, 2))
    np.testing.assert_allclose(y[1], 2 * one(1, 1))
    y = R.few_tokens(x, ids, gates, gu, dn, expert_widx=np.array([1, 0, -1]))
    np.testing.assert_allclose(y[0], 0.5 * one(0, 1))


def test_newton_schulz_maps_singular_values():
    rng = np.random.default_rng(2)
    coef = (3.4445, -4.7750, 2.0315)
    for shape in ((5, 9), (9, 5), (1, 4), (6, 6)):
        u, s, v = np.linalg.svd(rng.standard_normal(shape), full_matrices=False)
        s = s / np.sqrt((s * s).sum())
        want = s.copy()
        for _ in range(5):
            want = coef[0] * want + coef[1] * want ** 3 + coef[2] * want ** 5
        np.testing.assert_allclose(R.newton_schulz((u * s) @ v, coef, 5), (u * want) @ v, atol=1e-12)
    assert 0.6 < want.min() and want.max() < 1.3


@pytest.mark.parametrize("shape", [(24, 40), (130, 70), (128, 128)])
def test_the_formats_rounding_is_small(shape):
    """Factors rounded to fp16 move X by a few 2^-11 of its norm, also where
    u has few directions: the others stay empty. Small matrices are in fp32,
    whose rounding of G shows where u is next to singular."""
    rng = np.random.default_rng(3)
    coef = (3.4445, -4.7750, 2.0315)
    for rank in (min(shape), 4):
        x = rng.standard_normal((shape[0], rank)) @ rng.standard_normal((rank, shape[1]))
        x /= np.linalg.norm(x)
        a, b = R.newton_schulz(x, coef, 5), R.newton_schulz_held(x, coef, 5)
        assert 0 < np.linalg.norm(a - b) < (2.0 ** -8 if min(shape) > 64 else 2.0 ** -11) * np.linalg.norm(a)


def test_muon_without_a_gradient_does_not_move():
    p = np.ones((3, 4))
    z = np.zeros((3, 4))
    for eps in (0.0, 1e-7):
        q, m, x = R.muon_step(p, z, z, lr=0.1, momentum=0.9, nesterov=True, steps=5, coef=(3.4445, -4.775, 2.0315),
                              eps=eps, weight_decay=0.5, scale=1.0)
        assert np.array_equal(q, p * 0.95) and not x.any() and not m.any()
