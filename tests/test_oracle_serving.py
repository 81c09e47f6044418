"""Pins of the serving operators' oracle: closed forms and brute force on the CPU."""
import cmath
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import serving as ref


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotation_is_a_complex_product(adjacent):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 2, 24))
    freqs, positions = [1.0, 0.1, 1e-3, 2.0], [0, 7, 123456]
    y = ref.rotate(x, positions, freqs, adjacent)
    for t, p in enumerate(positions):
        for h in range(2):
            for i, f in enumerate(freqs):
                a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + 4)
                z = complex(x[t, h, a], x[t, h, b]) * cmath.exp(1j * p * f)
                assert abs(z - complex(y[t, h, a], y[t, h, b])) < 1e-9
            np.testing.assert_array_equal(y[t, h, 8:], x[t, h, 8:])
    np.testing.assert_array_equal(ref.rotate(x, positions, []), x)


def test_rotated_products_depend_on_the_distance_only():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 8))
    freqs = [1.0, 0.3, 0.1, 0.01]
    dot = lambda a, b: float((ref.rotate(q, [a], freqs) * ref.rotate(k, [b], freqs)).sum())  # noqa: E731
    assert abs(dot(5, 2) - dot(105, 102)) < 1e-10 and abs(dot(5, 2) - dot(5, 3)) > 1e-3


@pytest.mark.parametrize("place,shape", [(ref.key_place, (4, 2, 16, 8)), (ref.value_place, (4, 2, 16, 8))])
def test_places_are_one_to_one(place, shape):
    seen = np.zeros(shape, int)
    for t in range(64):
        for d in range(16):
            seen[place(t, d)] += 1
    assert (seen == 1).all()


def test_attention_closed_forms():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 9, 2, 4))
    zero = np.zeros((9, 4, 4))
    out, weight = ref.attend(zero, k, v, np.arange(9), 0.5)  # equal scores: running means
    for i in range(9):
        np.testing.assert_allclose(out[i, 3], v[:i + 1, 1].mean(0))
        np.testing.assert_allclose(weight[i, 0], np.abs(v[:i + 1, 0]).mean(0))
    out, _ = ref.attend(zero, k, v, np.arange(9), 0.5, window=3)
    np.testing.assert_allclose(out[8, 0], v[6:, 0].mean(0))
    np.testing.assert_allclose(out[1, 2], v[:2, 1].mean(0))
    one = np.zeros((1, 1, 4))
    one[0, 0, 0] = 1.0  # two keys with scores ln 3 and 0: weights 3/4, 1/4
    k2 = np.zeros((2, 1, 4))
    k2[0, 0, 0] = math.log(3)
    out, _ = ref.attend(one, k2, v[:2, :1], [1], 1.0)
    np.testing.assert_allclose(out[0, 0], 0.75 * v[0, 0] + 0.25 * v[1, 0])
    out, _ = ref.attend(one, k2, v[:2, :1], [-1], 1.0)
    assert not out.any()


def brute(weights, u, top_k, top_p, min_p):
    """The definition on exact weights."""
    w = [Fraction(x) for x in weights]
    order = sorted(range(len(w)), key=lambda i: (-w[i], i))
    if 0 < top_k < len(w):
        order = order[:top_k]
    if top_p < 1:
        mass, run, kept = sum(w[i] for i in order), Fraction(0), []
        for i in order:
            if kept and not run < Fraction(top_p) * mass:
                break
            kept.append(i)
            run += w[i]
        order = kept
    order = sorted(i for i in order if w[i] >= min(Fraction(min_p), 1) * max(w))
    mass, run = sum(w[i] for i in order), Fraction(0)
    for i in order:
        run += w[i]
        if run > Fraction(u) * mass:
            return i, w[i] / mass
    raise AssertionError


def test_choice_against_the_definition_on_exact_weights():
    rng = np.random.default_rng(3)
    for _ in range(400):
        n = int(rng.integers(1, 12))
        w = 2.0 ** -rng.integers(0, 6, n)  # logits ln 2^-j: ties, exact weights
        w /= w.max()
        k, p, m, u = (int(rng.integers(0, n + 2)), float(rng.choice([0.0, 0.3, 0.5, 0.81, 1.0])),
                      float(rng.choice([0.0, 0.3, 0.7, 2.0])), float(rng.integers(0, 1000)) / 1000 + 1e-5)
        want, prob = brute(w, u, k, p, m)
        # logits whose differences are exact multiples of ln 2 round: keep p and m off the borders
        if p == 0.5 or (w.sum() * p) % 0.03125 == 0:
            continue
        got, gp = ref.choose(np.log(w), u, 1.0, k, p, m)
        assert got == want and abs(gp - float(prob)) < 1e-12, (w, u, k, p, m)


def test_choice_special_rows():
    inf, nan = np.inf, np.nan
    assert ref.choose([-inf, nan], 0.5) == (-1, 0.0)
    assert ref.choose([1.0, 3.0, 3.0], 0.5, temperature=0.0) == (1, 1.0)
    assert ref.choose([1.0, nan, 2.0], 0.5, temperature=nan) == (2, 1.0)
    assert ref.choose([inf, 1.0, inf], 0.75) == (2, 0.5)
    assert ref.choose([0.0, 0.0, 0.0, 0.0], 0.6, top_k=2) == (1, 0.5)  # ties go to the lower indices
    assert ref.choose([0.0, 0.0, -inf], 1.0) == (1, 0.5)
    assert ref.choose([0.0, 5.0], 0.99, min_p=7.0)[0] == 1
    assert ref.choose([0.0, 5.0], 0.99, top_p=0.0)[0] == 1
