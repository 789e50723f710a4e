"""The oracle of 4 bits and rotation against what their definitions imply."""
import math

import numpy as np
import pytest

from oracle import cache4_oracle as O


def _values(block):
    codes, e = O.quantise(block)
    return np.array([O.value(c, e) for c in codes]), e


@pytest.mark.parametrize("power", [-60, -3, 0, 1, 40])
def test_values_of_the_format_are_kept(power):
    x = np.array([m * s for m in O.MAGNITUDES for s in (1, -1)] * 2) * 2.0 ** power
    got, e = _values(x)
    assert np.array_equal(got, x) and e == 127 + power
    assert np.array_equal(np.signbit(got), np.signbit(x))


def test_each_element_is_off_by_half_a_step_at_most():
    rng = np.random.default_rng(0)
    for _ in range(200):
        x = rng.standard_normal(32) * 10.0 ** rng.uniform(-6, 6)
        got, e = _values(x)
        size = np.abs(x) / 2.0 ** (e - 127)
        step = np.where(size <= 2, 0.25, np.where(size <= 4, 0.5, 1.0))
        assert (np.abs(got - x) <= step * 2.0 ** (e - 127)).all()
        assert 3.5 < size.max() <= 7


def test_the_scale_is_the_least_for_seven():
    block = lambda top: [top] + [0.1] * 31  # noqa: E731
    assert _values(block(7.0))[1] == 127
    assert _values(block(np.nextafter(7.0, 8)))[1] == 128
    assert _values(block(3.5))[1] == 126 and _values(block(np.nextafter(3.5, 4)))[1] == 127
    assert _values([0.0] * 32)[1] == 1
    assert _values(block(1e-45))[1] > 1 and _values([1e-45] * 32)[1] == 1
    got, e = _values(block(3.4028234663852886e38))     # the largest number: 6 scales stay finite in fp32
    assert e == 252 and got[0] == 6 * 2.0 ** 125 and np.isfinite(np.float32(got[0]))


@pytest.mark.parametrize("x,want", [(0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2), (3.5, 4), (5, 4), (7, 6),
                                    (-0.25, 0), (-5, -4)])
def test_ties_go_to_the_even_code(x, want):
    assert _values([6.0] * 31 + [x])[0][31] == want


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_blocks_that_are_not_finite(bad):
    assert O.quantise([1.0] * 31 + [bad]) == (None, 255)
    assert math.isnan(O.value(3, 255))


@pytest.mark.parametrize("interleaved", [False, True])
def test_a_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, angle = rng.standard_normal(48), rng.uniform(0, 7, 16)
    got = O.rotate(x, np.cos(angle), np.sin(angle), 32, interleaved).astype(np.float64)
    a, b = (slice(0, 32, 2), slice(1, 32, 2)) if interleaved else (slice(0, 16), slice(16, 32))
    z = (x[a] + 1j * x[b]) * np.exp(1j * angle)
    # inputs and tables rounded (two of 2^-24 a product), two products and a sum
    size = np.abs(x[a]) + np.abs(x[b])
    assert (np.abs(got[a] - z.real) <= 4 * 2.0 ** -24 * size).all()
    assert (np.abs(got[b] - z.imag) <= 4 * 2.0 ** -24 * size).all()
    assert np.array_equal(got[32:], x[32:].astype(np.float32))


def test_sections_take_their_own_positions():
    table = {"cos": np.zeros((9, 8), np.float32), "sin": np.zeros((9, 8), np.float32), "interleaved": False}
    table["cos"][:] = np.arange(9)[:, None]
    x = np.concatenate([np.ones(8), np.zeros(8)])[None, None]
    assert O.turn(x, table, [[2]])[0, 0, :8].tolist() == [2] * 8
    assert O.turn(x, {**table, "sections": (4, 0, 4)}, [[2, 5, 99]])[0, 0, :8].tolist() == [2] * 4 + [8] * 4
    assert O.turn(x, table, [[-3]])[0, 0, :8].tolist() == [0] * 8
