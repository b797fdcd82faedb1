"""Pins of the 4-bit row oracle (not gpu): the code table, rounding against hand-made
ties, the exponent against its definition by search, and the bound on what a row
loses."""
import numpy as np
import pytest

from oracle import quant4 as Q


def test_code_values():
    v = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    assert np.array_equal(Q.code_values(), np.array(v + [-x for x in v]))


@pytest.mark.parametrize("x,code", [
    (0.0, 0), (-0.0, 8), (0.25, 0), (0.26, 1), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (5.01, 7),
    (7.0, 7), (-0.75, 10), (-5.01, 15), (-0.25, 8),
])
def test_ties_go_to_the_even_code(x, code):
    assert Q.nearest_code(x) == code


def test_exponent_is_the_smallest_that_holds_the_block():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((300, 64)) * 2.0 ** rng.integers(-150, 120, (300, 1))
    x[0], x[1, :32], x[2, 5] = 0.0, 7.0, 7.0000001
    _, e = Q.encode(x)
    top = np.abs(x.reshape(300, 2, 32)).max(axis=-1)
    e = e.astype(int)
    assert np.all(top <= 7.0 * 2.0 ** (e - 127.0))
    assert np.all((top > 7.0 * 2.0 ** (e - 128.0)) | (e == 1))
    assert e[0].tolist() == [1, 1] and e[1, 0] == 127


def test_what_a_row_loses():
    """Half a step: a quarter of the power of two below a value, 2^-2 of the unit under it, one unit over 6."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((500, 128)) * np.exp(rng.standard_normal((500, 1)))
    c, e = Q.encode(x)
    unit = np.repeat(2.0 ** (e - 127.0), 32, axis=-1)
    a = np.abs(x) / unit
    half = np.where(a > 6, 1.0, np.where(a < 1, 0.25, 0.25 * 2.0 ** np.floor(np.log2(np.maximum(a, 1)))))
    assert np.all(np.abs(Q.decode(c, e) - x) <= half * unit * (1 + 1e-12))


def test_a_block_that_is_not_finite_is_nan():
    x = np.ones((3, 64))
    x[0, 3], x[1, 40], x[2, 63] = np.nan, np.inf, -np.inf
    c, e = Q.encode(x)
    assert (e == 255).tolist() == [[True, False], [False, True], [False, True]]
    v = Q.decode(c, e)
    assert np.isnan(v[0, :32]).all() and np.array_equal(v[0, 32:], np.ones(32)) and not c[0, :32].any()


def test_pack_round_trip():
    c = np.random.default_rng(4).integers(0, 16, (5, 64)).astype(np.uint8)
    b = Q.pack(c)
    assert b.shape == (5, 32) and b[0, 0] == c[0, 0] + 16 * c[0, 1]
    assert np.array_equal(Q.unpack(b), c)
