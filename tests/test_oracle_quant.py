"""Pins of the 8-bit row oracle (not gpu): the code table against torch's e4m3
type, rounding against torch's cast and hand-made ties, the exponent against
its definition by search, and the bound on what a row loses."""
import numpy as np
import pytest
import torch

from oracle import quant as Q


def test_code_values_are_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(Q.code_values(), t, equal_nan=True)


def test_nearest_code_is_torchs_cast():
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 6, 20000),
                        np.array([0.0, -0.0, 448, -448, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10])])
    x = x.astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(Q.nearest_code(x), want)


@pytest.mark.parametrize("x,code", [
    (17.0, 0x58), (19.0, 0x5a),              # halfway between 16, 18 and 18, 20: the even code
    (2.0 ** -10, 0x00), (3 * 2.0 ** -10, 0x02), (-2.0 ** -10, 0x80),
    (448.0, 0x7e), (1.0, 0x38), (-1.0, 0xb8),
])
def test_ties_and_ends(x, code):
    assert int(Q.nearest_code(x)) == code


def test_exponent_is_the_smallest_that_holds_the_row():
    rng = np.random.default_rng(2)
    tops = np.concatenate([2.0 ** rng.uniform(-149, 127, 300), 448.0 * 2.0 ** np.arange(-126.0, 119.0),
                           [0.0, 448.0, np.nextafter(448.0, 500), 3.3e38]])
    e = Q.exponent(tops)
    assert np.all(tops <= 448.0 * 2.0 ** (e - 127.0))
    assert np.all((e == 1) | (tops > 448.0 * 2.0 ** (e - 128.0)))
    assert e.min() >= 1 and e.max() <= 254


def test_rows_round_within_half_a_step_and_keep_nan():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((200, 64)) * 2.0 ** rng.integers(-60, 60, (200, 1))
    x[3, 5], x[4, 6], x[5, 7] = np.nan, np.inf, -np.inf
    x[6] = 0.0
    c, e = Q.encode(x)
    y = Q.decode(c, e)
    bad = ~np.isfinite(x)
    assert np.array_equal(np.isnan(y), bad) and np.all(c[bad] == 0x7f)
    step = np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * 2.0 ** (e[:, None] - 127.0))
    assert np.all((np.abs(y - x) <= step)[~bad])
    assert e[6] == 1 and not c[6].any()
    # encoding what a row stands for gives a row that stands for the same
    assert np.array_equal(Q.decode(*Q.encode(y)), y, equal_nan=True)


def test_a_planted_slip_is_seen(monkeypatch):
    x = np.array([[1.0, 500.0, -3.0]])
    good = Q.encode(x)
    monkeypatch.setattr(Q, "exponent", lambda top: np.full(np.shape(top), 127))
    assert not np.array_equal(Q.encode(x)[1], good[1])


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(4).standard_normal(5000) * 10.0
    assert np.array_equal(Q.bf16(x), torch.from_numpy(x).to(torch.bfloat16).double().numpy())
