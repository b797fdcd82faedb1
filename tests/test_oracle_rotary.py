"""Pins of the rotary oracle (not gpu), and the library's host frequencies against it."""
import math

import numpy as np
import pytest

import paper_2603_19610_amd as pv
from oracle import rope as R1
from oracle import rotary as R

SCALINGS = [
    dict(), dict(scaling="linear", factor=4.0), dict(scaling="parts", factor=8.0, orig_ctx=8192.0, alpha=1.0, beta=4.0),
    dict(scaling="yarn", factor=4.0, orig_ctx=32768.0, alpha=1.0, beta=32.0),
    dict(scaling="yarn", factor=40.0, orig_ctx=128.0, alpha=1.0, beta=32.0),      # every ramp end clamped
    dict(scaling="yarn", factor=2.0, orig_ctx=4096.0, alpha=7.9, beta=8.0),       # a ramp of a pair or none
]


@pytest.mark.parametrize("rot_dim", [8, 32, 64, 128, 256])
@pytest.mark.parametrize("kw", SCALINGS, ids=lambda k: f"{k.get('scaling')}{k.get('orig_ctx', '')}")
@pytest.mark.parametrize("base", [1e4, 1e6])
def test_host_frequencies(rot_dim, kw, base):
    """Off by the roundings of one exponential of an argument of up to ln(base) <= 14 (14 halves of a last place and
    its own), and a handful of products: under 32 of 2^-53."""
    f = np.array(pv.Rotary(rot_dim=rot_dim, base=base, **kw).frequencies())
    w = R.frequencies(rot_dim, base, **kw)
    assert f.shape == (rot_dim // 2,) and np.all(np.abs(f / w - 1) <= 32 * 2.0 ** -53)


def test_parts_and_yarn_keep_fast_pairs_and_interpolate_slow_ones():
    for kw in SCALINGS[2:4]:
        f, w = R.frequencies(128, 1e6, **kw), R.frequencies(128, 1e6)
        ratio = w / f
        assert ratio[0] == 1.0 and abs(ratio[-1] - kw["factor"]) < 1e-12 and np.all(np.diff(ratio) >= -1e-12)
        turns = kw["orig_ctx"] * w / (2 * math.pi)
        assert np.allclose(ratio[turns > 2 * kw["beta"]], 1.0)
        assert np.allclose(ratio[turns < 0.5 * kw["alpha"]], kw["factor"])


def test_half_layout_is_the_verify_rows_rotation():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((5, 3, 64)), np.array([0, 1, 77, 6432, 131000])
    want = R1.rotate(x, R1.pair_positions(pos, 64)[:, None], 1e6)
    assert np.allclose(R.rotate(x, pos, R.frequencies(64, 1e6)), want, rtol=0, atol=1e-9)
    p3, sec = np.stack([pos, pos + 3, pos * 0]), (8, 12, 12)
    want = R1.rotate(x, R1.pair_positions(p3, 64, sec)[:, None], 1e6)
    assert np.allclose(R.rotate(x, p3, R.frequencies(64, 1e6), sections=sec), want, rtol=0, atol=1e-9)


def test_interleaved_is_half_with_its_elements_permuted():
    rng = np.random.default_rng(2)
    x, pos, f = rng.standard_normal((4, 2, 96)), np.array([3, 0, 900, 7]), R.frequencies(64, 1e4)
    order = np.concatenate([np.arange(0, 64, 2), np.arange(1, 64, 2), np.arange(64, 96)])
    half = R.rotate(x[..., order], pos, f)
    inter = R.rotate(x, pos, f, layout="interleaved")
    assert np.allclose(inter[..., order], half, rtol=0, atol=1e-12)
    assert np.array_equal(inter[..., 64:], x[..., 64:])


def test_scores_depend_on_distance_alone():
    rng = np.random.default_rng(3)
    q, k, f = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64)), R.frequencies(64, 1e4)
    s = [(R.rotate(q, np.array([a + 9]), f) * R.rotate(k, np.array([a]), f)).sum() for a in (0, 5, 4000)]
    assert np.allclose(s, s[0], atol=1e-9)


def test_put_rows_skips_padding():
    c = R.put_rows(np.zeros((2, 1, 4, 1)), [5, -1, 0], np.arange(1, 4).reshape(3, 1, 1))
    assert c[1, 0, 1, 0] == 1 and c[0, 0, 0, 0] == 3 and c.sum() == 4


@pytest.mark.parametrize("kw,err", [
    (dict(layout="other"), ValueError), (dict(scaling="other"), ValueError), (dict(sections=(1, 2)), ValueError),
    (dict(rot_dim=12), pv.PvlmError), (dict(rot_dim=0), pv.PvlmError), (dict(rot_dim=264), ValueError),
    (dict(base=1.0), pv.PvlmError), (dict(base=math.nan), pv.PvlmError), (dict(mscale=0.0), pv.PvlmError),
    (dict(scaling="linear", factor=0.0), pv.PvlmError), (dict(scaling="parts", factor=2.0), pv.PvlmError),
    (dict(scaling="parts", factor=2.0, orig_ctx=64.0, alpha=4.0, beta=4.0), pv.PvlmError),
    (dict(scaling="yarn", factor=2.0, orig_ctx=math.inf, alpha=1.0, beta=4.0), pv.PvlmError),
])
def test_parameters_without_frequencies_are_refused(kw, err):
    with pytest.raises(err):
        pv.Rotary(**{**dict(rot_dim=64, base=1e4), **kw})
