"""The oracle of the 8-bit path against things other than itself: exact rational rounding, brute force over exponents,
torch's e4m3 type, and differences for the norms' gradients."""
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import act8


def test_code_values_are_the_ocp_type():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(act8.VALUES, t, equal_nan=True)
    assert act8.VALUES[0x7E] == 448.0 and act8.VALUES[1] == 2.0 ** -9


def test_encode_is_nearest_even_at_every_code_and_midpoint():
    pos = [Fraction(float(v)) for v in act8.VALUES[:127]]
    for c, v in enumerate(pos):
        assert act8.encode(np.array([float(v)]))[0] == c
        if c:
            mid = (pos[c - 1] + v) / 2
            near = (v - mid) / 1024
            got = act8.encode(np.array([float(mid - near), float(mid), float(mid + near), -float(mid)]))
            even = c if c % 2 == 0 else c - 1
            assert list(got) == [c - 1, even, c, even | 0x80], c
    assert list(act8.encode(np.array([np.nan, np.inf, -np.inf]))) == [0x7F, 0x7F, 0xFF]


@pytest.mark.parametrize("p", [-149, -126, -118, -117, -60, -1, 0, 8, 9, 60, 127])
def test_group_exponent_by_brute_force(p):
    for f in (Fraction(1), Fraction(7, 4), Fraction(7, 4) + Fraction(1, 1 << 23), Fraction(2) - Fraction(1, 1 << 23)):
        a = f * Fraction(2) ** p
        if Fraction(float(np.float32(float(a)))) != a:
            continue
        e = next(e for e in range(-126, 200) if a / Fraction(2) ** e <= 448)
        assert act8.group_exponent(np.array([float(a)]))[0] == e
    assert act8.group_exponent(np.array([0.0]))[0] == -126


def test_tiles_hold_every_code_once():
    n, k = 37, 300
    codes = np.random.default_rng(0).integers(0, 256, (n, k)).astype(np.uint8)
    t = act8.tiles(codes)
    assert t.shape == (3, 3, 2, 4, 16, 16)
    assert t[17 // 16, 200 // 128, (200 % 32) // 16, (200 % 128) // 32, 1, 200 % 16] == codes[17, 200]
    flat = t.transpose(0, 4, 1, 3, 2, 5).reshape(48, 384)
    assert np.array_equal(flat[:n, :k], codes) and not flat[n:].any() and not flat[:, k:].any()


def test_values_stay_within_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 300)) * 10.0 ** rng.integers(-6, 6, (5, 1))
    codes, exps = act8.quant_rows(x)
    v = act8.values_rows(codes, exps, 300)
    e = exps[:, :3].astype(int) - 127
    step = np.maximum(np.abs(x) / 16, np.repeat(2.0 ** (e - 10), 128, 1)[:, :300])
    assert np.all(np.abs(v - x) <= step) and not codes[:, 300:].any()


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradients_against_differences(rms):
    rng = np.random.default_rng(2)
    x, dy = rng.standard_normal((4, 23)) * 2 + 0.5, rng.standard_normal((4, 23))
    g, b = 1 + 0.3 * rng.standard_normal(23), rng.standard_normal(23)
    b = np.zeros(23) if rms else b
    loss = lambda x, g, b: float((act8.norm(x, g, b, 1e-5, rms)[0] * dy).sum())
    _, mean, rstd = act8.norm(x, g, b, 1e-5, rms)
    dx, dg, db = act8.norm_bwd(dy, x, g, mean, rstd, rms)
    h = 1e-6
    for d, grad, at in ((rng.standard_normal(x.shape), dx, 0), (rng.standard_normal(23), dg, 1), (rng.standard_normal(23), db, 2)):
        args = [x, g, b]
        hi, lo = list(args), list(args)
        hi[at], lo[at] = args[at] + h * d, args[at] - h * d
        assert abs((loss(*hi) - loss(*lo)) / (2 * h) - (grad * d).sum()) < 1e-7
