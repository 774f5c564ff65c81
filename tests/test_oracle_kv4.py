"""The 4-bit format's oracle against its own definition."""
import numpy as np

from oracle import gemv as og
from oracle import kv4


def test_exponents_by_search_and_in_closed_form():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((300, 32)) * np.exp2(rng.integers(-140, 127, (300, 1)))
    x[:40] = 0
    x[np.arange(40), 3] = np.exp2(np.arange(-20, 20.)) * 7      # the border itself
    x[40, :] = 0
    assert np.array_equal(kv4.exponents(x), kv4.exponents_fast(x))


def test_rounding_goes_to_the_nearest_code_and_ties_to_even():
    a = np.linspace(0, 7, 7 * 64 + 1)
    got = kv4.round_to_grid(a)
    near = np.abs(a[:, None] - kv4.GRID).min(1)
    assert np.array_equal(np.abs(a - got), near)
    for x, want in ((0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2), (3.5, 4), (5, 4), (7, 6)):
        assert kv4.round_to_grid(np.array([x]))[0] == want


def test_every_value_is_within_half_a_step_and_bf16():
    rng = np.random.default_rng(1)
    u = og.f32_to_bf16((rng.standard_normal((500, 128)) * np.exp2(rng.integers(-100, 100, (500, 1))))
                       .astype(np.float32))
    x = og.bf16_to_f32(u).astype(np.float64)
    y = kv4.stored(u)
    step = np.ldexp(1.0, kv4.exponents_fast(x.reshape(500, 4, 32)))[..., None]
    a = np.abs(x.reshape(500, 4, 32)) / step
    width = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert np.all(np.abs(x - y).reshape(500, 4, 32) <= width / 2 * step)
    assert np.array_equal(og.bf16_to_f32(og.f32_to_bf16(y.astype(np.float32))), y)


def test_special_groups():
    u = np.zeros((3, 128), np.uint16)
    u[0, 5] = 0x7f80          # +inf in group 0
    u[1, 127] = 0x7fc1        # NaN in group 3
    u[2, 40] = 0x7f7f         # the largest finite value
    y = kv4.stored(u)
    assert np.all(np.isnan(y[0, :32])) and np.all(y[0, 32:] == 0)
    assert np.all(np.isnan(y[1, 96:])) and np.all(y[1, :96] == 0)
    assert y[2, 40] == 6 * 2.0 ** 125
