"""The oracle of the rotation by position against complex numbers, against differences, and by hand."""
import numpy as np
import pytest

from oracle import seq_oracle as O


def test_by_hand():
    x = np.array([[[[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]]]])
    z = O.rotary(x, [[1], [3]], [np.pi / 2, np.pi / 3], (1, 1))[0]["z"][0, 0, 0]   # pairs (0, 2) by a quarter, (1, 3) by a half
    assert np.allclose(z, [-3, -2, 1, -4, 5, 6])
    z = O.rotary(x, [[1], [3]], [np.pi / 2, np.pi / 3], (1, 1), interleaved=True)[0]["z"][0, 0, 0]   # pairs (0, 1), (2, 3)
    assert np.allclose(z, [-2, 1, -3, -4, 5, 6])


@pytest.mark.parametrize("interleaved", [False, True])
def test_against_complex_numbers(interleaved):
    g = np.random.default_rng(1)
    x, positions, freqs = g.standard_normal((2, 3, 5, 12)), g.integers(-50, 50, (2, 2, 5)), g.uniform(0, 2, 4)
    z = O.rotary(x, positions, freqs, (3, 1), interleaved=interleaved)[0]["z"]
    lo, hi = (slice(0, 8, 2), slice(1, 8, 2)) if interleaved else (slice(0, 4), slice(4, 8))
    for b in range(2):
        for t in range(5):
            turned = (x[b, :, t, lo] + 1j * x[b, :, t, hi]) * np.exp(1j * np.array([positions[b, 0, t]] * 3 + [positions[b, 1, t]]) * freqs)
            assert np.allclose(z[b, :, t, lo], turned.real) and np.allclose(z[b, :, t, hi], turned.imag)
    assert np.array_equal(z[..., 8:], x[..., 8:])


@pytest.mark.parametrize("normed", [False, True])
def test_gradients_against_differences(normed):
    g = np.random.default_rng(2)
    x, dz, positions, freqs = g.standard_normal((2, 3, 4, 8)), g.standard_normal((2, 3, 4, 8)), g.integers(0, 9, (1, 4)), g.uniform(0, 2, 3)
    w = g.uniform(0.5, 1.5, 8) if normed else None
    of = lambda x, w: (O.rotary(x, positions, freqs, (3,), w, 0.1)[0]["z"] * dz).sum()
    res = O.rotary(x, positions, freqs, (3,), w, 0.1, dz=dz)[0]
    step = g.standard_normal(x.shape)
    assert abs((of(x + 1e-5 * step, w) - of(x - 1e-5 * step, w)) / 2e-5 - (res["dx"] * step).sum()) < 1e-7
    if normed:
        step = g.standard_normal(8)
        assert abs((of(x, w + 1e-5 * step) - of(x, w - 1e-5 * step)) / 2e-5 - (res["dw"] * step).sum()) < 1e-7
