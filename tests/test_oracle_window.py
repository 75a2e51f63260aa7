"""Pins of oracle/window_oracle.py: against brute force, central differences and a library's attention."""
import numpy as np
import pytest
import torch

from oracle import window_oracle as W


@pytest.mark.parametrize("n,window,sinks", [(1, 1, 0), (7, 3, 0), (7, 3, 2), (9, 100, 4), (6, 1, 6), (8, 2, 100)])
def test_sees(n, window, sinks):
    m = W.sees(n, window, sinks)
    for i in range(n):
        for j in range(n):
            want = j <= i and (j in range(sinks) or i - j < window)
            assert m[i, j] == want


def test_a_window_over_everything_is_causal_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 33, 8))
    t = [torch.from_numpy(x)[None] for x in (q, k, v)]
    want = torch.nn.functional.scaled_dot_product_attention(*t, is_causal=True)[0].numpy()
    assert np.abs(W.attention(q, k, v, 33, 0)[0] - want).max() < 1e-12
    assert np.abs(W.attention(q, k, v, 1, 33)[0] - want).max() < 1e-12


def test_window_of_one_is_the_value_itself():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 12, 4))
    assert np.array_equal(W.attention(q, k, v, 1, 0)[0], v)


def test_gradients_by_differences():
    rng = np.random.default_rng(2)
    q, k, v, do = rng.standard_normal((4, 11, 4))
    args = (4, 2, 0.7)
    grads = W.gradients(q, k, v, do, *args)
    f = lambda *x: float((W.attention(*x, *args)[0] * do).sum())
    for which in range(3):
        for at in [(0, 0), (1, 3), (5, 1), (10, 2)]:
            x = [q.copy(), k.copy(), v.copy()]
            x[which][at] += 1e-5
            up = f(*x)
            x[which][at] -= 2e-5
            assert abs((up - f(*x)) / 2e-5 - grads[which][at]) < 1e-8


def test_rotate_is_complex_multiplication_and_inverts():
    rng = np.random.default_rng(3)
    x, pos = rng.standard_normal((5, 2, 8)), rng.integers(-100, 1000, (5, 2))
    axis, freq = [0, 1, -1, 1], [1.0, 0.3, 0.0, 0.01]
    for halves in (False, True):
        y = W.rotate(x, pos, axis, freq, halves)
        a = [0, 1, 2, 3] if halves else [0, 2, 4, 6]
        b = [4, 5, 6, 7] if halves else [1, 3, 5, 7]
        z = (x[..., a] + 1j * x[..., b]) * np.exp(1j * np.stack(
            [pos[:, max(u, 0)] * f for u, f in zip(axis, freq)], -1))[:, None]
        assert np.abs(y[..., a] - z.real).max() < 1e-12 and np.abs(y[..., b] - z.imag).max() < 1e-12
        assert np.abs(W.rotate(y, pos, axis, freq, halves, inverse=True) - x).max() < 1e-12
