"""The float64 oracle of layer norm, its gradient and 8-bit layers (CPU): worked
values, brute force in pure Python, and gradients against differences."""
import math

import numpy as np
import pytest

from oracle import norm_q8_ref as Q


def test_layer_norm_worked_row():
    # 1, 3: mean 2, variance 1; with eps = 3 the deviations are halved
    y, mean, rstd = Q.layer_norm_ref([[1.0, 3.0]], [2.0, 4.0], [10.0, 20.0], eps=3.0)
    assert mean[0] == 2.0 and rstd[0] == 0.5
    assert y.tolist() == [[9.0, 22.0]]


def test_layer_norm_brute_force():
    g = np.random.default_rng(0)
    x, w, b = g.standard_normal((3, 7)) + 5, g.standard_normal(7), g.standard_normal(7)
    y, _, _ = Q.layer_norm_ref(x, w, b, 1e-5)
    for r in range(3):
        mu = math.fsum(x[r]) / 7
        var = math.fsum((v - mu) ** 2 for v in x[r]) / 7
        for c in range(7):
            assert abs(y[r, c] - ((x[r, c] - mu) / math.sqrt(var + 1e-5) * w[c] + b[c])) < 1e-12


def test_layer_norm_single_channel_is_beta():
    y, _, rstd = Q.layer_norm_ref([[3.0], [-7.0]], [5.0], [0.25], 1e-4)
    assert (y == 0.25).all() and np.allclose(rstd, 100.0)


@pytest.mark.parametrize("C", [1, 2, 5])
def test_layer_norm_gradient_against_differences(C):
    g = np.random.default_rng(C)
    x, w, b = g.standard_normal((4, C)), 1 + 0.2 * g.standard_normal(C), g.standard_normal(C)
    dy = g.standard_normal((4, C))
    loss = lambda x, w, b: float((Q.layer_norm_ref(x, w, b, 1e-2)[0] * dy).sum())  # noqa: E731
    _, mean, rstd = Q.layer_norm_ref(x, w, b, 1e-2)
    grads = Q.layer_norm_backward_ref(dy, x, mean, rstd, w)
    step = 1e-5
    for which, grad in enumerate(grads):
        args = [x, w, b]
        for i in np.ndindex(args[which].shape):
            up, dn = [a.copy() for a in args], [a.copy() for a in args]
            up[which][i] += step
            dn[which][i] -= step
            assert abs((loss(*up) - loss(*dn)) / (2 * step) - grad[i]) < 1e-6, (which, i)


def test_quantize_rows_worked():
    # 63.5 and 62.5 are ties: to the even neighbour
    q, s = Q.quantize_rows_ref([[254.0, 127.0, -125.0, 0.0, 254.0], [0.0] * 5])
    assert q.tolist() == [[127, 64, -62, 0, 127], [0] * 5]
    assert s.tolist() == [2.0, 0.0]


def test_quantize_rows_not_finite_and_tiny():
    q, s = Q.quantize_rows_ref([[1.0, np.nan], [np.inf, 1.0], [2.0 ** -119, 0.0], [2.0 ** -118, 0.0]])
    assert np.isnan(s[:2]).all() and s[2] == 0 and s[3] > 0
    assert q.tolist() == [[0, 0], [0, 0], [0, 0], [127, 0]]


def test_quantize_rows_error_is_half_a_step():
    x = np.random.default_rng(3).standard_normal((6, 40))
    q, s = Q.quantize_rows_ref(x)
    assert np.abs(q).max() == 127
    assert (np.abs(q * s[:, None] - x) <= s[:, None] * (0.5 + 1e-12)).all()


def test_linear_q8_worked():
    y = Q.linear_q8_ref([[1, -2], [127, 127]], [0.5, 2.0], [[3, 4], [-128, 127], [0, 1]],
                        [1.0, 0.25, 8.0], bias=[0.0, 1.0, 2.0], residual=[[1, 1, 1], [0, 0, 0]])
    assert y.tolist() == [[0.5 * -5 + 1, 0.5 * -382 * 0.25 + 2, 0.5 * -2 * 8 + 3],
                          [2.0 * 889, 2 * -127 * 0.25 + 1, 2 * 127 * 8 + 2]]
    z = Q.linear_q8_ref([[1]], [1.0], [[1]], [1.0], gelu=True)
    assert abs(z[0, 0] - 0.8413447460685429) < 1e-15
