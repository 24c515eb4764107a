"""Pins of the oracle's gated block and 8-bit products (CPU): finite differences, closed forms, brute force."""
import math

import numpy as np
import pytest

from oracle import lrd_oracle as o

ACTS = [o.ACT_SILU, o.ACT_GELU, o.ACT_GELU_TANH]


def _case(M, K, N, seed):
    g = np.random.default_rng(seed)
    return g.standard_normal((M, K)), g.standard_normal((2 * N, K)) * K ** -0.5, g.standard_normal(2 * N) * 0.1, g.standard_normal((M, N))


@pytest.mark.parametrize("act", ACTS)
def test_activation_closed_forms_and_derivative(act):
    x = np.linspace(-9.0, 9.0, 181)
    v, d = o.activation(x, act)
    want = [lambda t: t / (1.0 + math.exp(-t)), lambda t: 0.5 * t * (1.0 + math.erf(t / math.sqrt(2.0))),
            lambda t: 0.5 * t * (1.0 + math.tanh(math.sqrt(2.0 / math.pi) * (t + 0.044715 * t ** 3)))][act]
    assert np.abs(v - [want(t) for t in x]).max() <= 1e-14 * 9
    h = 1e-5                                             # central difference: h^2 / 6 |f'''| (below 2) + 2^-53 |f| / h
    assert np.abs((o.activation(x + h, act)[0] - o.activation(x - h, act)[0]) / (2 * h) - d).max() <= 2 * h * h / 6 + 9 * 2.0 ** -52 / h
    far_v, far_d = o.activation(np.array([-500.0, 500.0]), act)
    assert far_v[0] == 0 or abs(far_v[0]) < 1e-200
    assert far_v[1] == 500.0 and far_d[1] == 1.0 and abs(far_d[0]) < 1e-200


@pytest.mark.parametrize("act", ACTS)
def test_block_gradients_against_differences(act):
    M, K, N = 4, 5, 3
    X, W, b, dH = _case(M, K, N, 11 + act)
    H, P = o.glu_fwd(X, W, b, act)
    for m in range(M):                                   # brute force
        for n in range(N):
            g = sum(X[m, k] * W[n, k] for k in range(K)) + b[n]
            u = sum(X[m, k] * W[N + n, k] for k in range(K)) + b[N + n]
            assert abs(H[m, n] - o.activation(g, act)[0] * u) <= 1e-13
    grads = o.glu_bwd(dH, X, W, P, act)
    loss = lambda X, W, b: float((o.glu_fwd(X, W, b, act)[0] * dH).sum())
    h = 1e-5
    for name, t in (("dX", X), ("dW", W), ("db", b)):
        for at in np.ndindex(t.shape):
            keep = t[at]
            t[at] = keep + h
            up = loss(X, W, b)
            t[at] = keep - h
            down = loss(X, W, b)
            t[at] = keep
            assert abs((up - down) / (2 * h) - grads[name][at]) <= 1e-7, (name, at)


def test_quantized_rows():
    X = np.array([[127.0, -127.0, 63.5, 0.5, 1.5, -2.5, -0.5, 0.0], [0.0] * 8, [1.0, -2.0, 0.25, 3.0, 0.0, -3.0, 1.5, 0.1],
                  [np.inf, 1, 2, 3, 4, 5, 6, 7], [np.nan, 1, 2, 3, 4, 5, 6, 7]])
    q, s = o.i8_quantize(X)
    assert s[0] == 1.0 and list(q[0]) == [127, -127, 64, 0, 2, -2, 0, 0]         # ties to even
    assert s[1] == 0.0 and not q[1].any()
    assert s[2] == np.float32(3.0) * np.float32(1.0 / 127.0) and q[2, 3] == 127 and q[2, 5] == -127
    assert np.abs(q[2] * float(s[2]) - X[2]).max() <= float(s[2]) * 0.5 * (1 + 1e-6)
    assert np.isnan(s[3:]).all() and not q[3:].any()


def test_products_of_8_bit_integers():
    g = np.random.default_rng(3)
    a, w = g.integers(-128, 128, (3, 7)), g.integers(-128, 128, (4, 7))
    s, t, b = g.random(3), g.random(4), g.standard_normal(4)
    y = o.i8_product(a, s, w, t, b)
    for i in range(3):
        for j in range(4):
            assert abs(y[i, j] - (s[i] * t[j] * int(sum(int(p) * int(q) for p, q in zip(a[i], w[j]))) + b[j])) <= 1e-9
