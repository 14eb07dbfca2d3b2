"""Pins of the 8-bit oracle: closed forms, invariances and a brute-force sum."""
import numpy as np

import oracle
from oracle import encoder as enc
from oracle import quant


def test_codes_in_closed_form():
    # a largest value of 127: the codes are the values, rounded to even halfway
    u = np.array([[127.0, 0.5, 1.5, -2.5, -0.5, 3.49, -126.51, 0.0]])
    q, scale = quant.codes(u)
    assert q.tolist() == [[127, 0, 2, -2, 0, 3, -127, 0]] and scale.tolist() == [1.0]
    # any positive factor leaves the codes and multiplies the scale; a sign turns them
    for f in (2.0 ** -20, 3.0, 1e30):
        qf, sf = quant.codes(u * f)
        assert (qf == q).all() and np.allclose(sf, f, rtol=1e-15)
    assert (quant.codes(-u)[0] == -q).all()


def test_codes_of_empty_and_unfinished_rows():
    q, scale = quant.codes(np.array([[0.0, 0.0], [np.nan, 1.0], [np.inf, 1.0], [1.0, -1.0]]))
    assert q.tolist() == [[0, 0], [0, 0], [0, 0], [127, -127]]
    assert scale[0] == 0 and np.isnan(scale[1:3]).all() and scale[3] == 1 / 127


def test_values_are_within_half_a_step():
    r = np.random.default_rng(1)
    u = r.normal(size=(50, 33)) * np.exp(r.normal(size=(50, 1)) * 5)
    q, scale = quant.codes(u)
    assert np.abs(q).max(1).tolist() == [127] * 50
    assert (np.abs(q * scale[:, None] - u) <= scale[:, None] * (0.5 + 1e-12)).all()


def test_rms_against_its_definition():
    r = np.random.default_rng(2)
    s, g = r.normal(size=(40, 29)) * 3, r.normal(size=29)
    n = s / np.sqrt((s ** 2).mean(1, keepdims=True) + 0.3) * g
    q, scale = quant.rms(s, g, 0.3)
    q1, scale1 = quant.codes(n)
    assert (q == q1).all() and np.allclose(scale, scale1, rtol=1e-14)
    # one value: s / |s| without eps
    q, scale = quant.rms(np.array([[-3.0]]), np.array([2.0]), 0.0)
    assert q[0, 0] == -127 and np.allclose(scale, 2 / 127, rtol=1e-15)
    q, scale = quant.rms(np.zeros((1, 4)), np.ones(4), 0.0)
    assert not q.any() and scale[0] == 0


def test_layer_norm_against_the_encoder_oracle():
    r = np.random.default_rng(3)
    x, y, g, b = r.normal(size=(40, 24)), r.normal(size=(40, 24)), r.normal(size=24), r.normal(size=24)
    q, scale = quant.layer(x + y, g, b, 1e-6)
    q1, scale1 = quant.codes(enc.add_layernorm(x, y, g, b, 1e-6)[1])
    assert (q == q1).all() and np.allclose(scale, scale1, rtol=1e-13)


def test_linear_against_loops_and_the_float_oracle():
    r = np.random.default_rng(4)
    M, N, K = 5, 32, 48
    X, W = r.integers(-128, 128, (M, K)), r.integers(-128, 128, (N, K))
    xs, ws, b = r.random(M), r.random(N), r.normal(size=N)
    mask = r.integers(0, 2, (2, 3)).astype(np.uint8)
    Wk = quant.keep(W, mask, 16, 16)
    Y, A = quant.linear(X, xs, Wk, ws, b)
    for m in range(M):
        for n in range(N):
            t = sum(int(X[m, k]) * int(W[n, k]) for k in range(K) if mask[n // 16, k // 16])
            assert abs(Y[m, n] - (t * xs[m] * ws[n] + b[n])) <= 1e-13 * (abs(t) + 1)
            assert abs(A[m, n] - abs(t) * xs[m] * ws[n]) <= 1e-13 * (abs(t) + 1)
    # whole numbers in float32 and scales of one: the block-sparse oracle
    f = lambda a: a.astype(np.float32)
    want = oracle.linear(f(X), f(W), "f32", 16, 16, mask, f(b), gelu=True)
    got = quant.linear(X, np.ones(M), Wk, np.ones(N), f(b), gelu=True)[0]
    assert np.abs(got - want).max() <= 1e-12 * np.abs(want).max()
