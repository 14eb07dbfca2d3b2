"""Pins of the finetuning oracle: closed forms, invariances, and gradients against
differences of the functions that they belong to."""
import numpy as np
import pytest

from oracle import encoder as enc
from oracle import finetune as ft


def window_index(s):
    i = np.arange(s)
    y, x = np.repeat(i, s), np.tile(i, s)
    return (y[:, None] - y[None, :] + s - 1) * (2 * s - 1) + x[:, None] - x[None, :] + s - 1


def test_a_constant_bias_leaves_attention_unchanged():
    r = np.random.default_rng(1)
    x = r.normal(size=(2 * 9, 3 * 2 * 8))
    table = np.full((25, 2), 0.7)
    got = ft.relpos_attention(x, table, window_index(3), 2, 2, 8)["out"]
    assert np.abs(got - enc.attention(x, 2, 9, 2, 8)).max() < 1e-13


def test_two_tokens_in_closed_form():
    # q = 0: the weights are the softmax of the biases, sigma(b_01 - b_00) for key 1
    x = np.zeros((2, 3 * 4))
    x[:, 8:] = [[1, 2, 3, 4], [5, 6, 7, 8]]
    table = np.array([[0.3], [-0.4], [1.1]])
    index = np.array([[1, 0], [2, 1]])
    got = ft.relpos_attention(x, table, index, 1, 1, 4)
    w = 1 / (1 + np.exp(-(0.3 + 0.4)))
    assert np.allclose(got["out"][0], x[0, 8:] + 4 * w, atol=1e-14)
    assert np.allclose(got["lse"][0, 0, 1], np.log(np.exp(1.1) + np.exp(-0.4)), atol=1e-14)


def test_labels_cut_a_window_into_separate_sequences():
    r = np.random.default_rng(2)
    x = r.normal(size=(9, 3 * 4))
    table = r.normal(size=(25, 1))
    idx = window_index(3)
    lab = np.array([[0, 0, 1, 0, 0, 1, 2, 2, -5]])
    got = ft.relpos_attention(x, table, idx, 1, 1, 4, region=lab)["out"]
    for part in ([0, 1, 3, 4], [2, 5], [6, 7]):
        alone = ft.relpos_attention(x[part], table, idx[np.ix_(part, part)], 1, 1, 4)["out"]
        assert np.allclose(got[part], alone, atol=1e-14)
    assert not got[8].any()


def test_rows_without_pairs():
    r = np.random.default_rng(3)
    x, g = r.normal(size=(3, 12)), r.normal(size=(3, 4))
    idx = np.array([[-1, -1, -1], [0, 1, -1], [1, 2, 2]])
    table = np.array([[0.5], [-np.inf], [-np.inf]])
    got = ft.relpos_attention(x, table, idx, 1, 1, 4, dout=g)
    assert not got["out"][[0, 2]].any() and np.all(got["lse"][0, 0, [0, 2]] == -np.inf)
    assert np.array_equal(got["out"][1], x[0, 8:]) and not got["dtable"].any()


@pytest.mark.parametrize("seed", [4, 5])
def test_attention_gradients_against_differences(seed):
    r = np.random.default_rng(seed)
    n, H, hd, idx = 3, 2, 4, window_index(2)
    lab = np.array([[0, 0, 1, 1], [0, -1, 0, 0]])
    x, table = r.normal(size=(n * 4, 3 * H * hd)), r.normal(size=(9, H))
    g = r.normal(size=(n * 4, H * hd))
    f = lambda x, t: (ft.relpos_attention(x, t, idx, n, H, hd, region=lab)["out"] * g).sum()
    got = ft.relpos_attention(x, table, idx, n, H, hd, region=lab, dout=g)
    for _ in range(4):
        dx, dt = r.normal(size=x.shape), r.normal(size=table.shape)
        h = 1e-5
        num = (f(x + h * dx, table + h * dt) - f(x - h * dx, table - h * dt)) / (2 * h)
        ana = (got["dqkv"] * dx).sum() + (got["dtable"] * dt).sum()
        assert abs(num - ana) < 1e-8 * (1 + abs(ana))


def test_distill_closed_forms():
    # one teacher entry: its q is 1, the loss t^2 times the cross entropy of that class
    z = np.array([[0.5, -1.0, 2.0]])
    loss, d = ft.distill(z, np.array([[2]]), np.array([[9.0]]), 2.0, np.array([3.0]))
    p = np.exp(z / 2) / np.exp(z / 2).sum()
    assert np.allclose(loss, -4 * np.log(p[0, 2])) and np.allclose(d, 6 * (p - [[0, 0, 1]]))
    # the teacher's logits are the student's: nothing to learn, whatever their common shift
    loss, d = ft.distill(z, np.array([[1, 2, 0]]), z[:, [1, 2, 0]] + 5, 1.5, np.ones(1))
    assert np.allclose(loss, 0, atol=1e-15) and np.allclose(d, 0, atol=1e-15)
    # a class named twice has both shares; no valid id, no loss
    one = ft.distill(z, np.array([[1, 1]]), np.array([[0.3, 0.3]]), 1.0, np.ones(1))
    two = ft.distill(z, np.array([[1, 7]]), np.array([[0.3, 4.0]]), 1.0, np.ones(1))
    assert np.allclose(one[1], two[1]) and np.allclose(one[0] + np.log(2), two[0])
    none = ft.distill(z, np.array([[-1, 3]]), np.array([[0.3, 4.0]]), 1.0, np.ones(1))
    assert not none[0].any() and not none[1].any()


def test_distill_gradient_against_differences():
    r = np.random.default_rng(6)
    z, t = r.normal(size=(3, 11)), r.normal(size=(3, 5))
    ids = np.array([[1, 5, 9, 0, 3], [2, 2, -1, 10, 4], [7, -1, -1, 12, 7]])
    g = r.normal(size=3)
    d = ft.distill(z, ids, t, 3.0, g)[1]
    for _ in range(4):
        dz = r.normal(size=z.shape)
        f = lambda h: (ft.distill(z + h * dz, ids, t, 3.0) * g).sum()
        assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - (d * dz).sum()) < 1e-8


def test_gradients_of_the_step_against_differences():
    """The operators behind each other: the loss's central differences in directions of the
    table and of qkv against the oracle's gradients."""
    r = np.random.default_rng(5)
    idx, nb = np.clip(np.arange(9)[None, :] - np.arange(9)[:, None] + 3, 0, 5), 6
    H, hd, V, n_seq = 2, 4, 11, 2
    x, t = r.normal(0, 1, (n_seq * 9, 3 * H * hd)), r.normal(0, 0.5, (nb, H))
    W = r.normal(0, 0.4, (V, H * hd))
    ids = np.stack([r.permutation(V)[:3] for _ in range(n_seq * 9)])
    top = r.normal(0, 2, ids.shape)
    g = np.ones(n_seq * 9)

    def loss(x, t):
        out = ft.relpos_attention(x, t, idx, n_seq, H, hd)["out"]
        return ft.distill(out @ W.T, ids, top, 2.0).sum()
    out = ft.relpos_attention(x, t, idx, n_seq, H, hd)["out"]
    dz = ft.distill(out @ W.T, ids, top, 2.0, g)[1]
    grads = ft.relpos_attention(x, t, idx, n_seq, H, hd, dout=dz @ W)
    eps = 1e-5
    for _ in range(4):
        ux, ut = r.normal(0, 1, x.shape), r.normal(0, 1, t.shape)
        diff = (loss(x + eps * ux, t + eps * ut) - loss(x - eps * ux, t - eps * ut)) / (2 * eps)
        exact = (grads["dqkv"] * ux).sum() + (grads["dtable"] * ut).sum()
        # the third derivative's term, eps^2 of values of order 10, and the loss's own 2^-53
        # over eps
        assert abs(diff - exact) <= 1e-7 * max(1.0, abs(exact)) + 1e-8
