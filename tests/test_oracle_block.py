"""The oracle of the selective state space block against what defines it: sums written out, differences of the forward functions."""
import numpy as np
import pytest

from oracle import block as O
from oracle import sequence as S


def rand(rng, *shape):
    return rng.standard_normal(shape)


def test_causal_conv_is_the_sum_over_the_line():
    rng = np.random.default_rng(1)
    x, w, bias, before = rand(rng, 2, 6, 3), rand(rng, 3, 4), rand(rng, 3), rand(rng, 2, 3, 3)
    y, final = O.causal_conv(x, w, bias, "none", [6, 2], before)
    for b, n in enumerate((6, 2)):
        row = lambda t: x[b, t] if t >= 0 else before[b, 3 + t]  # noqa: E731
        for t in range(6):
            want = bias + sum(w[:, j] * row(t - 3 + j) for j in range(4)) if t < n else np.zeros(3)
            np.testing.assert_allclose(y[b, t], want, rtol=1e-13, atol=1e-14)
        np.testing.assert_array_equal(final[b], np.stack([row(n - 3 + j) for j in range(3)]))


def test_scan_is_the_sum_over_pairs():
    rng = np.random.default_rng(2)
    B, T, D, N, G = 2, 6, 4, 3, 2
    x, dt, b, c, gate = rand(rng, B, T, D), rand(rng, B, T, D), rand(rng, B, T, G, N), rand(rng, B, T, G, N), rand(rng, B, T, D)
    A, skip, bias, h0 = -rng.uniform(0.1, 2, (D, N)), rand(rng, D), rand(rng, D), rand(rng, B, D, N)
    lengths = [6, 3]
    y, final = O.selective_scan(x, dt, A, b, c, skip, gate, bias, True, lengths, h0)
    delta = np.log(1 + np.exp(dt + bias))
    for i in range(B):
        for d in range(D):
            g = d // 2
            for n_t in range(T + 1):  # state behind n_t tokens
                if n_t > lengths[i]:
                    continue
                h = np.exp(A[d] * delta[i, :n_t, d].sum()) * h0[i, d]
                for s in range(n_t):
                    h = h + np.exp(A[d] * delta[i, s + 1:n_t, d].sum()) * delta[i, s, d] * x[i, s, d] * b[i, s, g]
                if n_t == lengths[i]:
                    np.testing.assert_allclose(final[i, d], h, rtol=1e-12)
                if n_t:
                    z = gate[i, n_t - 1, d]
                    want = (c[i, n_t - 1, g] @ h + skip[d] * x[i, n_t - 1, d]) * z / (1 + np.exp(-z))
                    np.testing.assert_allclose(y[i, n_t - 1, d], want, rtol=1e-11, atol=1e-13)
        assert not y[i, lengths[i]:].any()


def test_scan_with_one_decay_for_all_is_linear_attention():
    """dt = 1, A the same for every channel: S_t = l S_{t-1} + b_t x_t^T, the other operator's recurrence."""
    rng = np.random.default_rng(3)
    x, b, c = rand(rng, 1, 9, 5), rand(rng, 1, 9, 1, 4), rand(rng, 1, 9, 1, 4)
    y, final = O.selective_scan(x, np.ones_like(x), np.full((5, 4), -0.3), b, c)
    o, state = S.linattn(c, b, x[:, :, None], [-0.3], 1.0)
    np.testing.assert_allclose(y, o[:, :, 0], rtol=1e-12)
    np.testing.assert_allclose(final[0], state[0, 0].T, rtol=1e-12)


def _difference(loss, at, i, d, h=1e-6):
    up, down = ([x + s * d if j == i else x for j, x in enumerate(at)] for s in (h, -h))
    return (loss(up) - loss(down)) / (2 * h)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("lengths", [None, [5, 1], [0, 7]])
def test_conv_gradients_against_differences(act, lengths):
    rng = np.random.default_rng(4)
    at = [rand(rng, 2, 7, 3), rand(rng, 3, 4), rand(rng, 3), rand(rng, 2, 3, 3)]
    d_y, d_final = rand(rng, 2, 7, 3), rand(rng, 2, 3, 3)

    def loss(v):
        y, final = O.causal_conv(v[0], v[1], v[2], act, lengths, v[3])
        return (y * d_y).sum() + (final * d_final).sum()

    for i, g in enumerate(O.causal_conv_backward(*at[:3], d_y, act, lengths, at[3], d_final)):
        d = rand(rng, *at[i].shape)
        # curvature 1e-12 times a third derivative, rounding 1e-16 / 1e-6 of the loss
        assert abs(_difference(loss, at, i, d) - (g * d).sum()) <= 1e-7 * (np.abs(g * d).sum() + 1)


@pytest.mark.parametrize("softplus,gated", [(True, True), (False, False)])
@pytest.mark.parametrize("lengths", [None, [5, 1], [0, 7]])
def test_scan_gradients_against_differences(softplus, gated, lengths):
    rng = np.random.default_rng(5)
    B, T, D, N, G = 2, 7, 4, 3, 2
    at = [rand(rng, B, T, D), rng.uniform(0.1, 1, (B, T, D)), -rng.uniform(0.1, 2, (D, N)), rand(rng, B, T, G, N), rand(rng, B, T, G, N),
          rand(rng, D), rand(rng, B, T, D), rand(rng, D) * 0.1, rand(rng, B, D, N)]
    names = ("d_x", "d_dt", "d_A", "d_b", "d_c", "d_skip", "d_gate", "d_dt_bias", "d_initial")
    d_y, d_final = rand(rng, B, T, D), rand(rng, B, D, N)

    def loss(v):
        y, final = O.selective_scan(*v[:6], v[6] if gated else None, v[7], softplus, lengths, v[8])
        return (y * d_y).sum() + (final * d_final).sum()

    grads = O.selective_scan_backward(*at[:5], d_y, at[5], at[6] if gated else None, at[7], softplus, lengths, at[8], d_final)
    for i, name in enumerate(names):
        if name == "d_gate" and not gated:
            continue
        d = rand(rng, *at[i].shape)
        assert abs(_difference(loss, at, i, d) - (grads[name] * d).sum()) <= 1e-7 * (np.abs(grads[name] * d).sum() + 1), name


def test_layer_norm_is_group_norm_of_one_group():
    rng = np.random.default_rng(6)
    x, w, b, d_y = rand(rng, 4, 9), rand(rng, 9), rand(rng, 9), rand(rng, 4, 9)
    for got, want in zip(O.layer_norm(x, w, b, 1e-5), S.group_norm(x[:, None], w, b, 1, 1e-5)):
        np.testing.assert_allclose(got.ravel(), want.ravel(), rtol=1e-13)
    for got, want in zip(O.layer_norm_backward(x, w, 1e-5, d_y), S.group_norm_backward(x[:, None], w, b, 1, 1e-5, d_y[:, None])):
        np.testing.assert_allclose(got.ravel(), want.ravel(), rtol=1e-12)
