"""The oracle of the sequence layers against what defines it: sums written out, and differences of the forward functions."""
import numpy as np
import pytest

from oracle import sequence as O


def rand(rng, *shape):
    return rng.standard_normal(shape)


def problem(rng, B=2, T=7, H=4, Hq=2, Hk=4, Hv=1, dk=3, dv=5):
    return (rand(rng, B, T, Hq, dk), rand(rng, B, T, Hk, dk), rand(rng, B, T, Hv, dv), -rng.uniform(0.01, 1, H), rand(rng, B, H, dk, dv))


def test_linattn_is_the_sum_over_pairs():
    rng = np.random.default_rng(1)
    q, k, v, g, S0 = problem(rng)
    lengths, scale = [7, 4], 0.3
    o, final = O.linattn(q, k, v, g, scale, lengths, S0)
    for b in range(2):
        for h in range(4):
            want = np.exp(g[h] * lengths[b]) * S0[b, h]
            for t in range(7):
                if t >= lengths[b]:
                    assert not o[b, t, h].any()
                    continue
                row = np.exp(g[h] * (t + 1)) * scale * (q[b, t, h // 2] @ S0[b, h])
                for s in range(t + 1):
                    row = row + scale * np.exp(g[h] * (t - s)) * (q[b, t, h // 2] @ k[b, s, h]) * v[b, s, 0]
                np.testing.assert_allclose(o[b, t, h], row, rtol=1e-12, atol=1e-13)
                want = want + np.exp(g[h] * (lengths[b] - 1 - t)) * np.outer(k[b, t, h], v[b, t, 0])
            np.testing.assert_allclose(final[b, h], want, rtol=1e-12, atol=1e-13)


def test_linattn_without_decay_and_with_none_left():
    rng = np.random.default_rng(2)
    q, k, v, _, S0 = problem(rng, H=2, Hq=2, Hk=2, Hv=2)
    o, final = O.linattn(q, k, v, [0.0, -np.inf], 1.0, None, S0)
    np.testing.assert_allclose(final[:, 0], S0[:, 0] + np.einsum("bti,btj->bij", k[:, :, 0], v[:, :, 0]), rtol=1e-12)
    np.testing.assert_allclose(o[:, :, 1], np.einsum("bti,bti->bt", q[:, :, 1], k[:, :, 1])[..., None] * v[:, :, 1], rtol=1e-12)


def _difference(loss, x, d, h=1e-6):
    return (loss(x + h * d) - loss(x - h * d)) / (2 * h)


@pytest.mark.parametrize("lengths", [None, [7, 3], [0, 7]])
def test_linattn_gradients_against_differences(lengths):
    rng = np.random.default_rng(3)
    q, k, v, g, S0 = problem(rng)
    d_o, d_final = rand(rng, 2, 7, 4, 5), rand(rng, 2, 4, 3, 5)

    def loss(*x):
        o, final = O.linattn(x[0], x[1], x[2], g, 0.7, lengths, x[3])
        return (o * d_o).sum() + (final * d_final).sum()

    grads = O.linattn_backward(q, k, v, g, d_o, 0.7, lengths, S0, d_final)
    at = [q, k, v, S0]
    for i in range(4):
        d = rand(rng, *at[i].shape)
        got = _difference(lambda x: loss(*(x if j == i else at[j] for j in range(4))), at[i], d)
        np.testing.assert_allclose((grads[i] * d).sum(), got, rtol=1e-7, atol=1e-7)


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("gated", [False, True])
def test_group_norm_gradients_against_differences(act, gated):
    rng = np.random.default_rng(4)
    x, gate = 2 + rand(rng, 2, 5, 6), rand(rng, 2, 5, 6) if gated else None
    w, b, d_y = rand(rng, 6), rand(rng, 6), rand(rng, 2, 5, 6)
    grads = O.group_norm_backward(x, w, b, 3, 1e-5, d_y, act, gate)
    at = [x, w, b, gate]
    for i in range(4 if gated else 3):
        d = rand(rng, *at[i].shape)

        def loss(t):
            y = [t if j == i else at[j] for j in range(4)]
            return (O.group_norm(y[0], y[1], y[2], 3, 1e-5, act, y[3])[0] * d_y).sum()

        np.testing.assert_allclose((grads[i] * d).sum(), _difference(loss, at[i], d), rtol=1e-6, atol=1e-7)


def test_group_norm_normalises_each_group():
    rng = np.random.default_rng(5)
    x = 3 + 2 * rand(rng, 2, 9, 8)
    y, mean, rstd = O.group_norm(x, None, None, 4, 0.0)
    y = y.reshape(2, 9, 4, 2)
    np.testing.assert_allclose(y.mean((1, 3)), 0, atol=1e-12)
    np.testing.assert_allclose((y ** 2).mean((1, 3)), 1, rtol=1e-12)
    np.testing.assert_allclose(mean, x.reshape(2, 9, 4, 2).mean((1, 3)))
    np.testing.assert_allclose(rstd, 1 / x.reshape(2, 9, 4, 2).std((1, 3)))
