"""Oracle of the sequence layers in 64 bits, token by token from the definitions: linear attention with a decay for each
head and its gradients, group norm with an activation and its gradients.  numpy only.

Every function takes and returns plain arrays; ``magnitude=True`` evaluates the same sums over absolute values, the scale
that rounding errors are measured against.
"""
import numpy as np
from scipy.special import erf


def _heads(x, H):
    """(B, T, heads, d) with every head written out."""
    return np.repeat(np.asarray(x, np.float64), H // x.shape[2], axis=2)


def _lengths(lengths, B, T):
    return np.full(B, T) if lengths is None else np.clip(np.asarray(lengths, np.int64), 0, T)


def linattn(q, k, v, log_decay, scale, lengths=None, initial=None, magnitude=False):
    """(o, final state): S_t = l S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t."""
    H, B, T = len(log_decay), q.shape[0], q.shape[1]
    f = np.abs if magnitude else (lambda x: x)
    n = _lengths(lengths, B, T)
    live = (np.arange(T) < n[:, None])[..., None, None]
    q, k, v = (f(np.where(live, _heads(x, H), 0.0)) for x in (q, k, v))
    l = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    S = np.zeros((B, H, k.shape[-1], v.shape[-1])) if initial is None else f(np.array(initial, np.float64))
    o = np.zeros((B, T, H, v.shape[-1]))
    for t in range(T):
        new = l * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        S = np.where(live[:, t, :, :, None], new, S)
        o[:, t] = abs(scale) * np.einsum("bhi,bhij->bhj", q[:, t], S) if magnitude else scale * np.einsum("bhi,bhij->bhj", q[:, t], S)
    return np.where(live, o, 0.0), S


def linattn_backward(q, k, v, log_decay, d_o, scale, lengths=None, initial=None, d_final=None, magnitude=False):
    """(d_q, d_k, d_v, d_initial)."""
    H, B, T = len(log_decay), q.shape[0], q.shape[1]
    f = np.abs if magnitude else (lambda x: x)
    shared = [x.shape[2] for x in (q, k, v)]
    n = _lengths(lengths, B, T)
    live = (np.arange(T) < n[:, None])[..., None, None]
    q, k, v, d_o = (f(np.where(live, _heads(x, H), 0.0)) for x in (q, k, v, d_o))
    scale = abs(scale) if magnitude else scale
    l = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    S = np.zeros((B, H, k.shape[-1], v.shape[-1])) if initial is None else f(np.array(initial, np.float64))
    E = np.zeros_like(S) if d_final is None else f(np.array(d_final, np.float64))
    d_q, d_k, d_v = (np.zeros_like(x) for x in (q, k, v))
    for t in range(T):
        S = np.where(live[:, t, :, :, None], l * S + k[:, t, :, :, None] * v[:, t, :, None, :], S)
        d_q[:, t] = scale * np.einsum("bhij,bhj->bhi", S, d_o[:, t])
    for t in reversed(range(T)):
        G = E + scale * q[:, t, :, :, None] * d_o[:, t, :, None, :]
        d_k[:, t] = np.einsum("bhij,bhj->bhi", G, v[:, t])
        d_v[:, t] = np.einsum("bhij,bhi->bhj", G, k[:, t])
        E = np.where(live[:, t, :, :, None], l * G, E)
    grads = [np.where(live, x, 0.0) for x in (d_q, d_k, d_v)]
    return (*(x.reshape(B, T, m, H // m, -1).sum(3) for x, m in zip(grads, shared)), E)


def _act(z, act):
    if act == "relu":
        return np.maximum(z, 0)
    if act == "silu":
        return z / (1 + np.exp(-z))
    return 0.5 * z * (1 + erf(z / np.sqrt(2))) if act == "gelu" else z


def _slope(z, act):
    if act == "relu":
        return (z > 0).astype(np.float64)
    if act == "silu":
        p = 1 / (1 + np.exp(-z))
        return p + z * p * (1 - p)
    if act == "gelu":
        return 0.5 * (1 + erf(z / np.sqrt(2))) + z * np.exp(-0.5 * z * z) / np.sqrt(2 * np.pi)
    return np.ones_like(z)


def group_norm(x, weight, bias, groups, eps, act="none", gate=None):
    """(y, mean, rstd) of x (N, S, C)."""
    N, S, C = x.shape
    g = np.asarray(x, np.float64).reshape(N, S, groups, C // groups)
    mean = g.mean((1, 3), keepdims=True)
    rstd = 1 / np.sqrt(((g - mean) ** 2).mean((1, 3), keepdims=True) + eps)
    z = ((g - mean) * rstd).reshape(N, S, C)
    z = z * (1.0 if weight is None else np.asarray(weight, np.float64)) + (0.0 if bias is None else np.asarray(bias, np.float64))
    y = _act(z, act) if gate is None else z * _act(np.asarray(gate, np.float64), act)
    return y, mean.reshape(N, groups), rstd.reshape(N, groups)


def group_norm_backward(x, weight, bias, groups, eps, d_y, act="none", gate=None):
    """(d_x, d_weight, d_bias, d_gate)."""
    N, S, C = x.shape
    _, mean, rstd = group_norm(x, weight, bias, groups, eps)
    D = C // groups
    mean, rstd = (np.repeat(t, D, axis=1)[:, None, :] for t in (mean, rstd))
    xh = (np.asarray(x, np.float64) - mean) * rstd
    w = np.ones(C) if weight is None else np.asarray(weight, np.float64)
    z = xh * w + (0.0 if bias is None else np.asarray(bias, np.float64))
    d_y = np.asarray(d_y, np.float64)
    if gate is None:
        d_z, d_gate = d_y * _slope(z, act), None
    else:
        gate = np.asarray(gate, np.float64)
        d_z, d_gate = d_y * _act(gate, act), d_y * z * _slope(gate, act)

    def over_group(t):
        m = t.reshape(N, S, groups, D).mean((1, 3))
        return np.repeat(m, D, axis=1)[:, None, :]

    t = d_z * w
    d_x = rstd * (t - over_group(t) - xh * over_group(t * xh))
    return d_x, (d_z * xh).sum((0, 1)), d_z.sum((0, 1)), d_gate
