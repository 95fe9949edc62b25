"""Oracle of the selective state space block in 64 bits, token by token from the definitions: short causal convolution,
selective scan, layer norm, and their gradients.  numpy only.

Every function takes and returns plain arrays; ``magnitude=True`` evaluates the same sums over absolute values, the scale that
rounding errors are measured against.
"""
import numpy as np

from .sequence import _act, _lengths, _slope


def _f64(x):
    return np.asarray(x, np.float64)


def _line(x, lengths, initial, W):
    """The window that came in, the valid tokens, zeros from the length on; and which tokens are valid."""
    B, T, C = x.shape
    n = _lengths(lengths, B, T)
    live = (np.arange(T) < n[:, None])[..., None]
    before = np.zeros((B, W - 1, C)) if initial is None else _f64(initial)
    return np.concatenate((before, np.where(live, _f64(x), 0.0)), 1), live, n


def causal_conv(x, weight, bias, act="none", lengths=None, initial=None, magnitude=False):
    """(y, final window); with magnitude the sums before the activation over absolute values instead of y."""
    f = np.abs if magnitude else (lambda t: t)
    B, T, C = x.shape
    W = weight.shape[1]
    line, live, n = _line(x, lengths, initial, W)
    z = np.zeros((B, T, C)) + (0.0 if bias is None else f(_f64(bias)))
    for j in range(W):
        z += f(_f64(weight)[:, j] * line[:, j:j + T])
    final = np.stack([line[b, n[b]:n[b] + W - 1] for b in range(B)]) if B else np.zeros((0, W - 1, C))
    return np.where(live, z if magnitude else _act(z, act), 0.0), final


def causal_conv_backward(x, weight, bias, d_y, act="none", lengths=None, initial=None, d_final=None, magnitude=False):
    """(d_x, d_weight, d_bias, d_initial).  In magnitude a slope counts as 1 and what the errors of the sum before the activation
    move it by: terms of 1 may cancel in it, and it changes by no more than that sum does."""
    f = np.abs if magnitude else (lambda t: t)
    B, T, C = x.shape
    W, w = weight.shape[1], _f64(weight)
    line, live, n = _line(x, lengths, initial, W)
    z = np.zeros((B, T, C)) + (0.0 if bias is None else f(_f64(bias)))
    for j in range(W):
        z += f(w[:, j] * line[:, j:j + T])
    slope = _slope(z, act) if not magnitude else 1.0 if act == "none" else 1.0 + z
    d_z = f(np.where(live, _f64(d_y), 0.0)) * np.where(live, slope, 0.0)
    d_line, d_w = np.zeros_like(line), np.zeros((C, W))
    for j in range(W):
        d_line[:, j:j + T] += f(w[:, j]) * d_z
        d_w[:, j] = (d_z * f(line[:, j:j + T])).sum((0, 1))
    if d_final is not None:
        for b in range(B):
            d_line[b, n[b]:n[b] + W - 1] += f(_f64(d_final)[b])
    return np.where(live, d_line[:, W - 1:], 0.0), d_w, d_z.sum((0, 1)), d_line[:, :W - 1]


def _softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def _scan_operands(x, dt, A, b, c, skip, gate, dt_bias, softplus, lengths):
    B, T, D = x.shape
    N, E = A.shape[1], D // b.shape[2]
    live = (np.arange(T) < _lengths(lengths, B, T)[:, None])[..., None]
    clean = lambda t: np.where(live if t.ndim == 3 else live[..., None], _f64(t), 0.0)  # noqa: E731
    v = clean(dt) + (0.0 if dt_bias is None else _f64(dt_bias))
    delta = np.where(live, _softplus(v) if softplus else v, 0.0)
    slope = 1 / (1 + np.exp(-v)) if softplus else np.ones_like(v)
    wide = lambda t: np.repeat(clean(t), E, axis=2)  # noqa: E731  (B, T, D, N)
    g = None if gate is None else clean(gate)
    return live, clean(x), v, delta, slope, wide(b), wide(c), (np.zeros(D) if skip is None else _f64(skip)), g


def _silu(g):
    return g / (1 + np.exp(-g))


def selective_scan(x, dt, A, b, c, skip=None, gate=None, dt_bias=None, softplus=False, lengths=None, initial=None, magnitude=False):
    """(y, final state)."""
    f = np.abs if magnitude else (lambda t: t)
    B, T, D = x.shape
    live, x, _, delta, _, b, c, skip, g = _scan_operands(x, dt, A, b, c, skip, gate, dt_bias, softplus, lengths)
    A = _f64(A)
    h = np.zeros((B, D, A.shape[1])) if initial is None else f(_f64(initial))
    y = np.zeros((B, T, D))
    for t in range(T):
        h = np.where(live[:, t, :, None], np.exp(delta[:, t, :, None] * A) * h + f((delta[:, t] * x[:, t])[..., None] * b[:, t]), h)
        y[:, t] = (f(c[:, t]) * h).sum(-1) + f(skip * x[:, t])
    if g is not None:
        y = y * f(_silu(g))
    return np.where(live, y, 0.0), h


def selective_scan_backward(x, dt, A, b, c, d_y, skip=None, gate=None, dt_bias=None, softplus=False, lengths=None, initial=None,
                            d_final=None, magnitude=False):
    """A dict of d_x, d_dt, d_A, d_b, d_c, d_skip, d_gate, d_dt_bias, d_initial."""
    f = np.abs if magnitude else (lambda t: t)
    B, T, D = x.shape
    G = b.shape[2]
    live, x, v, delta, slope, b, c, skip, g = _scan_operands(x, dt, A, b, c, skip, gate, dt_bias, softplus, lengths)
    A = _f64(A)
    N = A.shape[1]
    x, b, c, skip, d_y = f(x), f(b), f(c), f(skip), f(np.where(live, _f64(d_y), 0.0))
    size = f(delta)  # (the factors exp(delta A) are positive either way)
    d_p = d_y if g is None else d_y * f(_silu(g))
    h, p = [np.zeros((B, D, N)) if initial is None else f(_f64(initial))], np.zeros((B, T, D))
    for t in range(T):
        h.append(np.exp(delta[:, t, :, None] * A) * h[-1] + (size[:, t] * x[:, t])[..., None] * b[:, t])
        p[:, t] = (c[:, t] * h[-1]).sum(-1) + skip * x[:, t]
    e = np.zeros((B, D, N)) if d_final is None else f(_f64(d_final))
    d_x, d_delta, d_A = np.zeros_like(x), np.zeros_like(x), np.zeros((D, N))
    d_b, d_c = np.zeros_like(b), np.zeros_like(c)
    for t in reversed(range(T)):
        d_c[:, t] = d_p[:, t, :, None] * h[t + 1]
        full = e + d_p[:, t, :, None] * c[:, t]
        d_b[:, t] = full * (size[:, t] * x[:, t])[..., None]
        r = (full * b[:, t]).sum(-1)
        e = np.exp(delta[:, t, :, None] * A) * full
        q = e * h[t]
        d_A += (q * size[:, t, :, None]).sum(0)
        d_delta[:, t] = (q * f(A)).sum(-1) + x[:, t] * r
        d_x[:, t] = size[:, t] * r + skip * d_p[:, t]
    d_dt = np.where(live, d_delta * slope, 0.0)
    per_group = lambda t: np.where(live[..., None], t.reshape(B, T, G, D // G, N).sum(3), 0.0)  # noqa: E731
    got = {"d_x": np.where(live, d_x, 0.0), "d_dt": d_dt, "d_A": d_A, "d_b": per_group(d_b), "d_c": per_group(d_c),
           "d_skip": (d_p * x).sum((0, 1)), "d_dt_bias": d_dt.sum((0, 1)), "d_initial": e}
    if g is not None:
        w = 1 / (1 + np.exp(-g))
        got["d_gate"] = np.where(live, d_y * p * (w * (1 + f(g) * (1 - w)) if magnitude else w * (1 + g * (1 - w))), 0.0)
    return got


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) of rows x (rows, C)."""
    x = _f64(x)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None] * (1.0 if weight is None else _f64(weight)) + (0.0 if bias is None else _f64(bias))
    return y, mean, rstd


def layer_norm_backward(x, weight, eps, d_y, d_total=None):
    """(d_x, d_weight, d_bias)."""
    _, mean, rstd = layer_norm(x, None, None, eps)
    xh = (_f64(x) - mean[:, None]) * rstd[:, None]
    d_y = _f64(d_y)
    t = d_y * (1.0 if weight is None else _f64(weight))
    d_x = rstd[:, None] * (t - t.mean(1, keepdims=True) - xh * (t * xh).mean(1, keepdims=True))
    return d_x + (0.0 if d_total is None else _f64(d_total)), (d_y * xh).sum(0), d_y.sum(0)
