"""The layer of paper_2405_05118_amd/selective.py against the same formulas in 64 bits.

Limits: eight stages in a row, each with a relative root mean square error below 2^-20 (sums of up to some hundred terms in 32 bits); sums
that cancel carry up to 16 times that: 8 * 16 * 2^-20 = 2^-13 of the root mean square.  A missing or exchanged term is of the size of
the result itself.
"""
import numpy as np
import pytest

from oracle import block as O

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
LIMIT = 8 * 16 * 2.0 ** -20
#         batch, length, width, channels, states, groups, taps
KINDS = {"few": (2, 37, 24, 20, 16, 1, 4), "one": (3, 1, 16, 12, 8, 1, 4), "ragged": (2, 130, 33, 42, 18, 2, 3)}


def flat(t):
    return t.reshape(-1, t.shape[-1])


def chain(w, x, stream, kind, lengths=None):
    """((out, total), what the gradients want, final state and window)."""
    B, T, _, C, N, G, _ = kind
    total = x + stream
    n = O.layer_norm(flat(total), w["norm_w"], w["norm_b"], 1e-5)[0].reshape(total.shape)
    u, gate = np.split(n @ w["w_in"], 2, axis=-1)
    v, window = O.causal_conv(u, w["conv_w"], w["conv_b"], "silu", lengths)
    dt, b, c = np.split(v @ w["w_x"], [C, C + G * N], axis=-1)
    b, c = b.reshape(B, T, G, N), c.reshape(B, T, G, N)
    y, state = O.selective_scan(v, dt, w["A"], b, c, w["skip"], gate, w["dt_bias"], True, lengths)
    return (y @ w["w_out"], total), (total, n, u, gate, v, dt, b, c, y), (state, window)


def slopes(w, x, stream, d_out, d_total, kind, lengths=None):
    _, (total, n, u, gate, v, dt, b, c, y), _ = chain(w, x, stream, kind, lengths)
    s = O.selective_scan_backward(v, dt, w["A"], b, c, d_out @ w["w_out"].T, w["skip"], gate, w["dt_bias"], True, lengths)
    d_q = np.concatenate([s["d_dt"], s["d_b"].reshape(*v.shape[:2], -1), s["d_c"].reshape(*v.shape[:2], -1)], axis=-1)
    d_v = d_q @ w["w_x"].T + s["d_x"]
    d_u, d_cw, d_cb, _ = O.causal_conv_backward(u, w["conv_w"], w["conv_b"], d_v, "silu", lengths)
    d_p = np.concatenate([d_u, s["d_gate"]], axis=-1)
    d_x, d_nw, d_nb = O.layer_norm_backward(flat(total), w["norm_w"], 1e-5, flat(d_p @ w["w_in"].T), flat(d_total))
    return {"x": d_x.reshape(x.shape), "w_in": flat(n).T @ flat(d_p), "w_x": flat(v).T @ flat(d_q), "w_out": flat(y).T @ flat(d_out),
            "conv_w": d_cw, "conv_b": d_cb, "norm_w": d_nw, "norm_b": d_nb, "A": s["d_A"], "skip": s["d_skip"], "dt_bias": s["d_dt_bias"]}


def random_weights(r, kind):
    _, _, W, C, N, G, taps = kind
    n = r.standard_normal
    return {"norm_w": 1 + 0.1 * n(W), "norm_b": 0.1 * n(W), "w_in": n((W, 2 * C)) * W ** -0.5, "conv_w": n((C, taps)) * 0.5, "conv_b": 0.1 * n(C),
            "w_x": n((C, C + 2 * G * N)) * C ** -0.5, "A": -np.exp(0.3 * n((C, N))), "skip": n(C), "dt_bias": n(C) - 1, "w_out": n((C, W)) * C ** -0.5}


def test_gradients_against_differences():
    kind = (2, 7, 5, 6, 3, 2, 3)
    r = np.random.default_rng(1)
    w, lengths = random_weights(r, kind), [7, 4]
    x, stream, d_out, d_total = (r.standard_normal((2, 7, 5)) for _ in range(4))
    grads = slopes(w, x, stream, d_out, d_total, kind, lengths)
    for name, g in grads.items():
        t = r.standard_normal(g.shape)
        ends = []
        for h in (1e-5, -1e-5):
            wh = dict(w) if name == "x" else dict(w, **{name: w[name] + h * t})
            out, total = chain(wh, x + h * t if name == "x" else x, stream, kind, lengths)[0]
            ends.append((out * d_out).sum() + (total * d_total).sum())
        # curvature 1e-10 times a third derivative, rounding 1e-16 / 1e-5 of the sum
        assert abs((ends[0] - ends[1]) / 2e-5 - (g * t).sum()) <= 1e-5 * (abs(g * t).sum() + 1), name


def near(got, ref, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    off = np.sqrt(np.mean((got - ref) ** 2) / (np.mean(ref ** 2) + 1e-60))
    assert off <= LIMIT, "%s: %.2g" % (what, off)


def layer_of(kind, w):
    from paper_2405_05118_amd.selective import SelectiveLayer

    layer = SelectiveLayer(*kind)
    for n, t in layer.weights.items():
        t.copy_(torch.from_numpy(w[n]))
    return layer, {n: t.double().cpu().numpy() for n, t in layer.weights.items()}


@gpu
@pytest.mark.parametrize("name,lengths", [("few", None), ("one", None), ("ragged", [130, 61])])
def test_layer(name, lengths):
    kind = KINDS[name]
    B, T, W = kind[:3]
    r = np.random.default_rng(4)
    layer, w = layer_of(kind, random_weights(r, kind))
    x, stream, d_out, d_total = (torch.from_numpy(r.standard_normal((B, T, W))).float().cuda() for _ in range(4))
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out, d_x = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    _, total = layer.forward(x, stream, out, n)
    layer.backward(d_out, d_total, d_x, n)
    x64, s64, o64, t64 = (t.double().cpu().numpy() for t in (x, stream, d_out, d_total))
    (ref, ref_total), _, (state, window) = chain(w, x64, s64, kind, lengths)
    near(out, ref, "out")
    near(total, ref_total, "total")
    near(layer.state, state, "state")
    near(layer.window, window, "window")
    grads = slopes(w, x64, s64, o64, t64, kind, lengths)
    near(d_x, grads.pop("x"), "x")
    for key, g in grads.items():
        near(layer.grads[key], g, key)


@gpu
def test_tokens_after_a_prompt():
    B, T, W, more = 2, 70, 24, 5
    kind = (B, T, W, 20, 16, 2, 4)
    r = np.random.default_rng(6)
    layer, w = layer_of(kind, random_weights(r, kind))
    x, stream = (torch.from_numpy(r.standard_normal((B, T + more, W))).float().cuda() for _ in range(2))
    (ref, _), _, (state, window) = chain(w, x.double().cpu().numpy(), stream.double().cpu().numpy(), (B, T + more, *kind[2:]))
    out = torch.empty(B, T, W, device="cuda")
    layer.forward(x[:, :T].contiguous(), stream[:, :T].contiguous(), out)
    near(out, ref[:, :T], "prompt")
    for t in range(more):
        one = torch.full((B, W), float("nan"), device="cuda")
        layer.step(x[:, T + t].contiguous(), stream[:, T + t].contiguous(), one)
        near(one, ref[:, T + t], "token %d" % t)
    near(layer.state, state, "state")
    near(layer.window, window, "window")


@gpu
def test_step_in_a_graph():
    """A token through the layer, captured once and replayed: the same bits as eager calls, with eager work in between."""
    kind = (3, 20, 32, 64, 16, 1, 4)
    layer, _ = layer_of(kind, random_weights(np.random.default_rng(8), kind))
    x, stream, out = (torch.randn(3, 32, generator=torch.Generator().manual_seed(i)).cuda() for i in range(3))
    layer.forward(torch.randn(3, 20, 32).cuda(), torch.randn(3, 20, 32).cuda(), torch.empty(3, 20, 32, device="cuda"))
    begin = layer.state.clone(), layer.window.clone()
    want = []
    for _ in range(3):
        layer.step(x, stream, out)
        want.append((out.clone(), layer.state.clone(), layer.window.clone()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step(x, stream, out)
    layer.state.copy_(begin[0]), layer.window.copy_(begin[1])
    for o, s, v in want:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(layer.state, s) and torch.equal(layer.window, v)
        torch.randn(1000, device="cuda").sum()


@gpu
def test_command(capsys):
    from paper_2405_05118_amd import selective

    off, first, loss = selective.main(["--length", "70", "--tokens", "5", "--width", "32", "--channels", "48", "--steps", "2"])
    assert off <= LIMIT and np.isfinite(first) and np.isfinite(loss)
    assert "tokens after a prompt" in capsys.readouterr().out


@gpu
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_command_as_it_is(seed):
    """The command's own sizes and steps: numbers to the end."""
    from paper_2405_05118_amd import selective

    off, first, loss = selective.main(["--seed", str(seed)])
    assert off <= LIMIT and np.isfinite(first) and np.isfinite(loss)


def test_channels_that_do_not_fall_into_groups_are_refused():
    from paper_2405_05118_amd.selective import SelectiveLayer

    with pytest.raises(ValueError):
        SelectiveLayer(1, 4, 8, 10, groups=3)
