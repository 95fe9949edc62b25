"""The layer of paper_2405_05118_amd/retention.py against the same formulas in 64 bits.

Limits: five stages in a row, each with a relative root mean square error below 2^-20 (sums of up to some hundred terms in 32 bits); a
row of the group norm whose scores cancel carries up to 16 times that: 5 * 16 * 2^-20 < 2^-13.6 of the root mean square.  A missing
or exchanged term is of the size of the result itself.
"""
import numpy as np
import pytest

from oracle import sequence as O

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
LIMIT = 5 * 16 * 2.0 ** -20
KINDS = {"few": (2, 37, 24, 4, 2, 16, 8), "one": (3, 1, 16, 2, 2, 16, 12), "ragged": (2, 130, 33, 6, 3, 20, 12)}


def split(p, B, T, H, Hk, dk, dv):
    q, k, v, gate = np.split(p, np.cumsum([Hk * dk, Hk * dk, H * dv]), axis=-1)
    return q.reshape(B, T, Hk, dk), k.reshape(B, T, Hk, dk), v.reshape(B, T, H, dv), gate


def chain(w, x, kind, lengths=None):
    B, T, _, H, Hk, dk, dv = kind
    q, k, v, gate = split(x @ w["w_in"], B, T, H, Hk, dk, dv)
    o, state = O.linattn(q, k, v, w["log_decay"], dk ** -0.5, lengths)
    rows = lambda t: t.reshape(B * T, 1, H * dv)  # noqa: E731
    z, _, _ = O.group_norm(rows(o), w["norm_w"], w["norm_b"], H, 1e-5, "silu", rows(gate))
    return z.reshape(B, T, -1) @ w["w_out"], (q, k, v, rows(gate), rows(o), z.reshape(B, T, -1)), state


def slopes(w, x, d_y, kind, lengths=None):
    B, T, _, H, Hk, dk, dv = kind
    _, (q, k, v, gate, o, z), _ = chain(w, x, kind, lengths)
    d_z = (d_y @ w["w_out"].T).reshape(B * T, 1, -1)
    d_o, d_w, d_b, d_gate = O.group_norm_backward(o, w["norm_w"], w["norm_b"], H, 1e-5, d_z, "silu", gate)
    d_q, d_k, d_v, _ = O.linattn_backward(q, k, v, w["log_decay"], d_o.reshape(B, T, H, dv), dk ** -0.5, lengths)
    d_p = np.concatenate([t.reshape(B, T, -1) for t in (d_q, d_k, d_v, d_gate)], axis=-1)
    flat = lambda t: t.reshape(B * T, -1)  # noqa: E731
    return {"x": d_p @ w["w_in"].T, "w_in": flat(x).T @ flat(d_p), "w_out": flat(z).T @ flat(d_y), "norm_w": d_w, "norm_b": d_b}


def test_gradients_against_differences():
    kind = (2, 7, 5, 4, 2, 3, 4)
    B, T, W, H, Hk, dk, dv = kind
    r = np.random.default_rng(1)
    w = {"w_in": r.standard_normal((W, 2 * Hk * dk + 2 * H * dv)), "w_out": r.standard_normal((H * dv, W)),
         "norm_w": 1 + 0.1 * r.standard_normal(H * dv), "norm_b": 0.1 * r.standard_normal(H * dv), "log_decay": np.log([0.5, 0.9, 0.99, 1.0])}
    x, d_y, lengths = r.standard_normal((B, T, W)), r.standard_normal((B, T, W)), [7, 4]
    grads = slopes(w, x, d_y, kind, lengths)
    for name, g in grads.items():
        t = r.standard_normal(g.shape)
        ends = []
        for h in (1e-5, -1e-5):
            wh = dict(w) if name == "x" else dict(w, **{name: w[name] + h * t})
            ends.append((chain(wh, x + h * t if name == "x" else x, kind, lengths)[0] * d_y).sum())
        # curvature 1e-10 times a third derivative, rounding 1e-16 / 1e-5 of the sum
        assert abs((ends[0] - ends[1]) / 2e-5 - (g * t).sum()) <= 1e-5 * (abs(g * t).sum() + 1), name


def near(got, ref, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    off = np.sqrt(np.mean((got - ref) ** 2) / (np.mean(ref ** 2) + 1e-60))
    assert off <= LIMIT, "%s: %.2g" % (what, off)


@gpu
@pytest.mark.parametrize("name,lengths", [("few", None), ("one", None), ("ragged", [130, 61])])
def test_layer(name, lengths):
    from paper_2405_05118_amd.retention import RetentionLayer

    kind = KINDS[name]
    B, T, W = kind[:3]
    layer = RetentionLayer(*kind, seed=3)
    r = np.random.default_rng(4)
    layer.norm_w.copy_(torch.from_numpy(1 + 0.2 * r.standard_normal(layer.norm_w.shape[0])))
    layer.norm_b.copy_(torch.from_numpy(0.2 * r.standard_normal(layer.norm_w.shape[0])))
    w = {n: getattr(layer, n).double().cpu().numpy() for n in ("w_in", "w_out", "norm_w", "norm_b", "log_decay")}
    x, d_y = (torch.from_numpy(r.standard_normal((B, T, W))).float().cuda() for _ in range(2))
    x64, d64 = x.double().cpu().numpy(), d_y.double().cpu().numpy()
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y, d_x = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    layer.forward(x, y, n)
    layer.backward(x, d_y, d_x, n)
    ref, _, state = chain(w, x64, kind, lengths)
    near(y, ref, "y")
    near(layer.state, state, "state")
    grads = slopes(w, x64, d64, kind, lengths)
    near(d_x, grads.pop("x"), "x")
    for key, g in grads.items():
        near(layer.grads[key], g, key)


@gpu
def test_tokens_after_a_prompt():
    from paper_2405_05118_amd.retention import RetentionLayer

    B, T, W, more = 2, 70, 24, 5
    kind = (4, 2, 16, 8)
    layer = RetentionLayer(B, T, W, *kind, seed=5)
    x = torch.randn(B, T + more, W, generator=torch.Generator().manual_seed(6)).cuda()
    w = {n: getattr(layer, n).double().cpu().numpy() for n in ("w_in", "w_out", "norm_w", "norm_b", "log_decay")}
    ref, _, state = chain(w, x.double().cpu().numpy(), (B, T + more, W, *kind))
    y = torch.empty(B, T, W, device="cuda")
    layer.forward(x[:, :T].contiguous(), y)
    near(y, ref[:, :T], "prompt")
    for t in range(more):
        near(layer.step(x[:, T + t].contiguous(), torch.full((B, W), float("nan"), device="cuda")), ref[:, T + t], "token %d" % t)
    near(layer.state, state, "state")


@gpu
def test_command(capsys):
    from paper_2405_05118_amd import retention

    off, first, loss = retention.main(["--batch", "2", "--length", "70", "--tokens", "4", "--width", "48", "--heads", "4", "--key-heads", "2",
                                       "--dk", "16", "--dv", "16", "--steps", "12"])
    assert off <= 2.0 ** -10 and loss < 0.9 * first  # (the largest element of a row that cancels: eight times LIMIT)
    assert "tokens after a prompt" in capsys.readouterr().out


def test_layer_refuses_heads_that_do_not_divide():
    from paper_2405_05118_amd.retention import RetentionLayer

    with pytest.raises(ValueError):
        RetentionLayer(1, 4, 8, 6, 4, 8, 8)
