"""One layer of a sequence model out of the library's entry points, on a residual stream: layer norm with the stream's sum, projections,
a short causal convolution, the selective state space scan with a gate, and the projection back.

    r' = r + x;  n = norm(r');  (u | gate) = n W_in;  c = silu(conv(u));  (dt | b | c) = c W_x;  y = scan(c, softplus(dt), b, c) silu(gate)
    x' = y W_out

What comes in is the layer before's output x and the stream r, what goes out x' and r': the sum is taken by the next layer's norm.
u and the gate are columns of one projection, dt, b and c of another, and their gradients columns of theirs: no operator
wants a copy of its own.  All of a layer's buffers belong to it; a call allocates nothing.
``python -m paper_2405_05118_amd.selective`` runs a prompt through two layers, then tokens one at a time from the states that it
left, compares those with the whole sequence in one call, and takes some steps of training.
"""
import argparse
import math

import torch

from . import binding as mdh
from .retention import _product

_F32 = torch.float32


class SelectiveLayer:
    """Weights, states and buffers for ``batch`` sequences of up to ``length`` tokens of a stream of ``width`` float32 channels;
    ``channels`` of the scan, with ``states`` each, in ``groups`` that share b and c; ``taps`` of the convolution."""

    def __init__(self, batch, length, width, channels, states=16, groups=1, taps=4, seed=0):
        if channels % groups:
            raise ValueError("%d channels do not fall into %d groups" % (channels, groups))
        self.batch, self.length, self.width, self.channels, self.states, self.groups, self.taps = (
            batch, length, width, channels, states, groups, taps)
        self.eps = 1e-5
        shared = groups * states
        self.parts = (channels, shared, shared)
        g = torch.Generator().manual_seed(seed)
        rows = batch * length

        def new(*shape):
            return torch.empty(shape, dtype=_F32, device="cuda")

        def weight(n, m):
            return (torch.randn(n, m, generator=g) * n ** -0.5).cuda()

        self.weights = {
            "norm_w": torch.ones(width, device="cuda"), "norm_b": torch.zeros(width, device="cuda"),
            "w_in": weight(width, 2 * channels), "conv_w": (torch.randn(channels, taps, generator=g) * taps ** -0.5).cuda(),
            "conv_b": torch.zeros(channels, device="cuda"), "w_x": weight(channels, channels + 2 * shared),
            # decays of 1, 2, .. a unit of time, time steps of 0.001 to 0.1 through the softplus
            "A": -torch.arange(1.0, states + 1).repeat(channels, 1).cuda(), "skip": torch.ones(channels, device="cuda"),
            "dt_bias": torch.log(torch.expm1(torch.exp(torch.rand(channels, generator=g) * math.log(100.0) + math.log(1e-3)))).cuda(),
            "w_out": weight(channels, width),
        }
        self.grads = {n: torch.empty_like(w) for n, w in self.weights.items()}
        self.state, self.window = new(batch, channels, states), new(batch, taps - 1, channels)
        # activations of a call and their gradients
        self.total, self.n, self.d_n = new(rows, width), new(rows, width), new(rows, width)
        self.mean, self.rstd = new(rows), new(rows)
        self.p, self.d_p = new(rows, 2 * channels), new(rows, 2 * channels)
        self.u, self.d_u, self.d_scan = new(rows, channels), new(rows, channels), new(rows, channels)
        self.q, self.d_q = new(rows, channels + 2 * shared), new(rows, channels + 2 * shared)
        self.y, self.d_y = new(rows, channels), new(rows, channels)
        sizes = (batch, length, channels, states, groups)
        self.checkpoints = torch.empty(mdh.mdh_selective_scan_checkpoints_size(sizes), dtype=torch.uint8, device="cuda")
        self.workspace = torch.empty(self._workspace_bytes(sizes), dtype=torch.uint8, device="cuda")

    def _workspace_bytes(self, sizes):
        """The most that any call of the layer asks for; those on one stream follow one another and can share it."""
        M, W, C, Q = self.batch * self.length, self.width, self.channels, self.q.shape[1]
        products = [(r, *d) for r in (M, self.batch) for d in ((2 * C, W), (Q, C), (W, C))]
        products += [(M, C, W), (C, W, M), (M, C, Q), (C, Q, M), (M, W, 2 * C), (W, 2 * C, M)]
        need = [mdh.mdh_selective_scan_workspace_size(sizes, _F32, True), mdh.mdh_layer_norm_workspace_size((M, W), _F32),
                mdh.mdh_causal_conv_workspace_size((self.batch, self.length, C, self.taps), _F32)]
        need += [mdh.mdh_workspace_size(mdh.MDH_BMATMUL, (1, *p, ta, tb, 0)) for p in products for ta in (0, 1) for tb in (0, 1)]
        return max(max(need), 4)

    def _columns(self, q, *lead):
        """Views of dt, b and c (groups apart) in the columns of q."""
        dt, b, c = q.split(self.parts, dim=1)
        return (dt.unflatten(0, lead), b.unflatten(1, (self.groups, self.states)).unflatten(0, lead),
                c.unflatten(1, (self.groups, self.states)).unflatten(0, lead))

    def _norm(self, x, stream, total, n, mean=None, rstd=None):
        w = self.weights
        mdh.mdh_layer_norm(x, w["norm_w"], w["norm_b"], n, self.eps, residual=stream, total=total, mean=mean, rstd=rstd)

    def forward(self, x, stream, out, lengths=None):
        """x, stream, out: (batch, length, width); returns (out, the stream with x added, a buffer of the layer).  States and windows
        begin at zero and are left as they are after every sequence's last token (``lengths`` (batch,) int32: after that many.  What
        x and the stream hold behind them goes through norm and projections like any row: finite, where gradients are wanted)."""
        B, T, C, w, ws = self.batch, self.length, self.channels, self.weights, self.workspace
        rows = x.view(B * T, -1)
        self._norm(rows, stream.view(B * T, -1), self.total, self.n, self.mean, self.rstd)
        _product(self.n, w["w_in"], self.p, workspace=ws)
        u, gate = self.p.view(B, T, 2 * C).split(C, dim=2)
        mdh.mdh_causal_conv(u, w["conv_w"], w["conv_b"], self.u.view(B, T, C), mdh.MDH_ACT_SILU, lengths, None, self.window)
        _product(self.u, w["w_x"], self.q, workspace=ws)
        dt, b, c = self._columns(self.q, B, T)
        mdh.mdh_selective_scan(self.u.view(B, T, C), dt, w["A"], b, c, self.y.view(B, T, C), w["skip"], gate, w["dt_bias"], True, lengths,
                               None, self.state, checkpoints=self.checkpoints, workspace=ws)
        _product(self.y, w["w_out"], out.view(B * T, -1), workspace=ws)
        return out, self.total.view(B, T, -1)

    def backward(self, d_out, d_stream, d_x, lengths=None):
        """Gradients after forward(..., lengths): d_x of x and of the stream alike, from those of what went out (d_stream: None = zeros);
        those of the weights in ``self.grads``."""
        B, T, C, w, g, ws = self.batch, self.length, self.channels, self.weights, self.grads, self.workspace
        d_rows = d_out.view(B * T, -1)
        _product(d_rows, w["w_out"], self.d_y, trans_b=True, workspace=ws)
        _product(self.y, d_rows, g["w_out"], trans_a=True, workspace=ws)
        u, gate = self.p.view(B, T, 2 * C).split(C, dim=2)
        d_u, d_gate = self.d_p.view(B, T, 2 * C).split(C, dim=2)
        dt, b, c = self._columns(self.q, B, T)
        d_dt, d_b, d_c = self._columns(self.d_q, B, T)
        mdh.mdh_selective_scan_backward(self.u.view(B, T, C), dt, w["A"], b, c, self.d_y.view(B, T, C), self.d_scan.view(B, T, C), d_dt,
                                        g["A"], d_b, d_c, self.checkpoints, w["skip"], gate, w["dt_bias"], True, lengths, None, g["skip"],
                                        d_gate, g["dt_bias"], None, ws)
        _product(self.d_q, w["w_x"], self.d_u, trans_b=True, workspace=ws)
        _product(self.u, self.d_q, g["w_x"], trans_a=True, workspace=ws)
        self.d_u += self.d_scan
        mdh.mdh_causal_conv_backward(u, w["conv_w"], w["conv_b"], self.d_u.view(B, T, C), d_u, g["conv_w"], g["conv_b"], mdh.MDH_ACT_SILU,
                                     lengths, workspace=ws)
        _product(self.d_p, w["w_in"], self.d_n, trans_b=True, workspace=ws)
        _product(self.n, self.d_p, g["w_in"], trans_a=True, workspace=ws)
        mdh.mdh_layer_norm_backward(self.total, w["norm_w"], self.mean, self.rstd, self.d_n, d_x.view(B * T, -1), g["norm_w"], g["norm_b"],
                                    None if d_stream is None else d_stream.view(B * T, -1), ws)
        return d_x

    def step(self, x, stream, out):
        """One more token of every sequence, x, stream, out: (batch, width), from the states and windows and onto them; returns (out,
        the stream with x added, a buffer of the layer)."""
        B, C, w, ws = self.batch, self.channels, self.weights, self.workspace
        self._norm(x, stream, self.total[:B], self.n[:B])
        _product(self.n[:B], w["w_in"], self.p[:B], workspace=ws)
        u, gate = self.p[:B].split(C, dim=1)
        mdh.mdh_causal_conv_step(u, w["conv_w"], w["conv_b"], self.window, self.u[:B], mdh.MDH_ACT_SILU)
        _product(self.u[:B], w["w_x"], self.q[:B], workspace=ws)
        dt, b, c = self._columns(self.q[:B], B)
        mdh.mdh_selective_scan_step(self.u[:B], dt, w["A"], b, c, self.state, self.y[:B], w["skip"], gate, w["dt_bias"], True)
        _product(self.y[:B], w["w_out"], out, workspace=ws)
        return out, self.total[:B]


def _through(layers, x, outs, lengths=None):
    """The stream behind all layers, their last output added."""
    stream = torch.zeros_like(x)
    for layer, out in zip(layers, outs):
        x, stream = layer.forward(x, stream, out, lengths)
    return stream + x


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, n in (("batch", 2), ("length", 300), ("tokens", 12), ("width", 256), ("channels", 512), ("states", 16), ("groups", 1), ("layers", 2),
                    ("steps", 20), ("seed", 0)):
        a.add_argument("--" + name, type=int, default=n)
    a = a.parse_args(argv)
    T, shape = a.length + a.tokens, (a.width, a.channels, a.states, a.groups, 4)
    whole = [SelectiveLayer(a.batch, T, *shape, a.seed + i) for i in range(a.layers)]
    short = [SelectiveLayer(a.batch, a.length, *shape, a.seed + i) for i in range(a.layers)]
    x = torch.randn(a.batch, T, a.width, generator=torch.Generator().manual_seed(a.seed + 100)).cuda()
    outs = [torch.empty_like(x) for _ in whole]
    y = _through(whole, x, outs)
    _through(short, x[:, :a.length].contiguous(), [torch.empty_like(x[:, :a.length]).contiguous() for _ in short])
    rest, ones = torch.empty_like(x[:, a.length:]), [torch.empty_like(x[:, 0]) for _ in short]
    for t in range(a.tokens):
        token, stream = x[:, a.length + t].contiguous(), torch.zeros_like(x[:, 0])
        for layer, one in zip(short, ones):
            token, stream = layer.step(token, stream, one)
        rest[:, t] = stream + token
    off = float((rest - y[:, a.length:]).abs().max() / y.abs().max()) if a.tokens else 0.0
    print("%d tokens after a prompt of %d: at most %.1e of the largest output from one call" % (a.tokens, a.length, off))
    # training: the layers learn the outputs of others
    others = [SelectiveLayer(a.batch, T, *shape, a.seed + 50 + i) for i in range(a.layers)]
    target = _through(others, x, outs)
    d_x, first, loss = torch.empty_like(x), None, None
    for _ in range(a.steps):
        d_y = _through(whole, x, outs) - target
        loss = float(d_y.square().mean())
        first = loss if first is None else first
        d_y /= a.batch * T
        d_stream = d_out = d_y  # both reach the sum behind the last layer
        for layer in reversed(whole):
            d_stream = d_out = layer.backward(d_out, d_stream, d_x).clone()
        # steps of length 0.1 at most: a scan's gradients grow with the cube of what goes in, and longer ones end in NaN
        size = sum(float(grad.square().sum()) for layer in whole for grad in layer.grads.values()) ** 0.5
        for layer in whole:
            for name, grad in layer.grads.items():
                layer.weights[name].add_(grad, alpha=-0.1 / max(1.0, size))
            layer.weights["A"].clamp_(max=-1e-3)  # (states that grow are not the scan's)
    if a.steps:
        print("%d steps of training: mean squared error %.4f -> %.4f" % (a.steps, first, loss))
    return off, first, loss


if __name__ == "__main__":
    main()
