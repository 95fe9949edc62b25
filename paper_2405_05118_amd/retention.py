"""One layer of a sequence model out of the library's entry points: projections, linear attention with a decay for each head,
a gated group norm over each head, and the projection back.

    p = x W_in = (q | k | v | gate);  o = linattn(q, k, v);  z = norm_h(o) silu(gate);  y = z W_out

q, k, v and the gate are columns of p and their gradients columns of d_p: no operator wants a copy of its own.  All of a
layer's buffers belong to it; a call allocates nothing.  ``python -m paper_2405_05118_amd.retention`` runs a prompt, then tokens
one at a time from the state that it left, compares those with the whole sequence in one call, and takes some steps of training.
"""
import argparse

import torch

from . import binding as mdh

_F32 = torch.float32


def _product(A, B, C, trans_a=False, trans_b=False, workspace=None):
    mdh.mdh_matmul_ex(A[None], B[None], C[None], trans_a, trans_b, False, None, workspace)


class RetentionLayer:
    """Weights, states and buffers for ``batch`` sequences of up to ``length`` tokens of ``width`` float32 channels.  ``heads``
    heads of values share ``key_heads`` heads of keys and queries."""

    def __init__(self, batch, length, width, heads, key_heads, dk, dv, seed=0):
        if heads % key_heads:
            raise ValueError("%d heads cannot share %d heads of keys" % (heads, key_heads))
        self.batch, self.length, self.width, self.heads, self.key_heads, self.dk, self.dv = batch, length, width, heads, key_heads, dk, dv
        self.scale, self.eps = dk ** -0.5, 1e-5
        qk, vg = key_heads * dk, heads * dv
        self.columns = (qk, qk, vg, vg)
        g = torch.Generator().manual_seed(seed)
        rows = batch * length

        def new(*shape):
            return torch.empty(shape, dtype=_F32, device="cuda")

        def weight(n, m):
            return (torch.randn(n, m, generator=g) * n ** -0.5).cuda()

        # memories of 8 to 8 * 2^(heads - 1) tokens
        self.log_decay = torch.log1p(-(2.0 ** (-3.0 - torch.arange(heads, dtype=torch.float64)))).to(_F32).cuda()
        self.w_in, self.w_out = weight(width, 2 * (qk + vg)), weight(vg, width)
        self.norm_w, self.norm_b = torch.ones(vg, device="cuda"), torch.zeros(vg, device="cuda")
        self.state = new(batch, heads, dk, dv)
        # activations of a call and their gradients
        self.p, self.d_p = new(rows, 2 * (qk + vg)), new(rows, 2 * (qk + vg))
        self.o, self.d_o, self.z, self.d_z = (new(rows, vg) for _ in range(4))
        self.mean, self.rstd = new(rows, heads), new(rows, heads)
        self.grads = {n: torch.empty_like(getattr(self, n)) for n in ("w_in", "w_out", "norm_w", "norm_b")}
        self.workspace = torch.empty(self._workspace_bytes(), dtype=torch.uint8, device="cuda")

    def _workspace_bytes(self):
        """The most that any call of the layer asks for; those on one stream follow one another and can share it."""
        M, K, n, W = self.batch * self.length, self.w_in.shape[1], self.heads * self.dv, self.width
        # dims of the products, their transposed operands
        products = [(r, *d) for r in (M, self.batch) for d in ((K, W), (W, n))] + [(M, n, W), (n, W, M), (M, W, K), (W, K, M)]
        need = [mdh.mdh_linattn_workspace_size((self.batch, self.length, self.heads, self.key_heads, self.key_heads, self.heads, self.dk,
                                                self.dv), _F32, True),
                mdh.mdh_group_norm_workspace_size((M, 1, n, self.heads), _F32, True)]
        need += [mdh.mdh_workspace_size(mdh.MDH_BMATMUL, (1, *p, ta, tb, 0)) for p in products for ta in (0, 1) for tb in (0, 1)]
        return max(max(need), 4)

    def _parts(self, p, *lead):
        """Views of q, k, v (heads apart) and of the gate in the columns of p."""
        q, k, v, gate = p.split(self.columns, dim=1)
        return (q.unflatten(1, (self.key_heads, self.dk)).unflatten(0, lead), k.unflatten(1, (self.key_heads, self.dk)).unflatten(0, lead),
                v.unflatten(1, (self.heads, self.dv)).unflatten(0, lead), gate)

    def _norm(self, rows):
        mdh.mdh_group_norm(self.o[:rows], self.norm_w, self.norm_b, self.z[:rows], self.heads, self.eps, mdh.MDH_ACT_SILU,
                           self._parts(self.p[:rows], rows)[3], self.mean[:rows], self.rstd[:rows], self.workspace)

    def forward(self, x, y, lengths=None):
        """x, y: (batch, length, width).  The states begin at zero and are left as they are after every sequence's last token
        (``lengths`` (batch,) int32: after that many)."""
        B, T = self.batch, self.length
        _product(x.view(B * T, -1), self.w_in, self.p, workspace=self.workspace)
        q, k, v, _ = self._parts(self.p, B, T)
        mdh.mdh_linattn(q, k, v, self.log_decay, self.o.view(B, T, self.heads, self.dv), self.scale, lengths, None, self.state,
                        workspace=self.workspace)
        self._norm(B * T)
        _product(self.z, self.w_out, y.view(B * T, -1), workspace=self.workspace)
        return y

    def backward(self, x, d_y, d_x, lengths=None):
        """Gradients after forward(x, ..., lengths): d_x, and those of the weights in ``self.grads``."""
        B, T, g, ws = self.batch, self.length, self.grads, self.workspace
        rows, d_rows = x.view(B * T, -1), d_y.view(B * T, -1)
        q, k, v, gate = self._parts(self.p, B, T)
        d_q, d_k, d_v, d_gate = self._parts(self.d_p, B, T)
        _product(d_rows, self.w_out, self.d_z, trans_b=True, workspace=ws)
        _product(self.z, d_rows, g["w_out"], trans_a=True, workspace=ws)
        mdh.mdh_group_norm_backward(self.o, self.norm_w, self.norm_b, self.mean, self.rstd, self.d_z, self.d_o, g["norm_w"],
                                    g["norm_b"], self.heads, mdh.MDH_ACT_SILU, gate, d_gate, ws)
        mdh.mdh_linattn_backward(q, k, v, self.log_decay, self.d_o.view(B, T, self.heads, self.dv), d_q, d_k, d_v, self.scale, lengths,
                                 workspace=ws)
        _product(self.d_p, self.w_in, d_x.view(B * T, -1), trans_b=True, workspace=ws)
        _product(rows, self.d_p, g["w_in"], trans_a=True, workspace=ws)
        return d_x

    def step(self, x, y):
        """One more token of every sequence, x, y: (batch, width), from the states and onto them."""
        B = self.batch
        _product(x, self.w_in, self.p[:B], workspace=self.workspace)
        q, k, v, _ = self._parts(self.p[:B], B)
        mdh.mdh_linattn_step(q, k, v, self.log_decay, self.state, self.o[:B].view(B, self.heads, self.dv), self.scale)
        self._norm(B)
        _product(self.z[:B], self.w_out, y, workspace=self.workspace)
        return y


def main(argv=None):
    a = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, n in (("batch", 2), ("length", 500), ("tokens", 12), ("width", 512), ("heads", 8), ("key-heads", 4), ("dk", 64), ("dv", 64),
                    ("steps", 20), ("seed", 0)):
        a.add_argument("--" + name, type=int, default=n)
    a = a.parse_args(argv)
    shape = (a.batch, a.width, a.heads, a.key_heads, a.dk, a.dv, a.seed)
    whole, short = RetentionLayer(a.batch, a.length + a.tokens, *shape[1:]), RetentionLayer(a.batch, a.length, *shape[1:])
    g = torch.Generator().manual_seed(a.seed + 1)
    x = torch.randn(a.batch, a.length + a.tokens, a.width, generator=g).cuda()
    y, rest = torch.empty_like(x), torch.empty_like(x[:, a.length:])
    whole.forward(x, y)
    short.forward(x[:, :a.length].contiguous(), torch.empty_like(x[:, :a.length]))
    one = torch.empty_like(x[:, 0])
    for t in range(a.tokens):
        rest[:, t] = short.step(x[:, a.length + t].contiguous(), one)
    off = float((rest - y[:, a.length:]).abs().max() / y.abs().max()) if a.tokens else 0.0
    print("%d tokens after a prompt of %d: at most %.1e of the largest output from one call" % (a.tokens, a.length, off))
    # training: the layer learns the outputs of another one
    with_other = RetentionLayer(a.batch, a.length + a.tokens, *shape[1:-1], a.seed + 2)
    target, d_y, d_x = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    with_other.forward(x, target)
    first = loss = None
    for _ in range(a.steps):
        whole.forward(x, y)
        torch.sub(y, target, out=d_y)
        loss = float(d_y.square().mean())
        first = loss if first is None else first
        d_y /= a.batch * (a.length + a.tokens)
        whole.backward(x, d_y, d_x)
        for name, grad in whole.grads.items():
            getattr(whole, name).add_(grad, alpha=-0.3)
    if a.steps:
        print("%d steps of training: mean squared error %.4f -> %.4f" % (a.steps, first, loss))
    return off, first, loss


if __name__ == "__main__":
    main()
