"""Group norm with an activation, channels last: parity with the 64-bit oracle through the C ABI, and what it refuses.

Limits (u = 2^-24, m values a group).  Statistics: sums of m values, at most m / 256 of them one after the other, then a tree: their
error, of random sign, is below e = (24 + 4 sqrt(m / 256)) u of the mean absolute value.  What x - mean loses against a large mean
is in A = 1 + max|x| rstd.  z carries e A (|w| (1 + |xh|) + |b|); no activation's slope exceeds 1.13 and the exponentials are within
a few u.  Gradients: the same over t = dz w, xh and the group's means of both.  bf16 outputs are rounded once, 2^-8 of them.
"""
import numpy as np
import pytest

import paper_2405_05118_amd as mdh
from oracle import sequence as O

torch = pytest.importorskip("torch")
U = 2.0 ** -24
E_NULL, E_SIZE, E_WS, E_UNSUP = 1, 2, 5, 6
gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ACTS = {"none": mdh.MDH_ACT_NONE, "relu": mdh.MDH_ACT_RELU, "silu": mdh.MDH_ACT_SILU, "gelu": mdh.MDH_ACT_GELU}


def rand(seed, *shape, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype)


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def within(got, ref, limit, what):
    got = np64(got)
    assert np.isfinite(got).all(), what
    worst = np.max(np.abs(got - ref) / (limit + 1e-37), initial=0)
    assert worst <= 1, "%s: %.2f times its limit" % (what, worst)


class Problem:
    def __init__(self, dtype, N, S, C, G, act="none", gate=False, affine=True, offset=1.0, eps=1e-5, seed=0):
        self.dtype, self.N, self.S, self.C, self.G, self.act, self.eps = dtype, N, S, C, G, act, eps
        self.x = (rand(seed + 1, N, S, C) * (0.5 + rand(seed + 2, C).abs()) + offset * rand(seed + 3, C)).to(dtype)
        self.gate = rand(seed + 4, N, S, C, dtype=dtype) if gate else None
        self.w, self.b = (1 + 0.3 * rand(seed + 5, C), 0.3 * rand(seed + 6, C)) if affine else (None, None)
        self.d_y = rand(seed + 7, N, S, C, dtype=dtype)

    def workspace(self, backward):
        n = mdh.mdh_group_norm_workspace_size((self.N, self.S, self.C, self.G), self.dtype, backward)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None

    def run(self, lay=lambda t: t.cuda(), out=None):
        cu = lambda t: None if t is None else t.cuda()  # noqa: E731
        x, gate, d_y = lay(self.x), None if self.gate is None else lay(self.gate), lay(self.d_y)
        y, dx, dg = (torch.full_like(self.x, float("nan"), device="cuda") if out is None else out(self.x) for _ in range(3))
        mean, rstd = (torch.full((self.N, self.G), float("nan"), device="cuda") for _ in range(2))
        dw, db = (torch.full((self.C,), float("nan"), device="cuda") for _ in range(2))
        mdh.mdh_group_norm(x, cu(self.w), cu(self.b), y, self.G, self.eps, ACTS[self.act], gate, mean, rstd, self.workspace(False))
        mdh.mdh_group_norm_backward(x, cu(self.w), cu(self.b), mean, rstd, d_y, dx, dw, db, self.G, ACTS[self.act], gate,
                                    None if gate is None else dg, self.workspace(True))
        return y, mean, rstd, dx, dw, db, dg if gate is not None else None

    def check(self, **kw):
        x, w, b, gate, d_y = (np64(t) for t in (self.x, self.w, self.b, self.gate, self.d_y))
        N, S, C, G = self.N, self.S, self.C, self.G
        D, m = C // G, S * (C // G)
        ry, rmean, rrstd = O.group_norm(x, w, b, G, self.eps, self.act, gate)
        rdx, rdw, rdb, rdg = O.group_norm_backward(x, w, b, G, self.eps, d_y, self.act, gate)
        y, mean, rstd, dx, dw, db, dg = self.run(**kw)
        e = (24 + 4 * np.sqrt(m / 256)) * U
        each = lambda t: np.repeat(t, D, axis=1)[:, None, :]  # noqa: E731
        grouped = lambda t, f: each(f(t.reshape(N, S, G, D), (1, 3)))  # noqa: E731
        A = 1 + grouped(np.abs(x), np.max) * each(rrstd)
        xh = np.abs(x - each(rmean)) * each(rrstd)
        w1, b1 = (1.0 if w is None else np.abs(w)), (0.0 if b is None else np.abs(b))
        ez = e * A * (w1 * (1 + xh) + b1)
        half = 2.0 ** -8 if self.dtype == BF16 else 0.0
        f = 1.0 if gate is None else np.abs(gate)
        z = w1 * xh + b1
        within(mean, rmean, e * np.abs(x).reshape(N, S, G, D).mean((1, 3)), "mean")
        within(rstd, rrstd, 2 * e * A.reshape(N, G, D).max(2) * rrstd, "rstd")
        within(y, ry, 1.2 * ez * f + 8 * U * (np.abs(ry) + z * f) + half * np.abs(ry), "y")
        # |slope'| < 1.2, so an error of z moves dz by no more than that times dy; relu's slope has no such bound where z is near 0
        edz = np.abs(d_y) * (1.2 * ez if gate is None else 8 * U * (1 + f)) + 16 * U * np.abs(d_y) * (1 if gate is None else 1 + f)
        dz = np.abs(d_y) * (1.2 if gate is None else f)
        t, et = dz * w1, edz * w1
        mean_of = lambda v: grouped(v, np.mean)  # noqa: E731
        exh = e * A * (1 + xh)
        edx = each(rrstd) * (et + mean_of(et) + xh * mean_of(et * xh + t * exh) + exh * mean_of(t * xh)
                             + 2 * e * A * (t + mean_of(t) + xh * mean_of(t * xh)))
        within(dx, rdx, edx + half * np.abs(rdx), "d_x")
        rows = (64 + 8 * np.sqrt(N * S)) * U
        within(dw, rdw, (edz * xh + dz * exh + rows * dz * xh).sum((0, 1)), "d_weight")
        within(db, rdb, (edz + rows * dz).sum((0, 1)), "d_bias")
        if gate is not None:
            within(dg, rdg, np.abs(d_y) * 1.2 * (ez + 16 * U * z) + half * np.abs(rdg), "d_gate")


ROWS = [(1, 1, 8, 1), (1, 1, 1, 1), (3, 1, 4096, 32), (70, 1, 512, 4), (5, 1, 120, 24), (9, 1, 35, 5), (2, 1, 96, 96), (600, 1, 64, 2),
        (2, 1, 20000, 1), (3, 1, 5160, 8), (1000, 1, 24, 3)]
IMAGES = [(2, 49, 64, 32), (1, 2, 8, 8), (3, 1021, 120, 24), (1, 4096, 32, 4), (2, 300, 33, 11), (2, 64, 7, 1), (4, 17, 256, 16),
          (1, 9000, 8, 2), (1, 20011, 3, 3), (2, 100, 640, 2), (1, 700, 1028, 4), (33, 5, 48, 6), (1, 3000, 2600, 8)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", ROWS + IMAGES)
def test_parity(dtype, N, S, C, G):
    Problem(dtype, N, S, C, G, "silu", gate=(C % 3 != 0)).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("N,S,C,G", [(6, 1, 256, 8), (2, 77, 48, 6), (1, 6000, 16, 4)])
def test_activations(dtype, act, gate, N, S, C, G):
    Problem(dtype, N, S, C, G, act, gate).check()


@gpu
@pytest.mark.parametrize("N,S,C,G", [(6, 1, 256, 8), (2, 77, 48, 6), (1, 6000, 16, 4)])
def test_relu(N, S, C, G):
    """Its slope jumps at 0, so a z within rounding of 0 has either slope: values that are not there.  As a gate's activation it is
    taken of the gate, which has no rounding."""
    Problem(F32, N, S, C, G, "relu", gate=True).check()
    p = Problem(F32, N, S, C, G, "relu")
    y = np64(p.run()[0])
    ref, _, _ = O.group_norm(np64(p.x), np64(p.w), np64(p.b), G, p.eps, "relu")
    assert (y >= 0).all() and np.abs(y - ref).max() <= 2e-5
    bias = 20 + p.b
    p.b = torch.where(torch.arange(C) % 2 == 0, bias, -bias)  # far from 0 on either side
    p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", [(4, 1, 128, 4), (2, 77, 48, 6), (1, 6000, 16, 4)])
def test_without_weight_and_bias_and_with_a_large_mean(dtype, N, S, C, G):
    Problem(dtype, N, S, C, G, "silu", affine=False).check()
    Problem(dtype, N, S, C, G, "silu", offset=1000.0).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", [(3, 1, 128, 4), (2, 77, 48, 6), (1, 6000, 16, 4)])
def test_one_value_a_group(dtype, N, S, C, G):
    """Variance 0: x is its mean, and what comes out is the bias."""
    p = Problem(dtype, N, S, C, G, "none")
    p.x = torch.full((N, S, C), 3.0, dtype=dtype)
    y, mean, rstd, dx, dw, db, _ = p.run()
    assert torch.equal(y.cpu(), p.b.to(dtype).expand(N, S, C)) and (mean == 3).all()
    assert torch.allclose(rstd, torch.full_like(rstd, p.eps ** -0.5), rtol=1e-6)
    assert torch.isfinite(dx.float()).all() and not dw.any()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", [(3, 1, 128, 4), (2, 77, 48, 6), (2, 6000, 16, 4)])
def test_nan_and_infinity_stay_in_their_group(dtype, N, S, C, G):
    p = Problem(dtype, N, S, C, G, "silu", gate=True)
    good = p.run()
    D = C // G
    p.x[0, S // 2, D] = float("nan")        # group 1 of entry 0
    p.x[N - 1, 0, 3 * D] = float("inf")     # group 3 of the last entry
    got = p.run()
    bad = torch.zeros(N, G, dtype=torch.bool)
    bad[0, 1] = bad[N - 1, 3] = True
    rows = bad.repeat_interleave(D, 1)[:, None, :].expand(N, S, C).cuda()
    for i in (0, 3):  # y, d_x
        assert torch.isnan(got[i][rows]).all() and torch.equal(got[i][~rows], good[i][~rows])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", [(7, 1, 128, 4), (2, 77, 48, 6), (1, 6000, 16, 4), (3, 50, 30, 5)])
def test_strides(dtype, N, S, C, G):
    p = Problem(dtype, N, S, C, G, "silu", gate=True)

    def slice_of(before, after):
        def lay(t):
            wide = torch.full((N, S, before + C + after), float("nan"), dtype=dtype, device="cuda")
            wide[..., before:before + C] = t.cuda()
            return wide[..., before:before + C]
        return lay

    for lay in (slice_of(C, 2 * C), slice_of(1, 4), slice_of(8, 8)):
        p.check(lay=lay)
        p.check(lay=lay, out=lambda x: lay(torch.zeros_like(x)))


@gpu
def test_images_of_four_dimensions():
    p = Problem(F32, 2, 35, 24, 4, "silu")
    y = p.run()[0]
    x4, y4 = p.x.cuda().view(2, 5, 7, 24), torch.empty(2, 5, 7, 24, device="cuda")
    mdh.mdh_group_norm(x4, p.w.cuda(), p.b.cuda(), y4, 4, p.eps, mdh.MDH_ACT_SILU, workspace=p.workspace(False))
    assert torch.equal(y4.view_as(y), y)
    with pytest.raises(TypeError):  # a window of an image: positions are not evenly spaced
        mdh.mdh_group_norm(x4[:, :, 1:5], None, None, y4[:, :, 1:5].contiguous(), 4)


@gpu
def test_empty():
    x = torch.empty(0, 1, 16, device="cuda")
    none = torch.empty(0, 4, device="cuda")
    mdh.mdh_group_norm(x, None, None, x, 4)
    dw, db = torch.full((16,), 7.0, device="cuda"), torch.full((16,), 7.0, device="cuda")
    n = mdh.mdh_group_norm_workspace_size((0, 1, 16, 4), F32, True)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    mdh.mdh_group_norm_backward(x, None, None, none, none, x, x, dw, db, 4, workspace=ws)
    assert not dw.any() and not db.any()


@gpu
@pytest.mark.parametrize("N,S,C,G", [(500, 1, 256, 8), (2, 77, 48, 6), (2, 6000, 16, 4)])
def test_same_bits_on_another_stream_and_in_a_graph(N, S, C, G):
    p = Problem(BF16, N, S, C, G, "silu", gate=True)
    want = p.run()
    x, gate, d_y, w, b = (t.cuda() for t in (p.x, p.gate, p.d_y, p.w, p.b))
    got = [torch.empty_like(t) for t in want]
    wf, wb = p.workspace(False), p.workspace(True)

    def call():
        mdh.mdh_group_norm(x, w, b, got[0], G, p.eps, mdh.MDH_ACT_SILU, gate, got[1], got[2], wf)
        mdh.mdh_group_norm_backward(x, w, b, got[1], got[2], d_y, got[3], got[4], got[5], G, mdh.MDH_ACT_SILU, gate, got[6], wb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in got:
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, got))


@gpu
def test_gradients_against_differences():
    p = Problem(F32, 2, 40, 24, 4, "gelu", gate=True)
    _, _, _, dx, dw, db, dg = (np64(t) for t in p.run())
    at, d_y = [np64(t) for t in (p.x, p.w, p.b, p.gate)], np64(p.d_y)
    rng = np.random.default_rng(1)
    for i, g in enumerate((dx, dw, db, dg)):
        d, h = rng.standard_normal(at[i].shape), 1e-6
        up, down = ([t + s * d if j == i else t for j, t in enumerate(at)] for s in (h, -h))
        want = sum(s * (O.group_norm(*v[:3], 4, p.eps, "gelu", v[3])[0] * d_y).sum() for s, v in ((1, up), (-1, down))) / (2 * h)
        assert abs((g * d).sum() - want) <= 2e-5 * np.abs(g * d).sum()


def _raw(sizes, dtype=0, x=64, y=64, act=0, strides=None, ws=1 << 20, nws=1 << 40):
    st = None if strides is None else mdh.binding._sizes(strides)
    return mdh.lib().mdh_group_norm(mdh.binding._sizes(sizes), dtype, x, None, st, None, None, 1e-5, act, y, None, None, ws, nws, None)


def test_more_images_than_a_launch_has_are_refused():
    sizes = mdh.binding._sizes((1 << 24, 2, 16, 4))
    assert mdh.lib().mdh_group_norm(sizes, 0, 64, None, None, None, None, 1e-5, 0, 64, None, None, 1 << 20, 1 << 60, None) == E_SIZE
    assert mdh.lib().mdh_group_norm_backward(sizes, 0, 64, None, 64, None, None, None, 64, 64, 0, 64, None, None, None, 1 << 20, 1 << 60,
                                             None) == E_SIZE


def test_refusals():
    ok = (2, 5, 16, 4)
    for sizes in ((-1, 5, 16, 4), (2, -5, 16, 4), (2, 5, 0, 4), (2, 5, 16, 0), (2, 5, 16, 3), (1 << 20, 1 << 20, 16, 4)):
        assert _raw(sizes) == E_SIZE
    assert _raw(ok, dtype=2) == E_UNSUP and _raw(ok, act=4) == E_UNSUP and _raw(ok, act=-1) == E_UNSUP
    assert _raw(ok, x=None) == E_NULL and _raw(ok, y=None) == E_NULL
    assert _raw(ok, x=66) == E_UNSUP and _raw(ok, dtype=1, y=65) == E_UNSUP
    assert _raw(ok, strides=[16, 16, 8]) == E_SIZE  # outputs on one another
    assert _raw((0, 5, 16, 4), x=None, y=None) == 0 and _raw((2, 0, 16, 4), x=None, y=None) == 0
    need = mdh.mdh_group_norm_workspace_size((1, 100000, 64, 4), F32, False)
    if need:
        assert _raw((1, 100000, 64, 4), ws=None) == E_WS and _raw((1, 100000, 64, 4), nws=need - 1) == E_WS
    back = lambda **k: mdh.lib().mdh_group_norm_backward(mdh.binding._sizes(ok), 0, k.get("x", 64), k.get("gate"), k.get("dy", 64), None,  # noqa: E731
                                                         None, None, k.get("mean", 64), 64, 0, k.get("dx", 64), None, None, None, 1 << 20, 1 << 40, None)
    for name in ("x", "dy", "mean", "dx"):
        assert back(**{name: None}) == E_NULL
    assert back(gate=64) == E_NULL  # a gate without room for its gradient
    x = torch.zeros(2, 5, 16)
    with pytest.raises(TypeError):
        mdh.mdh_group_norm(x, None, None, x, 4)
    with pytest.raises(ValueError):
        mdh.mdh_group_norm_backward(x, None, None, None, None, x, x, None, None, 4, gate=x)


def test_binding_refuses_fewer_than_two_dimensions():
    """(C,) would be C rows of C channels.  Refused before a pointer is asked for: these tensors are not on the GPU either."""
    for x in (torch.zeros(64), torch.zeros(())):
        with pytest.raises(ValueError):
            mdh.mdh_group_norm(x, None, None, x, 4)
        with pytest.raises(ValueError):
            mdh.mdh_group_norm(x, None, None, x, 4, gate=x)
        with pytest.raises(ValueError):
            mdh.mdh_group_norm_backward(x, None, None, x, x, x, x, None, None, 4)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", [(5, 1, 128, 4), (2, 77, 48, 6), (1, 6000, 16, 4), (2, 1, 20000, 1)])
def test_relu_of_minus_infinity(dtype, N, S, C, G):
    """Channels whose gate or bias is -infinity: relu and its slope are 0 there, as for any other negative number."""
    p = Problem(dtype, N, S, C, G, "relu", gate=True)
    off = torch.arange(C) % 3 == 1
    p.gate[..., off] = -1.0
    p.check()
    want = p.run()
    p.gate[..., off] = -float("inf")
    got = p.run()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ref = O.group_norm(np64(p.x), np64(p.w), np64(p.b), G, p.eps, "relu", np64(p.gate))[0]
    assert not ref[..., off.numpy()].any() and not got[0][..., off.cuda()].any()
    p = Problem(dtype, N, S, C, G, "relu")
    p.b[off] = -1e30
    want = p.run()
    p.b[off] = -float("inf")
    assert all(torch.equal(a, b) for a, b in zip(p.run()[:6], want[:6]))


# (counts of a share, such as 82 and 110, whose product with their reciprocal need not be 1)
PARTS = [(16, 1312, 64, 32), (16, 1760, 64, 32), (2, 77, 48, 6), (1, 6000, 16, 4), (3, 1, 128, 4), (2, 1, 20000, 1)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", PARTS)
def test_one_value_a_group_in_any_number_of_parts(dtype, N, S, C, G):
    p = Problem(dtype, N, S, C, G, "none")
    p.x = torch.full((N, S, C), 3.0, dtype=dtype)
    y, mean, rstd, dx, dw, _, _ = p.run()
    assert torch.equal(y.cpu(), p.b.to(dtype).expand(N, S, C)) and (mean == 3).all()
    assert torch.allclose(rstd, torch.full_like(rstd, p.eps ** -0.5), rtol=1e-6)
    assert torch.isfinite(dx.float()).all() and not dw.any()


@gpu
@pytest.mark.parametrize("N,S,C,G", PARTS)
def test_means_whose_square_is_no_float(N, S, C, G):
    """Values around 1e20 (bf16: 2.5e19, in steps of 1.4e17): differences from their mean square to 1e34, they themselves to infinity."""
    for dtype, mean in ((F32, 1e20), (BF16, 2.5e19)):
        p = Problem(dtype, N, S, C, G, "none")
        p.x = (mean + 1e17 * rand(3, N, S, C)).to(dtype)
        p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("N,S,C,G", PARTS + [(3, 1, 24, 8), (70, 1, 512, 4), (2, 1021, 35, 5), (2, 3000, 8, 8), (1, 700, 1028, 4)])
def test_one_value_a_group_whatever_it_is(dtype, N, S, C, G):
    """Another constant for every group, most of whose sums are rounded: the mean is the value, the output the bias."""
    p = Problem(dtype, N, S, C, G, "none")
    values = torch.tensor([1000.3, 0.1, -12345.678, 1e-3, 7.7e8, -3.3e20, 1 / 3, 1e-20, 65537.0, -1.1])
    at = torch.arange(N * G).reshape(N, G) % len(values)
    group = values[at].to(dtype)
    p.x = group.repeat_interleave(C // G, 1)[:, None, :].expand(N, S, C).contiguous()
    y, mean, rstd, dx, dw, _, _ = p.run()
    assert torch.equal(mean.cpu(), group.float())
    assert torch.equal(y.cpu(), p.b.to(dtype).expand(N, S, C))
    moderate = (values[at].abs() <= 2000).cuda()
    assert torch.allclose(rstd[moderate], torch.full_like(rstd[moderate], p.eps ** -0.5), rtol=1e-6)
    assert torch.isfinite(rstd).all() and torch.isfinite(dx.float()).all() and not dw.any()


@gpu
def test_an_image_of_as_many_positions_as_are_taken():
    """2^31 - 1 positions of one channel, all of what is in them at the end: no position's number, nor what is added to it, may wrap.
    Sums of m values: relative errors of (24 + 4 sqrt(m / 256)) u = 7e-4 of the mean and the variance, two of them and a rounding
    of 2^-8 in the outputs."""
    m, tail = 2 ** 31 - 1, 1000
    x, d_y = torch.zeros(1, m, 1, dtype=BF16, device="cuda"), torch.zeros(1, m, 1, dtype=BF16, device="cuda")
    x[:, -tail:], d_y[:, -tail // 2:] = 1024.0, 1.0
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    mean, rstd, dw, db = (torch.full((1, 1) if i < 2 else (1,), float("nan"), device="cuda") for i in range(4))
    ws = torch.empty(mdh.mdh_group_norm_workspace_size((1, m, 1, 1), BF16, True), dtype=torch.uint8, device="cuda")
    mdh.mdh_group_norm(x, None, None, y, 1, 1e-5, mean=mean, rstd=rstd, workspace=ws)
    mdh.mdh_group_norm_backward(x, None, None, mean, rstd, d_y, dx, dw, db, 1, workspace=ws)
    rmean = tail * 1024 / m
    rrstd = (tail * 1024 ** 2 / m - rmean ** 2 + 1e-5) ** -0.5
    low, high = -rmean * rrstd, (1024 - rmean) * rrstd
    t1, t2 = tail / 2 / m, tail / 2 * high / m
    near = lambda got, want, limit: abs(float(got) - want) <= limit * abs(want)  # noqa: E731
    assert near(mean, rmean, 1e-3) and near(rstd, rrstd, 1e-3) and near(dw, tail / 2 * high, 2e-3) and float(db) == tail / 2
    assert near(y[0, 0, 0], low, 2e-3 + 2 ** -8) and near(y[0, -1, 0], high, 2e-3 + 2 ** -8)
    for t in (y[0, :-tail, 0], y[0, -tail:, 0], dx[0, :-tail, 0], dx[0, -tail:-tail // 2, 0], dx[0, -tail // 2:, 0]):
        assert bool((t == t[0]).all())
    # (t - t1 - xh t2: about half of the first term is left)
    assert near(dx[0, -1, 0], rrstd * (1 - t1 - high * t2), 8e-3 + 2 ** -8) and near(dx[0, -tail, 0], rrstd * (-t1 - high * t2), 8e-3 + 2 ** -8)


@pytest.mark.parametrize("sizes", [(1, 1, 1 << 29, 1 << 21), (3, 1, 1 << 30, 1 << 30), (0, 1, 1 << 29, 1), (1, 1, 1 << 29, 1)])
def test_more_channels_than_a_launch_adds_up_are_refused(sizes):
    """Gradients of weight and bias take a workgroup for 32 channels: fewer than 2^29, whatever the channels' groups are."""
    assert mdh.lib().mdh_group_norm_backward(mdh.binding._sizes(sizes), 0, 64, None, 64, None, None, None, 64, 64, 0, 64, None, 64, 64, 1 << 20,
                                             1 << 60, None) == E_SIZE


def test_a_workspace_that_is_missing_or_small_is_refused():
    for sizes in ((1, 100000, 64, 4), (2, 1, 20000, 1)):
        need = mdh.mdh_group_norm_workspace_size(sizes, F32, False)
        assert need > 0
        assert _raw(sizes, ws=None) == E_WS and _raw(sizes, nws=need - 1) == E_WS and _raw(sizes, ws=(1 << 20) + 8) == E_WS
    for sizes in ((1, 100000, 64, 4), (2, 1, 20000, 1), (5, 1, 64, 4)):
        need = mdh.mdh_group_norm_workspace_size(sizes, F32, True)
        assert need > 0
        for ws, n in ((None, 0), (1 << 20, need - 1), ((1 << 20) + 8, need)):
            assert mdh.lib().mdh_group_norm_backward(mdh.binding._sizes(sizes), 0, 64, None, 64, None, None, None, 64, 64, 0, 64, None, None, None,
                                                     ws, n, None) == E_WS
