"""Layer norm on a residual stream: parity with the 64-bit oracle through the C ABI at the widths, strides and values where it can go
wrong, and what it refuses.

Limits.  u = 2^-24.  A sum over a row is at most n = 80 + C / 1000 additions deep (32 of a lane, 10 between lanes, 16 between
wavefronts; wide rows: C / 1024 of a lane): the mean is off by n u m with m the mean of |x|, the differences from it and rstd by n u of
themselves and of m.  With k = 1 + m rstd that is 4 n u k of what a formula adds up in absolute values; a rounding to bf16 is 2^-8 of
the value, and sums over rows add a u for each.
"""
import numpy as np
import pytest

import paper_2405_05118_amd as mdh
from oracle import block as O

torch = pytest.importorskip("torch")
U = 2.0 ** -24
E_NULL, E_SIZE, E_WS, E_UNSUP = 1, 2, 5, 6
gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


def rand(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def cuda(t):
    return None if t is None else t.cuda()


def close(got, ref, limit, what, rounded=False):
    got = np64(got)
    assert np.isfinite(got).all(), what
    limit = limit + (2.0 ** -8 * np.abs(ref) if rounded else 0) + 1e-37
    worst = np.max(np.abs(got - ref) / limit, initial=0)
    assert worst <= 1, "%s: %.2f times its limit" % (what, worst)


class Problem:
    def __init__(self, dtype, rows, C, residual=True, affine=True, seed=0, offset=0.5):
        self.dtype, self.rows, self.C, self.eps = dtype, rows, C, 1e-5
        self.x = (rand(seed + 1, rows, C) + offset).to(dtype)
        self.res = (2 * rand(seed + 2, rows, C)).to(dtype) if residual else None
        self.w, self.b = (1 + 0.3 * rand(seed + 3, C), rand(seed + 4, C)) if affine else (None, None)
        self.d_y, self.d_total = rand(seed + 5, rows, C, dtype=dtype), rand(seed + 6, rows, C, dtype=dtype) if residual else None

    def stream(self):
        return self.x if self.res is None else (self.x.float() + self.res.float()).to(self.dtype)

    def empty(self, *shape, dtype=None):
        return torch.full(shape, NAN, dtype=dtype or self.dtype, device="cuda")

    def forward(self, lay=cuda, y=None):
        y = self.empty(self.rows, self.C) if y is None else y
        total = None if self.res is None else self.empty(self.rows, self.C)
        mean, rstd = self.empty(self.rows, dtype=F32), self.empty(self.rows, dtype=F32)
        mdh.mdh_layer_norm(lay(self.x), cuda(self.w), cuda(self.b), y, self.eps, None if self.res is None else lay(self.res), total, mean, rstd)
        return y, total, mean, rstd

    def backward(self, mean, rstd, lay=cuda, d_x=None):
        d_x = self.empty(self.rows, self.C) if d_x is None else d_x
        d_w, d_b = self.empty(self.C, dtype=F32), self.empty(self.C, dtype=F32)
        n = mdh.mdh_layer_norm_workspace_size((self.rows, self.C), self.dtype)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
        mdh.mdh_layer_norm_backward(lay(self.stream()), cuda(self.w), mean, rstd, lay(self.d_y), d_x, d_w, d_b,
                                    None if self.d_total is None else lay(self.d_total), ws)
        return d_x, d_w, d_b

    def check(self, **kw):
        half, s = self.dtype == BF16, np64(self.stream())
        y, total, mean, rstd = self.forward(**kw)
        if total is not None:
            assert torch.equal(total.cpu(), self.stream())
        ry, rmean, rrstd = O.layer_norm(s, np64(self.w), np64(self.b), self.eps)
        n = (80 + self.C / 1000) * U
        m = np.abs(s).mean(1)
        k = (1 + m * rrstd)[:, None]
        w, b = (np.ones(self.C), np.zeros(self.C)) if self.w is None else (np.abs(np64(self.w)), np.abs(np64(self.b)))
        xh = np.abs(s - rmean[:, None]) * rrstd[:, None]
        close(mean, rmean, 2 * n * m, "mean")
        close(rstd, rrstd, 4 * n * rrstd * k[:, 0], "rstd")
        close(y, ry, 4 * n * (k * (1 + xh) * w + b), "y", half)
        d_x, d_w, d_b = self.backward(mean, rstd, **kw)
        rx, rw, rb = O.layer_norm_backward(s, np64(self.w), self.eps, np64(self.d_y), np64(self.d_total))
        dy = np.abs(np64(self.d_y))
        t = dy * w
        size = rrstd[:, None] * (t + t.mean(1, keepdims=True) + (1 + xh) * (t * (1 + xh)).mean(1, keepdims=True))
        extra = 0 if self.d_total is None else U * np.abs(np64(self.d_total))
        close(d_x, rx, 8 * n * k * size + extra, "d_x", half)
        sums = self.rows * U
        close(d_w, rw, ((4 * n * k + sums) * dy * (1 + xh)).sum(0), "d_weight")
        close(d_b, rb, (sums * dy).sum(0), "d_bias")


WIDTHS = [1, 2, 7, 31, 64, 65, 250, 256, 500, 513, 1000, 1021, 1030, 2048, 2501, 4096, 4100, 5001, 8192, 10001, 16384, 16391, 33000]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", WIDTHS)
def test_parity(dtype, C):
    """Every number of lanes and pieces a row, with and without a residual."""
    Problem(dtype, 5, C, seed=C).check()
    Problem(dtype, 1, C, residual=False, affine=False, seed=C).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,C", [(3, 64), (70, 40), (5000, 16), (1100, 1000), (2100, 300), (1500, 2600), (700, 9000), (600, 17000)])
def test_more_rows_than_workgroups(dtype, rows, C):
    Problem(dtype, rows, C, seed=rows).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [24, 77, 700, 3001, 17001])
def test_strides(dtype, C):
    """Columns of wider rows at odd places; what lies beside an output stays; rows of more than one leading dimension."""
    p = Problem(dtype, 6, C)

    def odd(t):
        wide = torch.full((t.shape[0], C + 5), NAN, dtype=dtype, device="cuda")
        wide[:, 3:C + 3] = t.cuda()
        return wide[:, 3:C + 3]

    p.check(lay=odd)
    y, _, mean, rstd = p.forward()
    d_x = p.backward(mean, rstd)[0]
    for call, want in ((lambda o: p.forward(y=o), y), (lambda o: p.backward(mean, rstd, d_x=o), d_x)):
        wide = torch.full((6, C + 3), 7.0, dtype=dtype, device="cuda")
        call(wide[:, 1:C + 1])
        assert torch.equal(wide[:, 1:C + 1], want) and (wide[:, 0] == 7).all() and (wide[:, C + 1:] == 7).all()
    three, m3 = torch.empty(2, 3, C, dtype=dtype, device="cuda"), torch.empty(2, 3, device="cuda")
    mdh.mdh_layer_norm(p.stream().cuda().view(2, 3, C), p.w.cuda(), p.b.cuda(), three, p.eps, mean=m3)
    assert torch.equal(three.view(6, C), y) and torch.equal(m3.view(6), mean)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [40, 700, 3000, 17000])
def test_in_place(dtype, C):
    """The stream's sum where x or the residual was, y where x was, the gradient where that of y or of the sum was."""
    p = Problem(dtype, 9, C)
    y, total, mean, rstd = p.forward()
    d_x = p.backward(mean, rstd)[0]
    for at in (0, 1):
        x, res, out = p.x.cuda(), p.res.cuda(), torch.empty_like(y)
        mdh.mdh_layer_norm(x, p.w.cuda(), p.b.cuda(), out, p.eps, res, (x, res)[at])
        assert torch.equal(out, y) and torch.equal((x, res)[at], total)
    x = total.clone()
    mdh.mdh_layer_norm(x, p.w.cuda(), p.b.cuda(), x, p.eps)
    assert torch.equal(x, y)
    n = mdh.mdh_layer_norm_workspace_size((9, C), dtype)
    for at in (0, 1):
        both = [p.d_y.cuda(), p.d_total.cuda()]
        mdh.mdh_layer_norm_backward(total, p.w.cuda(), mean, rstd, both[0], both[at], None, None, both[1],
                                    torch.empty(n, dtype=torch.uint8, device="cuda"))
        assert torch.equal(both[at], d_x)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [1, 24, 110, 1028, 4096, 16384, 20000])
def test_one_value_a_row_whatever_it_is(dtype, C):
    """Another constant for every row, most of whose sums are rounded: the mean is the value, the output the bias."""
    values = torch.tensor([1000.3, 0.1, -12345.678, 1e-3, 7.7e8, -3.3e20, 1 / 3, 1e-20, 65537.0, -1.1]).to(dtype)
    p = Problem(dtype, len(values), C, residual=False)
    p.x = values[:, None].expand(-1, C).contiguous()
    y, _, mean, rstd = p.forward()
    assert torch.equal(mean.cpu(), values.float()) and torch.equal(y.cpu(), p.b.to(dtype).expand(len(values), C))
    assert torch.isfinite(rstd).all()
    d_x, d_w, _ = p.backward(mean, rstd)
    assert torch.isfinite(d_x.float()).all() and not d_w.any()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [2, 24, 110, 1028, 4096, 16384, 20000])
def test_rows_whose_sum_is_past_the_largest_number(dtype, C):
    """One value in all of a row gives the bias up to the largest one; with both signs the mean is near 0 and nothing is NaN; infinities still
    make their row NaN, and no other."""
    big = torch.finfo(dtype).max
    values = torch.tensor([big, -big, 1e38, -2.9e37, 3e35, 1.0, 1.0, 1.0]).to(dtype)
    p = Problem(dtype, len(values), C, residual=False)
    p.x = values[:, None].repeat(1, C)
    p.x[5] = torch.where(torch.arange(C) < C // 2, big, -big)
    p.x[6, C // 2], p.x[7, 0] = float("inf"), NAN
    y, _, mean, rstd = p.forward()
    assert torch.equal(mean[:5].cpu(), values[:5].float()) and torch.equal(y[:5].cpu(), p.b.to(dtype).expand(5, C))
    assert torch.isfinite(rstd[:6]).all() and torch.isfinite(mean[5]) and y[6:].isnan().all()
    # C products and sums of at most half of the largest number, off by u of that each; twice, for the half
    assert abs(float(mean[5]) - np64(p.x[5]).mean()) <= 2 * 2 * C * U * big / 2


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [30, 600, 4000, 18000])
def test_nan_and_infinity_stay_in_their_row(dtype, C):
    p = Problem(dtype, 7, C)
    want = p.forward()
    back = p.backward(*want[2:])[0]
    p.x[2, C // 2], p.x[5, 1] = NAN, float("inf")
    y, _, mean, rstd = p.forward()
    rest = [0, 1, 3, 4, 6]
    assert torch.equal(y[rest], want[0][rest]) and y[[2, 5]].isnan().all()
    assert torch.equal(p.backward(mean, rstd)[0][rest], back[rest])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_means(dtype):
    """Rows far from zero: 2000 times their spread in fp32, 30 times in bf16 (whose own steps are 1/8 there)."""
    for C in (100, 1000, 5000, 20000):
        Problem(dtype, 4, C, residual=False, offset=2000.0 if dtype == F32 else 30.0).check()


@gpu
def test_no_rows():
    p = Problem(F32, 0, 40)
    _, _, mean, rstd = p.forward()
    _, d_w, d_b = p.backward(mean, rstd)
    assert not d_w.any() and not d_b.any()


@gpu
def test_rows_past_2_31_elements():
    rows, C = 140000, 16384
    x = torch.zeros(rows, C, dtype=BF16, device="cuda")
    assert x.numel() > 1 << 31
    x[-3:] = rand(1, 3, C, dtype=BF16).cuda()
    y, mean, rstd = torch.full_like(x, NAN), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    mdh.mdh_layer_norm(x, None, None, y, mean=mean, rstd=rstd)
    few = torch.empty(3, C, dtype=BF16, device="cuda")
    mdh.mdh_layer_norm(x[-3:], None, None, few)
    assert torch.equal(y[-3:], few) and not y[:-3].any()


@gpu
@pytest.mark.parametrize("C", [100, 20000])
def test_gradients_of_rows_past_2_31_elements(C):
    """Operands and gradients as columns of one buffer whose last rows are past 2^31 elements: the bits of dense ones."""
    rows = 300
    p = Problem(BF16, rows, C)
    _, _, mean, rstd = p.forward()
    want = p.backward(mean, rstd)
    wide = torch.empty(rows, (1 << 31) // (rows - 20), dtype=BF16, device="cuda")
    assert wide[:-19].numel() > 1 << 31
    columns = iter(range(3, 6 * C, C + 5))

    def lay(t):
        at = next(columns)
        return wide[:, at:at + C].copy_(t)

    for got, ref in zip(p.backward(mean, rstd, lay, lay(p.x)), want):
        assert torch.equal(got, ref)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chip_full_of_work(dtype):
    """Every output with every compute unit busy, against 64 bits on the GPU; the same bits in three calls."""
    for rows, C in ((4096, 1024), (3000, 2501)):
        p = Problem(dtype, rows, C)
        s, d_y, w, b = (t.cuda().double() for t in (p.stream(), p.d_y, p.w, p.b))
        mean = s.mean(1, keepdim=True)
        rstd = ((s - mean).square().mean(1, keepdim=True) + p.eps).rsqrt()
        xh, t = (s - mean) * rstd, d_y * w
        want = [xh * w + b, rstd * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True)) + p.d_total.cuda().double(),
                (d_y * xh).sum(0), d_y.sum(0)]
        n, k = (80 + C / 1000) * U, 1 + s.abs().mean(1, keepdim=True) * rstd
        a, ta = 1 + xh.abs(), t.abs()
        limits = [4 * n * (k * a * w.abs() + b.abs()), 8 * n * k * rstd * (ta + ta.mean(1, keepdim=True) + a * (ta * a).mean(1, keepdim=True)) + n,
                  ((4 * n * k + rows * U) * d_y.abs() * a).sum(0), rows * U * d_y.abs().sum(0)]
        first = None
        for _ in range(3):
            y, _, m, r = p.forward()
            got = [y, *p.backward(m, r)]
            first = first or got
            assert all(torch.equal(i, j) for i, j in zip(first, got))
        for i, (g, r, limit) in enumerate(zip(got, want, limits)):
            assert ((g.double() - r).abs() <= limit + (2.0 ** -8 * r.abs() if dtype == BF16 and i < 2 else 0)).all(), i


@gpu
@pytest.mark.parametrize("rows,C", [(40, 100), (700, 2000)])
def test_same_bits_on_another_stream_and_in_a_graph(rows, C):
    p = Problem(BF16, rows, C)
    want = list(p.forward())
    want += p.backward(*want[2:])
    got = [torch.empty_like(t) for t in want]
    x, res, w, b, d_y, d_t = (cuda(t) for t in (p.x, p.res, p.w, p.b, p.d_y, p.d_total))
    ws = torch.empty(mdh.mdh_layer_norm_workspace_size((rows, C), BF16), dtype=torch.uint8, device="cuda")

    def call():
        mdh.mdh_layer_norm(x, w, b, got[0], p.eps, res, got[1], got[2], got[3])
        mdh.mdh_layer_norm_backward(got[1], w, got[2], got[3], d_y, got[4], got[5], got[6], d_t, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert all(torch.equal(i, j) for i, j in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in got:
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(i, j) for i, j in zip(want, got))


# ------------------------------------------------------------------ refusals: nothing is launched


def _raw(sizes, dtype=0, x=64, res=None, total=None, y=64, strides=None):
    S = mdh.binding._sizes
    return mdh.lib().mdh_layer_norm(S(sizes), dtype, x, res, None if strides is None else S(strides), None, None, 1e-5, total, y, None, None, None)


def _back(sizes, x=64, d_y=64, mean=64, rstd=64, d_x=64, ws=1 << 20, nws=1 << 50, strides=None):
    S = mdh.binding._sizes
    return mdh.lib().mdh_layer_norm_backward(S(sizes), 0, x, d_y, None, None if strides is None else S(strides), None, mean, rstd, d_x, None, None, ws,
                                             nws, None)


def test_refusals():
    ok = (4, 16)
    for sizes in ((-1, 16), (4, 0), (1 << 31, 16), (4, 1 << 24), (1 << 30, 5000), (1 << 22, 17000)):
        assert _raw(sizes) == E_SIZE
    assert _raw(ok, dtype=2) == E_UNSUP and _raw(ok, x=66) == E_UNSUP and _raw(ok, dtype=1, y=65) == E_UNSUP
    assert _raw(ok, x=None) == E_NULL and _raw(ok, y=None) == E_NULL and _raw(ok, res=64) == E_NULL  # no room for the sum
    assert _raw(ok, strides=[16, 16, 16, 8]) == E_SIZE and _raw(ok, res=64, total=64, strides=[16, 16, 0, 16]) == E_SIZE
    assert _raw((0, 16), x=None, y=None) == 0
    need = mdh.mdh_layer_norm_workspace_size(ok, F32)
    assert need > 0 and _back(ok, ws=None) == E_WS and _back(ok, nws=need - 1) == E_WS and _back(ok, ws=(1 << 20) + 8) == E_WS
    for name in ("x", "d_y", "mean", "rstd", "d_x"):
        assert _back(ok, **{name: None}) == E_NULL
    assert _back(ok, strides=[16, 16, 16, 15]) == E_SIZE


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(4, 16)
    with pytest.raises(TypeError):
        mdh.mdh_layer_norm(x, None, None, x)  # not on the GPU
    with pytest.raises(ValueError):
        mdh.mdh_layer_norm(x, None, None, x, residual=x)
    with pytest.raises(ValueError):
        mdh.mdh_layer_norm(x[0], None, None, x[0])
    with pytest.raises(ValueError):
        mdh.mdh_layer_norm_backward(torch.zeros(16), None, None, None, x, x, None, None)
    with pytest.raises((TypeError, ValueError)):
        mdh.mdh_layer_norm_backward(x, None, None, None, x[:2], x, None, None)
    with pytest.raises(TypeError):
        mdh.mdh_layer_norm_workspace_size((4, 16), torch.float64)
