"""The short causal convolution: parity with the 64-bit oracle through the C ABI, at the sizes, strides, lengths and values where it
can go wrong, and what it refuses.

Limits.  u = 2^-24; ``mag`` is a sum over absolute values.  W + 1 sums and products are off by (W + 2) u mag, an activation by 40 u of
what goes in (its exponential: |z| u of it, |z| <= 16 here), and changes by no more than 1.13 of its argument: (W + 64) u mag in
all.  A rounding to bf16 is 2^-8 of the value.  Sums over n tokens add n u.
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
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


def rand(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def close(got, ref, mag, dtype, n, what):
    got = np64(got)
    assert np.isfinite(got).all(), what
    limit = n * U * mag + (2.0 ** -8 * np.abs(ref) if dtype == BF16 else 0) + 1e-37
    worst = np.max(np.abs(got - ref) / limit, initial=0)
    assert worst <= 1, "%s: %.2f times its limit" % (what, worst)


def cuda(t):
    return None if t is None else t.cuda()


class Problem:
    def __init__(self, dtype, B, T, C, W, act="silu", lengths=None, windows=True, bias=True, seed=0):
        self.dtype, self.B, self.T, self.C, self.W, self.act = dtype, B, T, C, W, act
        self.x, self.d_y = rand(seed + 1, B, T, C, dtype=dtype), rand(seed + 2, B, T, C, dtype=dtype)
        self.w, self.b = rand(seed + 3, C, W) * W ** -0.5, rand(seed + 4, C) if bias else None
        self.before, self.d_after = (rand(seed + i, B, W - 1, C, dtype=dtype) if windows else None for i in (5, 6))
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)

    def lens(self):
        return None if self.lengths is None else self.lengths.numpy()

    def empty(self, *shape, dtype=None):
        return torch.full(shape, NAN, dtype=dtype or self.dtype, device="cuda")

    def forward(self, lay=cuda, y=None):
        y = self.empty(self.B, self.T, self.C) if y is None else y
        after = self.empty(self.B, self.W - 1, self.C)
        mdh.mdh_causal_conv(lay(self.x), self.w.cuda(), cuda(self.b), y, ACTS[self.act], cuda(self.lengths), cuda(self.before), after)
        return y, after

    def workspace(self):
        n = mdh.mdh_causal_conv_workspace_size((self.B, self.T, self.C, self.W), self.dtype)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None

    def backward(self, lay=cuda, d_x=None):
        d_x = self.empty(self.B, self.T, self.C) if d_x is None else d_x
        d_w, d_b, d_before = self.empty(self.C, self.W, dtype=F32), self.empty(self.C, dtype=F32), self.empty(self.B, self.W - 1, self.C)
        mdh.mdh_causal_conv_backward(lay(self.x), self.w.cuda(), cuda(self.b), lay(self.d_y), d_x, d_w, d_b, ACTS[self.act],
                                     cuda(self.lengths), cuda(self.before), cuda(self.d_after), d_before, self.workspace())
        return d_x, d_w, d_b, d_before

    def check(self, **kw):
        a = np64(self.x), np64(self.w), np64(self.b)
        rest = self.act, self.lens(), np64(self.before)
        (ref, after), (mag, _) = O.causal_conv(*a, *rest), O.causal_conv(*a, *rest, magnitude=True)
        y, got = self.forward(**kw)
        close(y, ref, mag, self.dtype, self.W + 64, "y")
        assert np.array_equal(np64(got), after)  # copies
        back = (*a, np64(self.d_y), *rest, np64(self.d_after))
        for got, r, m, what in zip(self.backward(**kw), O.causal_conv_backward(*back), O.causal_conv_backward(*back, magnitude=True),
                                   ("d_x", "d_weight", "d_bias", "d_initial_window")):
            sums = what in ("d_weight", "d_bias")
            close(got, r, m, F32 if sums else self.dtype, 2 * self.W + 128 + (self.B * self.T if sums else 0), what)


SHAPES = [(1, 1, 1, 4), (2, 1, 64, 4), (1, 2, 7, 3), (2, 3, 17, 4), (1, 7, 9, 8), (3, 8, 8, 2), (1, 9, 33, 4), (2, 31, 40, 5), (1, 33, 130, 6),
          (2, 64, 72, 7), (1, 65, 12, 8), (1, 130, 257, 4), (2, 200, 65, 1), (1, 1000, 24, 4), (5, 100, 1, 2)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,C,W", SHAPES)
def test_parity(dtype, B, T, C, W):
    Problem(dtype, B, T, C, W, seed=T).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("windows,bias", [(True, False), (False, True)])
def test_activations_and_what_may_be_left_out(dtype, act, windows, bias):
    Problem(dtype, 2, 77, 50, 4, act, windows=windows, bias=bias).check()


@gpu
@pytest.mark.parametrize("act", ["none", "relu"])
def test_whole_numbers_are_exact(act):
    """Sums of small whole numbers and a half: no rounding anywhere, and nothing at relu's corner."""
    p = Problem(F32, 2, 70, 20, 4, act)
    for t in (p.x, p.d_y, p.w, p.before, p.d_after):
        t.copy_((t * 3).round())
    p.b.copy_(p.b.round() + 0.5)
    a = np64(p.x), np64(p.w), np64(p.b)
    assert np.array_equal(np64(p.forward()[0]), O.causal_conv(*a, act, None, np64(p.before))[0])
    for got, want in zip(p.backward(), O.causal_conv_backward(*a, np64(p.d_y), act, None, np64(p.before), np64(p.d_after))):
        assert np.array_equal(np64(got), want)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths", [[0, 40, 1, 3], [40, 39, 2, 8], [0, 0, 0, 0], [-3, 1000, 9, 33]])
def test_lengths_with_anything_behind_them(dtype, lengths):
    """Tokens past an entry's length hold NaN and infinities: nothing of them is read, their outputs and gradients are 0."""
    p = Problem(dtype, 4, 40, 21, 4, lengths=lengths)
    for b, n in enumerate(min(max(n, 0), 40) for n in lengths):
        p.x[b, n:], p.d_y[b, n:] = NAN, float("inf")
    p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [NAN, float("inf")])
@pytest.mark.parametrize("W", [2, 4, 8])
def test_what_no_token_reads_is_in_no_gradient(dtype, bad, W):
    """The window before a sequence of no tokens, and a last token for all taps but its own."""
    p = Problem(dtype, 3, 200, 21, W, "none", lengths=[200, 0, 77])
    p.before[1], p.x[0, 199, 3], p.x[2, 76, 5] = 0, 0, 0
    d_x, d_w, d_b, d_before = p.backward()
    p.before[1], p.x[0, 199, 3], p.x[2, 76, 5] = bad, bad, bad
    got = p.backward()
    assert torch.equal(got[0], d_x) and torch.equal(got[2], d_b) and torch.equal(got[3], d_before)
    assert torch.equal(got[1][:, :-1], d_w[:, :-1])
    rest = [i for i in range(21) if i not in (3, 5)]
    assert torch.equal(got[1][rest], d_w[rest]) and not got[1][[3, 5], -1].isfinite().any()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("C", [24, 27])
def test_strides(dtype, C):
    """Columns of wider rows, at odd places; one token's values for all tokens; what lies beside an output stays."""
    p = Problem(dtype, 2, 45, C, 4)

    def odd(t):
        wide = torch.full((*t.shape[:2], C + 5), NAN, dtype=dtype, device="cuda")
        wide[..., 3:C + 3] = t.cuda()
        return wide[..., 3:C + 3]

    p.check(lay=odd)
    p.check(lay=lambda t: t.cuda().transpose(0, 1).contiguous().transpose(0, 1))
    plain = p.forward()[0], p.backward()[0]
    for i, call in ((0, lambda o: p.forward(y=o)), (1, lambda o: p.backward(d_x=o))):
        wide = torch.full((2, 45, C + 7), 7.0, dtype=dtype, device="cuda")
        call(wide[..., 1:C + 1])
        assert torch.equal(wide[..., 1:C + 1], plain[i]) and (wide[..., :1] == 7).all() and (wide[..., C + 1:] == 7).all()
    p.x = p.x[:, :1].expand(p.x.shape)
    p.check(lay=lambda t: t[:, :1].cuda().expand(t.shape) if t.stride(1) == 0 else t.cuda())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_tokens(dtype):
    p = Problem(dtype, 2, 0, 10, 4)
    assert torch.equal(p.forward()[1].cpu(), p.before)
    _, d_w, d_b, d_before = p.backward()
    assert torch.equal(d_before.cpu(), p.d_after) and not d_w.any() and not d_b.any()
    p = Problem(dtype, 0, 5, 10, 4)
    p.forward()
    _, d_w, d_b, _ = p.backward()
    assert not d_w.any() and not d_b.any()


@gpu
@pytest.mark.parametrize("T", [1, 2, 50])
def test_windows_in_place_and_in_slots(T):
    p = Problem(BF16, 3, T, 19, 4)
    y, after = p.forward()
    window, y2 = p.before.cuda(), torch.empty_like(y)
    mdh.mdh_causal_conv(p.x.cuda(), p.w.cuda(), p.b.cuda(), y2, mdh.MDH_ACT_SILU, None, window, window)
    assert torch.equal(y, y2) and torch.equal(window, after)
    pool = rand(9, 7, 3, 19, dtype=BF16).cuda()
    before = pool.clone()
    pool[5], pool[2] = p.before[0].cuda(), p.before[2].cuda()
    slots = torch.tensor([5, -1, 2], dtype=torch.int32, device="cuda")
    mdh.mdh_causal_conv(p.x.cuda(), p.w.cuda(), p.b.cuda(), y2, mdh.MDH_ACT_SILU, None, pool, pool, slots)
    assert torch.equal(pool[5], after[0]) and torch.equal(pool[2], after[2]) and torch.equal(y2[0], y[0]) and torch.equal(y2[2], y[2])
    rest = [0, 1, 3, 4, 6]
    assert torch.equal(pool[rest], before[rest])
    p.before[1] = 0  # an entry without a slot begins with zeros
    assert torch.equal(p.forward()[0][1], y2[1])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,C,W", [(1, 1, 4), (3, 64, 4), (2, 37, 2), (300, 24, 3), (1, 2048, 4), (4, 100, 8), (2, 16, 1)])
def test_step(dtype, B, C, W):
    p = Problem(dtype, B, 1, C, W)
    a = np64(p.x), np64(p.w), np64(p.b), "silu", None, np64(p.before)
    (ref, after), (mag, _) = O.causal_conv(*a), O.causal_conv(*a, magnitude=True)
    window, y = p.before.cuda(), p.empty(B, C)
    mdh.mdh_causal_conv_step(p.x[:, 0].cuda(), p.w.cuda(), p.b.cuda(), window, y, mdh.MDH_ACT_SILU)
    close(y, ref[:, 0], mag[:, 0], dtype, W + 64, "y")
    assert np.array_equal(np64(window), after)


@gpu
def test_step_in_slots_and_strides():
    p = Problem(BF16, 4, 1, 43, 4)
    x, y, window = p.x[:, 0].cuda(), p.empty(4, 43), p.before.cuda()
    mdh.mdh_causal_conv_step(x, p.w.cuda(), p.b.cuda(), window, y, mdh.MDH_ACT_SILU)
    pool = rand(3, 9, 3, 43, dtype=BF16).cuda()
    before = pool.clone()
    slots = torch.tensor([8, -1, 0, 9], dtype=torch.int32, device="cuda")
    pool[8], pool[0] = p.before[0].cuda(), p.before[2].cuda()
    wide = p.empty(4, 90)
    wide[:, 5:48] = x
    y2 = p.empty(4, 2, 43)[:, 1]
    mdh.mdh_causal_conv_step(wide[:, 5:48], p.w.cuda(), p.b.cuda(), pool, y2, mdh.MDH_ACT_SILU, slots)
    assert torch.equal(y2[0], y[0]) and torch.equal(y2[2], y[2]) and not y2[1].any() and not y2[3].any()
    assert torch.equal(pool[8], window[0]) and torch.equal(pool[0], window[2]) and torch.equal(pool[1:8], before[1:8])


@gpu
def test_past_2_31_elements():
    """The last sequence and the last slot of buffers whose offsets in elements do not fit 32 bits."""
    B, T, C = 3, 16384, 50000
    x, y = torch.zeros(B, T, C, dtype=BF16, device="cuda"), torch.full((B, T, C), NAN, dtype=BF16, device="cuda")
    assert x.numel() > 1 << 31
    x[2, -40:] = rand(1, 40, C, dtype=BF16).cuda()
    w, b = rand(2, C, 4).cuda(), rand(3, C).cuda()
    mdh.mdh_causal_conv(x, w, b, y, mdh.MDH_ACT_SILU)
    one = torch.empty(1, 40, C, dtype=BF16, device="cuda")
    mdh.mdh_causal_conv(x[2:, -40:], w, b, one, mdh.MDH_ACT_SILU)
    assert torch.equal(y[2, -40:], one[0])
    pool = y.view(B * T, 1, C)[:, :, :]
    slots = torch.tensor([B * T - 1], dtype=torch.int32, device="cuda")
    window, out, out2 = pool[-1:].clone(), torch.empty(1, C, dtype=BF16, device="cuda"), torch.empty(1, C, dtype=BF16, device="cuda")
    mdh.mdh_causal_conv_step(x[0, :1], w[:, :2].contiguous(), b, pool, out, mdh.MDH_ACT_NONE, slots)
    mdh.mdh_causal_conv_step(x[0, :1], w[:, :2].contiguous(), b, window, out2, mdh.MDH_ACT_NONE)
    assert torch.equal(out, out2) and torch.equal(pool[-1:], window)


@gpu
def test_gradients_past_2_31_elements():
    """Operands and gradients as columns of one buffer whose last tokens are past 2^31 elements: the bits of dense ones."""
    T = 150
    p = Problem(BF16, 2, T, 21, 4, lengths=[T, T - 9])
    want = [*p.forward(), *p.backward()]
    wide = torch.empty(2, T, (1 << 31) // T + 400, dtype=BF16, device="cuda")
    assert wide[0].numel() > 1 << 31
    columns = iter(range(3, 400, 30))

    def lay(t):
        at = next(columns)
        return wide[:, :, at:at + 21].copy_(t)

    for got, ref in zip([*p.forward(lay, lay(p.x)), *p.backward(lay, lay(p.x))], want):
        assert torch.equal(got, ref)


@gpu
def test_prompt_then_tokens():
    """A prompt and the tokens after it, one at a time, are one sequence, bit for bit."""
    p = Problem(BF16, 2, 30, 40, 4)
    whole, after = p.forward()
    window, y = p.before.cuda(), torch.empty_like(whole[:, :25])
    mdh.mdh_causal_conv(p.x[:, :25].contiguous().cuda(), p.w.cuda(), p.b.cuda(), y, mdh.MDH_ACT_SILU, None, window, window)
    assert torch.equal(y, whole[:, :25])
    for t in range(25, 30):
        one = torch.empty(2, 40, dtype=BF16, device="cuda")
        mdh.mdh_causal_conv_step(p.x[:, t].cuda(), p.w.cuda(), p.b.cuda(), window, one, mdh.MDH_ACT_SILU)
        assert torch.equal(one, whole[:, t])
    assert torch.equal(window, after)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_chip_full_of_work(dtype):
    """Every output with every compute unit busy, against 64 bits on the GPU; the same bits in three calls."""
    B, T, C, W = 4, 1024, 2056, 4
    p = Problem(dtype, B, T, C, W, windows=False)
    line = torch.nn.functional.pad(p.x.cuda().double(), (0, 0, W - 1, 0))
    w, b = p.w.cuda().double(), p.b.cuda().double()
    z = sum(w[:, j] * line[:, j:j + T] for j in range(W)) + b
    mag = sum(w[:, j].abs() * line[:, j:j + T].abs() for j in range(W)) + b.abs()
    f = torch.sigmoid(z)
    d_z = p.d_y.cuda().double() * f * (1 + z * (1 - f))
    d_zm = p.d_y.cuda().double().abs() * (1 + mag)
    turn = lambda t, q: sum(q[:, j] * torch.nn.functional.pad(t, (0, 0, 0, W - 1))[:, W - 1 - j:W - 1 - j + T] for j in range(W))  # noqa: E731
    want = [(z * f, mag), (turn(d_z, w), turn(d_zm, w.abs())),
            (torch.stack([(d_z * line[:, j:j + T]).sum((0, 1)) for j in range(W)], 1),
             torch.stack([(d_zm * line[:, j:j + T].abs()).sum((0, 1)) for j in range(W)], 1)), (d_z.sum((0, 1)), d_zm.sum((0, 1)))]
    first = None
    for _ in range(3):
        got = [p.forward()[0], *p.backward()[:3]]
        first = first or got
        assert all(torch.equal(a, c) for a, c in zip(first, got))
    for i, (g, (r, m)) in enumerate(zip(got, want)):
        n = 2 * W + 128 + (B * T if i > 1 else 0)
        limit = n * U * m + (2.0 ** -8 * r.abs() if dtype == BF16 and i < 2 else 0)
        assert ((g.double() - r).abs() <= limit).all(), i


@gpu
def test_same_bits_on_another_stream_and_in_a_graph():
    p = Problem(BF16, 2, 300, 70, 4, lengths=[300, 123])
    want = [*p.forward(), *p.backward()]
    got = [torch.empty_like(t) for t in want]
    x, d_y, w, b, n, before, d_after, ws = (cuda(t) for t in (p.x, p.d_y, p.w, p.b, p.lengths, p.before, p.d_after, p.workspace()))

    def call():
        mdh.mdh_causal_conv(x, w, b, got[0], mdh.MDH_ACT_SILU, n, before, got[1])
        mdh.mdh_causal_conv_backward(x, w, b, d_y, got[2], got[3], got[4], mdh.MDH_ACT_SILU, n, before, d_after, got[5], ws)

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


# ------------------------------------------------------------------ refusals: nothing is launched


def _raw(sizes, dtype=0, x=64, w=64, y=64, act=2, strides=None, after=None, slots=None, n=0):
    S = mdh.binding._sizes
    return mdh.lib().mdh_causal_conv(S(sizes), dtype, x, None if strides is None else S(strides), w, None, act, None, None, after, slots, n, y, None)


def _back(sizes, x=64, d_y=64, d_x=64, w=64, ws=1 << 20, nws=1 << 50, strides=None, d_after=None, d_before=None):
    S = mdh.binding._sizes
    return mdh.lib().mdh_causal_conv_backward(S(sizes), 0, x, d_y, None if strides is None else S(strides), w, None, 2, None, None, d_after,
                                              d_x, d_before, None, None, ws, nws, None)


def test_refuses_outputs_whose_rows_overlap():
    ok = (2, 5, 16, 4)
    for strides in ([80, 16, 80, 15], [80, 16, 15, 16], [80, 16, 80, -15]):
        assert _raw(ok, strides=strides) == E_SIZE
    assert _back(ok, strides=[80, 16, 80, 16, 80, 15]) == E_SIZE and _back(ok, strides=[80, 16, 80, 16, 15, 16]) == E_SIZE


def test_refuses_outputs_in_place():
    """A run of tokens reads rows of the one before it: y where x is, d_x where x or d_y is."""
    ok = (2, 500, 16, 4)
    for sizes in (ok, (1, 1, 1, 2), (2, 500, 16, 8)):
        for dtype in (0, 1):
            assert _raw(sizes, dtype=dtype, x=64, y=64) == E_UNSUP
        assert _back(sizes, x=64, d_y=128, d_x=64) == E_UNSUP and _back(sizes, x=64, d_y=128, d_x=128) == E_UNSUP
    wide = [500 * 40, 40] * 3
    assert _raw(ok, strides=wide[:4]) == E_UNSUP and _back(ok, strides=wide) == E_UNSUP
    assert _raw((2, 0, 16, 4)) == 0 and _raw((0, 5, 16, 4)) == 0  # no tokens


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_tap_in_place(dtype):
    p = Problem(dtype, 2, 300, 40, 1, windows=False)
    y, here = p.forward()[0], p.x.cuda()
    mdh.mdh_causal_conv(here, p.w.cuda(), p.b.cuda(), here, mdh.MDH_ACT_SILU)
    assert torch.equal(here, y)


def test_refusals():
    ok = (2, 5, 16, 4)
    for sizes in ((-1, 5, 16, 4), (2, -1, 16, 4), (2, 5, 0, 4), (2, 5, 16, 0), (1 << 16, 1 << 16, 16, 4), (2, 5, 1 << 24, 4), (1, (1 << 31) - 1, 8, 4)):
        assert _raw(sizes) == E_SIZE
    assert _raw((2, 5, 16, 9)) == E_UNSUP and _raw(ok, dtype=2) == E_UNSUP and _raw(ok, act=4) == E_UNSUP and _raw(ok, act=-1) == E_UNSUP
    assert _raw(ok, x=None) == E_NULL and _raw(ok, w=None) == E_NULL and _raw(ok, y=None) == E_NULL
    assert _raw(ok, x=66) == E_UNSUP and _raw(ok, dtype=1, y=65) == E_UNSUP and _raw(ok, w=62) == E_UNSUP and _raw(ok, after=66) == E_UNSUP
    assert _raw(ok, slots=64, n=-1) == E_SIZE
    assert _raw(ok, strides=[80, 16, 80, 0]) == E_SIZE and _raw(ok, strides=[80, 16, 0, 16]) == E_SIZE  # outputs on one another
    assert _raw((0, 5, 16, 4), x=None, y=None) == 0 and _raw((2, 0, 16, 4), x=None, y=None) == 0  # nothing to do
    assert _raw((1 << 12, 1 << 18, 1 << 12, 4)) == E_SIZE  # lanes of a launch
    need = mdh.mdh_causal_conv_workspace_size(ok, F32)
    assert need > 0 and _back(ok, ws=None) == E_WS and _back(ok, nws=need - 1) == E_WS and _back(ok, ws=(1 << 20) + 8) == E_WS
    for name in ("x", "d_y", "d_x", "w"):
        assert _back(ok, **{name: None}) == E_NULL
    assert _back(ok, strides=[80, 16, 80, 16, 80, 0]) == E_SIZE and _back(ok, d_after=64, d_before=64) == E_UNSUP
    step = lambda sizes, x=64, window=64, act=2: mdh.lib().mdh_causal_conv_step(mdh.binding._sizes(sizes), 0, x, None, 64, None, act, window, None, 0, 64,  # noqa: E731
                                                                                None)
    assert step((2, 0, 4)) == E_SIZE and step((2, 16, 9)) == E_UNSUP and step((2, 16, 4), act=9) == E_UNSUP
    assert step((2, 16, 4), x=None) == E_NULL and step((2, 16, 4), window=None) == E_NULL and step((0, 16, 4)) == 0


def test_binding_refuses_what_does_not_fit():
    x, w = torch.zeros(2, 5, 16), torch.zeros(16, 4)
    with pytest.raises(TypeError):
        mdh.mdh_causal_conv(x, w, None, x)  # not on the GPU
    with pytest.raises(ValueError):
        mdh.mdh_causal_conv(x, w, None, x[:, :3])
    with pytest.raises((TypeError, ValueError)):
        mdh.mdh_causal_conv(x, w[:8], None, x)
    with pytest.raises(ValueError):
        mdh.mdh_causal_conv(x, w, None, x, initial_window=torch.zeros(2, 4, 16))
    with pytest.raises(ValueError):
        mdh.mdh_causal_conv_backward(x, w, None, x, x[:1], None, None)
    with pytest.raises(ValueError):
        mdh.mdh_causal_conv_step(x[:, 0], w, None, torch.zeros(3, 3, 16), x[:, 0])
    with pytest.raises(TypeError):
        mdh.mdh_causal_conv_workspace_size((2, 5, 16, 4), torch.float64)
