"""Linear attention with a decay for each head: parity with the 64-bit oracle through the C ABI, at the sizes, strides, lengths
and values where it can go wrong, and what it refuses.

Limits.  Every output is a sum of products; ``mag`` is the same sum over absolute values.  In fp32 (u = 2^-24) a product and its
decays carry a few u, and n partial sums add n u at worst: |error| <= (dk + 2 T + 32) u mag; errors of random sign add as roots, so
the root mean square over all outputs stays below 2^-20 of theirs.  With bf16 operands a score or a state is rounded once (2^-8 of a
term) and the output once (2^-8 of it): 2^-7 mag more.  States are fp32 whatever the operands are.
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


def rand(seed, *shape, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype)


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def close(got, ref, mag, dtype, n, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), what
    limit = ((2.0 ** -7 if dtype == BF16 else 0) + n * U) * mag + 1e-37
    worst = np.max(np.abs(got - ref) / limit, initial=0)
    assert worst <= 1, "%s: %.2f times its limit" % (what, worst)
    rms = np.sqrt(np.mean((got - ref) ** 2)) if got.size else 0.0
    size = np.sqrt(np.mean(ref ** 2)) if got.size else 0.0
    assert rms <= (2.0 ** -7 if dtype == BF16 else 2.0 ** -20) * size, "%s: rms %.2g of %.2g" % (what, rms, size)


def decays(H, kind="mixed"):
    if kind == "none":
        return torch.zeros(H)
    if kind == "all":  # l = 0: no memory, and one head that forgets by thousands
        return torch.tensor([-float("inf")] * (H - 1) + [-3000.0])
    return torch.log1p(-torch.exp2(-torch.linspace(1, 9, H, dtype=torch.float64))).float()


class Problem:
    def __init__(self, dtype, B, T, H, dk, dv, Hq=None, Hk=None, Hv=None, lengths=None, states=True, decay="mixed", seed=0):
        self.dtype, self.B, self.T, self.H, self.dk, self.dv = dtype, B, T, H, dk, dv
        self.Hq, self.Hk, self.Hv = Hq or H, Hk or H, Hv or H
        self.scale = dk ** -0.5
        self.q, self.k = rand(seed + 1, B, T, self.Hq, dk, dtype=dtype), rand(seed + 2, B, T, self.Hk, dk, dtype=dtype)
        self.v, self.d_o = rand(seed + 3, B, T, self.Hv, dv, dtype=dtype), rand(seed + 4, B, T, H, dv, dtype=dtype)
        self.g = decays(H, decay)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
        self.S0, self.dS = (rand(seed + 5, B, H, dk, dv), rand(seed + 6, B, H, dk, dv)) if states else (None, None)
        self.sizes = (B, T, H, self.Hq, self.Hk, self.Hv, dk, dv)

    def args(self):
        return (*(np64(t) for t in (self.q, self.k, self.v)), np64(self.g))

    def lens(self):
        return None if self.lengths is None else self.lengths.numpy()

    def workspace(self, backward):
        n = mdh.mdh_linattn_workspace_size(self.sizes, self.dtype, backward)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None

    def forward(self, lay=lambda t: t.cuda(), out=None):
        o = torch.full((self.B, self.T, self.H, self.dv), float("nan"), dtype=self.dtype, device="cuda") if out is None else out
        final = torch.full((self.B, self.H, self.dk, self.dv), float("nan"), device="cuda")
        S0 = None if self.S0 is None else self.S0.cuda()
        mdh.mdh_linattn(lay(self.q), lay(self.k), lay(self.v), self.g.cuda(), o, self.scale,
                        None if self.lengths is None else self.lengths.cuda(), S0, final, workspace=self.workspace(False))
        return o, final

    def backward(self, lay=lambda t: t.cuda()):
        grads = [torch.full(t.shape, float("nan"), dtype=self.dtype, device="cuda") for t in (self.q, self.k, self.v)]
        dS0 = torch.full((self.B, self.H, self.dk, self.dv), float("nan"), device="cuda")
        S0, dS = (None if t is None else t.cuda() for t in (self.S0, self.dS))
        mdh.mdh_linattn_backward(lay(self.q), lay(self.k), lay(self.v), self.g.cuda(), lay(self.d_o), *grads, self.scale,
                                 None if self.lengths is None else self.lengths.cuda(), S0, dS, dS0, workspace=self.workspace(True))
        return (*grads, dS0)

    def check(self, backward=True, **kw):
        a, n = self.args(), self.dk + self.dv + 2 * self.T + 32
        S0, dS, d_o = np64(self.S0), np64(self.dS), np64(self.d_o)
        ref = O.linattn(*a, self.scale, self.lens(), S0)
        mag = O.linattn(*a, self.scale, self.lens(), S0, magnitude=True)
        o, final = self.forward(**kw)
        close(o, ref[0], mag[0], self.dtype, n, "o")
        close(final, ref[1], mag[1], F32, n, "final state")
        if not backward:
            return
        ref = O.linattn_backward(*a, d_o, self.scale, self.lens(), S0, dS)
        mag = O.linattn_backward(*a, d_o, self.scale, self.lens(), S0, dS, magnitude=True)
        for got, r, m, what in zip(self.backward(**kw), ref, mag, ("d_q", "d_k", "d_v", "d_initial_state")):
            close(got, r, m, F32 if what == "d_initial_state" else self.dtype, n * self.H, what)


# T around the sizes that a run of tokens may have, head widths that vector loads like and that they do not
SHAPES = [
    (1, 1, 1, 1, 1), (2, 1, 3, 64, 64), (1, 2, 2, 16, 8), (1, 31, 2, 32, 40), (2, 32, 1, 8, 8), (1, 33, 2, 64, 32), (1, 63, 1, 128, 128),
    (1, 64, 2, 64, 128), (2, 65, 2, 128, 64), (1, 129, 3, 80, 96), (1, 200, 2, 17, 31), (1, 257, 1, 256, 256), (1, 130, 1, 129, 250),
    (2, 300, 2, 100, 36), (1, 96, 2, 256, 24), (1, 70, 2, 24, 256), (1, 190, 1, 160, 144),
]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,H,dk,dv", SHAPES)
def test_parity(dtype, B, T, H, dk, dv):
    Problem(dtype, B, T, H, dk, dv, seed=T).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Hq,Hk,Hv", [(2, 2, 6), (6, 3, 3), (1, 1, 1), (6, 1, 2)])
def test_shared_heads(dtype, Hq, Hk, Hv):
    Problem(dtype, 2, 75, 6, 48, 40, Hq, Hk, Hv, lengths=[75, 66]).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths", [[0, 150, 1, 64], [150, 65, 149, 128], [0, 0, 0, 0], [-3, 1000, 63, 2]])
def test_lengths_with_anything_behind_them(dtype, lengths):
    """Tokens past an entry's length hold NaN and infinities: nothing of them is read, their outputs and gradients are 0."""
    p = Problem(dtype, 4, 150, 2, 40, 72, lengths=lengths)
    for b, n in enumerate(min(max(n, 0), 150) for n in lengths):
        for t, bad in ((p.q, float("nan")), (p.k, float("inf")), (p.v, float("nan")), (p.d_o, -float("inf"))):
            t[b, n:] = bad
    p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("decay", ["none", "all"])
def test_decays_of_one_and_of_zero(dtype, decay):
    Problem(dtype, 1, 140, 3, 32, 64, decay=decay).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_states(dtype):
    Problem(dtype, 2, 100, 2, 64, 64, states=False).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_long_sequence(dtype):
    """Long enough that one head's tokens are worked on in several places at once."""
    Problem(dtype, 1, 2500, 1, 64, 32, seed=7).check()
    Problem(dtype, 2, 1500, 1, 40, 72, lengths=[1500, 700], seed=8).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    """Slices of one projection; heads before tokens; rows at odd places; one token's values for all tokens."""
    p = Problem(dtype, 2, 70, 3, 40, 40)

    def fused(t):
        wide = torch.full((*t.shape[:3], 3, t.shape[3]), float("nan"), dtype=dtype, device="cuda")
        wide[:, :, :, 1] = t.cuda()
        return wide[:, :, :, 1]

    def heads_first(t):
        return t.cuda().transpose(1, 2).contiguous().transpose(1, 2)

    def odd(t):
        wide = torch.full((*t.shape[:3], t.shape[3] + 3), float("nan"), dtype=dtype, device="cuda")
        wide[..., 1:-2] = t.cuda()
        return wide[..., 1:-2]

    for lay in (fused, heads_first, odd):
        p.check(lay=lay)
    o = fused(torch.zeros(2, 70, 3, 40, dtype=dtype))
    plain, _ = p.forward()
    p.forward(out=o)
    assert torch.equal(o, plain)
    p.k = p.k[:, :1].expand(p.k.shape)
    p.check(lay=lambda t: t[:, :1].cuda().expand(t.shape) if t.stride(1) == 0 else t.cuda())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_tokens(dtype):
    """T = 0: the state passes through."""
    p = Problem(dtype, 2, 0, 2, 16, 24)
    _, final = p.forward()
    assert torch.equal(final.cpu(), p.S0)
    assert torch.equal(p.backward()[3].cpu(), p.dS)
    p = Problem(dtype, 0, 5, 2, 16, 24)
    p.forward(), p.backward()


@gpu
@pytest.mark.parametrize("T", [70, 1300])
def test_states_in_place_and_in_slots(T):
    p = Problem(BF16, 3, T, 2, 64, 64)
    o, final = p.forward()
    state, o2 = p.S0.cuda(), torch.empty_like(o)
    mdh.mdh_linattn(p.q.cuda(), p.k.cuda(), p.v.cuda(), p.g.cuda(), o2, p.scale, None, state, state, workspace=p.workspace(False))
    assert torch.equal(o, o2) and torch.equal(state, final)
    pool = rand(9, 7, 2, 64, 64).cuda()
    before = pool.clone()
    pool[5], pool[2] = p.S0[0].cuda(), p.S0[2].cuda()
    slots = torch.tensor([5, -1, 2], dtype=torch.int32, device="cuda")
    mdh.mdh_linattn(p.q.cuda(), p.k.cuda(), p.v.cuda(), p.g.cuda(), o2, p.scale, None, pool, pool, slots, p.workspace(False))
    assert torch.equal(pool[5], final[0]) and torch.equal(pool[2], final[2])
    assert torch.equal(o2[0], o[0]) and torch.equal(o2[2], o[2])
    rest = [0, 1, 3, 4, 6]
    assert torch.equal(pool[rest], before[rest])
    p.S0[1] = 0  # an entry without a slot begins with zeros
    assert torch.equal(p.forward()[0][1], o2[1])
    slots[1] = 7  # and one past the pool has none
    mdh.mdh_linattn(p.q.cuda(), p.k.cuda(), p.v.cuda(), p.g.cuda(), o, p.scale, None, None, pool, slots, p.workspace(False))
    assert torch.equal(pool[rest], before[rest])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,dk,dv", [(1, 1, 1, 1), (3, 4, 64, 64), (2, 6, 128, 128), (5, 2, 80, 96), (2, 2, 17, 31), (300, 4, 32, 24),
                                       (2, 1, 256, 256), (1, 2, 129, 252)])
def test_step(dtype, B, H, dk, dv):
    few = H // 2 if H % 2 == 0 else H
    p = Problem(dtype, B, 1, H, dk, dv, few, H, few)
    a = p.args()
    (o, S), (mo, mS) = O.linattn(*a, p.scale, None, np64(p.S0)), O.linattn(*a, p.scale, None, np64(p.S0), magnitude=True)
    state, got = p.S0.cuda(), torch.full((B, H, dv), float("nan"), dtype=dtype, device="cuda")
    mdh.mdh_linattn_step(p.q[:, 0].cuda(), p.k[:, 0].cuda(), p.v[:, 0].cuda(), p.g.cuda(), state, got, p.scale)
    close(got, o[:, 0], mo[:, 0], dtype, dk + 32, "o")
    close(state, S, mS, F32, 32, "state")


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,H,dk,dv", [(90, 3, 40, 128), (170, 2, 256, 100), (600, 1, 3, 4), (128, 1, 16, 256)])
def test_step_of_many_states(dtype, B, H, dk, dv):
    p = Problem(dtype, B, 1, H, dk, dv)
    a = p.args()
    (o, S), (mo, mS) = O.linattn(*a, p.scale, None, np64(p.S0)), O.linattn(*a, p.scale, None, np64(p.S0), magnitude=True)
    state, got = p.S0.cuda(), torch.full((B, H, dv), float("nan"), dtype=dtype, device="cuda")
    mdh.mdh_linattn_step(p.q[:, 0].cuda(), p.k[:, 0].cuda(), p.v[:, 0].cuda(), p.g.cuda(), state, got, p.scale)
    close(got, o[:, 0], mo[:, 0], dtype, dk + 32, "o")
    close(state, S, mS, F32, 32, "state")


@gpu
def test_step_in_slots_and_strides():
    p = Problem(BF16, 4, 1, 3, 32, 48)
    q, k, v = (t[:, 0].cuda() for t in (p.q, p.k, p.v))
    o, state = torch.empty(4, 3, 48, dtype=BF16, device="cuda"), p.S0.cuda()
    mdh.mdh_linattn_step(q, k, v, p.g.cuda(), state, o, p.scale)
    pool = rand(3, 9, 3, 32, 48).cuda()
    before = pool.clone()
    slots = torch.tensor([8, -1, 0, 9], dtype=torch.int32, device="cuda")
    pool[8], pool[0] = p.S0[0].cuda(), p.S0[2].cuda()
    wide = torch.full((4, 3, 80), float("nan"), dtype=BF16, device="cuda")
    wide[..., 3:35] = k
    o2 = torch.full((4, 6, 48), float("nan"), dtype=BF16, device="cuda")[:, ::2]
    mdh.mdh_linattn_step(q, wide[..., 3:35], v, p.g.cuda(), pool, o2, p.scale, slots)
    assert torch.equal(o2[0], o[0]) and torch.equal(o2[2], o[2]) and not o2[1].any() and not o2[3].any()
    assert torch.equal(pool[8], state[0]) and torch.equal(pool[0], state[2])
    assert torch.equal(pool[1:8], before[1:8])


@gpu
def test_step_past_2_31_elements():
    """The last slot of a pool of 9 GB: its offset in elements does not fit 32 bits."""
    H, d, n = 4, 128, 33000
    pool = torch.empty(n, H, d, d, device="cuda")
    assert pool.numel() > 1 << 31
    slots = torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    p = Problem(F32, 1, 1, H, d, d)
    pool[n - 1] = p.S0[0].cuda()
    o, state, o2 = torch.empty(1, H, d, device="cuda"), p.S0.cuda(), torch.empty(1, H, d, device="cuda")
    q, k, v = (t[:, 0].cuda() for t in (p.q, p.k, p.v))
    mdh.mdh_linattn_step(q, k, v, p.g.cuda(), pool, o, p.scale, slots)
    mdh.mdh_linattn_step(q, k, v, p.g.cuda(), state, o2, p.scale)
    assert torch.equal(o, o2) and torch.equal(pool[n - 1], state[0])


@gpu
def test_prompt_then_tokens():
    """A prompt and the tokens after it, one at a time, are one sequence."""
    p = Problem(F32, 2, 90, 2, 64, 64, states=False)
    whole, last = p.forward()
    state = torch.empty_like(last)
    first = Problem(F32, 2, 90, 2, 64, 64, states=False)
    q, k, v = (t.cuda() for t in (p.q, p.k, p.v))
    o = torch.empty(2, 85, 2, 64, device="cuda")
    first.T, first.sizes = 85, (2, 85, 2, 2, 2, 2, 64, 64)
    mdh.mdh_linattn(q[:, :85], k[:, :85], v[:, :85], p.g.cuda(), o, p.scale, None, None, state, workspace=first.workspace(False))
    parts = [o]
    for t in range(85, 90):
        one = torch.empty(2, 2, 64, device="cuda")
        mdh.mdh_linattn_step(q[:, t], k[:, t], v[:, t], p.g.cuda(), state, one, p.scale)
        parts.append(one[:, None])
    mag = O.linattn(*p.args(), p.scale, magnitude=True)
    close(torch.cat(parts, 1), np64(whole), 2 * mag[0], F32, p.dk + 2 * p.T + 32, "o")
    close(state, np64(last), 2 * mag[1], F32, p.dk + 2 * p.T + 32, "state")


@gpu
def test_gradients_against_differences():
    """The kernels' gradients along random directions against differences of the oracle's forward function."""
    p = Problem(F32, 1, 100, 2, 24, 40, Hk=1, lengths=[97])
    grads = [np64(t) for t in p.backward()]
    at = [np64(t) for t in (p.q, p.k, p.v, p.S0)]

    def loss(x):
        o, final = O.linattn(x[0], x[1], x[2], np64(p.g), p.scale, [97], x[3])
        return (o * np64(p.d_o)).sum() + (final * np64(p.dS)).sum()

    rng = np.random.default_rng(1)
    for i in range(4):
        d, h = rng.standard_normal(at[i].shape), 1e-5
        up, down = ([x + s * d if j == i else x for j, x in enumerate(at)] for s in (h, -h))
        want = (loss(up) - loss(down)) / (2 * h)
        # the loss is linear in each operand: the difference is exact but for 64-bit rounding
        assert abs((grads[i] * d).sum() - want) <= 2e-5 * np.abs(grads[i] * d).sum()


@gpu
def test_same_bits_on_another_stream_and_in_a_graph():
    p = Problem(BF16, 2, 1100, 2, 64, 64, Hk=1)
    o, final = p.forward()
    grads = p.backward()
    args = [t.cuda() for t in (p.q, p.k, p.v, p.g)]
    S0, dS, d_o = p.S0.cuda(), p.dS.cuda(), p.d_o.cuda()
    o2, final2, g2 = torch.empty_like(o), torch.empty_like(final), [torch.empty_like(t) for t in grads]
    ws = p.workspace(True)

    def call():
        mdh.mdh_linattn(*args, o2, p.scale, None, S0, final2, workspace=ws)
        mdh.mdh_linattn_backward(*args, d_o, *g2[:3], p.scale, None, S0, dS, g2[3], workspace=ws)

    def same():
        return torch.equal(o, o2) and torch.equal(final, final2) and all(torch.equal(a, b) for a, b in zip(grads, g2))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in (o2, final2, *g2):
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert same()


def _pairs(p, magnitude):
    """o and the gradients in 64 bits on the GPU, from the products of all pairs of tokens (no shared heads, no states)."""
    f = torch.abs if magnitude else (lambda t: t)
    q, k, v, d_o = (f(t.cuda().double()).transpose(1, 2).contiguous() for t in (p.q, p.k, p.v, p.d_o))
    i = torch.arange(p.T, device="cuda")
    near = torch.where(i[:, None] >= i, torch.exp(p.g.cuda().double()[:, None, None] * (i[:, None] - i).clamp_min(0)), 0.0) * p.scale
    scores, d_scores = (q @ k.transpose(2, 3).contiguous()) * near, (d_o @ v.transpose(2, 3).contiguous()) * near
    turn = lambda t: t.transpose(2, 3).contiguous()  # noqa: E731
    got = scores @ v, d_scores @ k, turn(d_scores) @ q, turn(scores) @ d_o
    return [t.transpose(1, 2) for t in got]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,H,dk,dv", [(4, 1024, 16, 128, 128), (4, 1000, 16, 100, 90), (8, 512, 16, 64, 64), (2, 1024, 16, 64, 128),
                                         (4, 512, 12, 192, 256), (6, 700, 16, 63, 33)])
def test_chip_full_of_work(dtype, B, T, H, dk, dv):
    """Every output, with every compute unit busy: three calls in a row, each compared."""
    p = Problem(dtype, B, T, H, dk, dv, states=False)
    ref, mag = _pairs(p, False), _pairs(p, True)
    n = dk + dv + 2 * T + 32
    for _ in range(3):
        o, _ = p.forward()
        for got, r, m, what in zip((o, *p.backward()[:3]), ref, mag, ("o", "d_q", "d_k", "d_v")):
            limit = ((2.0 ** -7 if dtype == BF16 else 0) + n * U) * m + 1e-37
            off = (got.double() - r).abs()
            assert (off <= limit).all(), "%s: %.2f times its limit, %d outputs" % (what, (off / limit).max(), int((off > limit).sum()))
            assert off.square().mean().sqrt() <= (2.0 ** -7 if dtype == BF16 else 2.0 ** -20) * r.square().mean().sqrt(), what


# ------------------------------------------------------------------ refusals: nothing is launched


def _raw(sizes, dtype=0, q=64, strides=None, decay=64, o=64, final=None, initial=None, ws=None, nws=0, slots=None, n=0):
    """mdh_linattn on made-up addresses, for calls that are refused before one is used."""
    B = mdh.binding
    st = None if strides is None else B._sizes(strides)
    return mdh.lib().mdh_linattn(B._sizes(sizes), dtype, q, 64, 64, st, decay, 1.0, None, initial, final, slots, n, o, ws, nws, None)


def test_refusals():
    ok = (1, 8, 4, 4, 2, 1, 16, 16)
    assert _raw((1, -1) + ok[2:]) == E_SIZE and _raw((-1,) + ok[1:]) == E_SIZE
    for i in range(2, 8):
        assert _raw(ok[:i] + (0,) + ok[i + 1:]) == E_SIZE
    assert _raw((1, 8, 4, 3, 2, 1, 16, 16)) == E_SIZE  # three heads of q for four
    assert _raw((1, 8, 4, 4, 4, 4, 257, 16)) == E_UNSUP and _raw((1, 8, 4, 4, 4, 4, 16, 300)) == E_UNSUP
    assert _raw(ok, dtype=2) == E_UNSUP
    assert _raw(ok, q=None) == E_NULL and _raw(ok, o=None) == E_NULL and _raw(ok, decay=None) == E_NULL
    assert _raw(ok, q=66) == E_UNSUP and _raw(ok, final=72) == E_UNSUP and _raw(ok, initial=8) == E_UNSUP
    assert _raw(ok, slots=64, n=-1) == E_SIZE
    assert _raw(ok, strides=[512, 64, 16, 256, 32, 16, 128, 16, 16, 512, 0, 16]) == E_SIZE  # outputs on one another
    assert _raw((0,) + ok[1:], q=None, o=None) == 0  # nothing to do
    lib, S = mdh.lib(), mdh.binding._sizes
    back = lambda sizes, ws, n: lib.mdh_linattn_backward(S(sizes), 0, 64, 64, 64, 64, None, 64, 1.0, None, None, None, 64, 64, 64, None,  # noqa: E731
                                                         ws, n, None)
    need = mdh.mdh_linattn_workspace_size(ok, F32, True)
    assert need > 0 and back(ok, None, 0) == E_WS and back(ok, 64, need - 1) == E_WS and back(ok, 72, need) == E_WS
    step = lambda sizes, state=64, q=64: lib.mdh_linattn_step(S(sizes), 0, q, 64, 64, None, 64, 1.0, state, None, 0, 64, None)  # noqa: E731
    assert step((1, 4, 4, 4, 4, 16, 0)) == E_SIZE and step((1, 4, 3, 4, 4, 16, 16)) == E_SIZE and step((1, 4, 4, 4, 4, 16, 512)) == E_UNSUP
    assert step((1, 4, 4, 4, 4, 16, 16), state=None) == E_NULL and step((1, 4, 4, 4, 4, 16, 16), q=None) == E_NULL


def test_more_lanes_than_a_launch_has_are_refused():
    many = 1 << 24
    assert _raw((many, 1, 1, 1, 1, 1, 16, 16)) == E_SIZE and _raw((many // 2, 1, 1, 1, 1, 1, 16, 256)) == E_SIZE
    S = mdh.binding._sizes
    assert mdh.lib().mdh_linattn_step(S((many // 2, 2, 2, 2, 2, 16, 16)), 0, 64, 64, 64, None, 64, 1.0, 64, None, 0, 64, None) == E_SIZE


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(1, 4, 2, 8)
    g = torch.zeros(2)
    with pytest.raises(TypeError):
        mdh.mdh_linattn(x, x, x, g, x)  # not on the GPU
    with pytest.raises(ValueError):
        mdh.mdh_linattn(x, x[:, :3], x, g, x)
    with pytest.raises(ValueError):
        mdh.mdh_linattn_backward(x, x, x, g, x, x[:, :3], x, x)
    with pytest.raises(ValueError):
        mdh.mdh_linattn_step(x[:, 0], x[:, 0, :, :4], x[:, 0], g, torch.zeros(1, 2, 8, 8), x[:, 0])
    with pytest.raises(TypeError):
        mdh.mdh_linattn_workspace_size((1, 4, 2, 2, 2, 2, 8, 8), torch.float64)


@pytest.mark.parametrize("sizes", [(1, 64, 40000, 1, 40000, 40000, 256, 8), (1, 2, 40000, 40000, 1, 40000, 256, 8), (1, 64, 40000, 40000, 40000, 2, 8, 256)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_shared_heads_whose_sums_are_out_of_reach_are_refused(sizes, dtype):
    """64 tokens of the fp32 gradients of all heads take more than 2^31 bytes, though no operand does."""
    S = mdh.binding._sizes
    strides = S([x for heads, d in zip((*sizes[3:6], sizes[2], *sizes[3:6]), (8, 8, 8, 8, 256, 256, 256)) for x in (1 << 24, 1 << 17, d if heads > 1 else 0)])
    assert mdh.lib().mdh_linattn_backward(S(sizes), dtype, 64, 64, 64, 64, strides, 64, 1.0, None, None, None, 64, 64, 64, None, 1 << 20, 1 << 60,
                                          None) == E_SIZE


# rows of less than 16 bytes on either side of the state, which are read element by element (heads of 5 and 7: in bf16 only)
NARROW = [(2, 130, 2, 3, 3, [130, 65]), (1, 70, 1, 3, 256, None), (1, 70, 1, 200, 5, [67]), (1, 2500, 1, 3, 5, None),
          (3, 1500, 1, 5, 2, [1500, 0, 999]), (2, 100, 3, 100, 3, [33, 100]), (1, 129, 2, 1, 140, None), (2, 66, 1, 256, 1, [64, 66]),
          (1, 700, 2, 7, 70, [650])]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,H,dk,dv,lengths", NARROW)
def test_narrow_heads(dtype, B, T, H, dk, dv, lengths):
    p = Problem(dtype, B, T, H, dk, dv, lengths=lengths, seed=T)
    for b, n in enumerate(lengths or []):
        for t in (p.q, p.k, p.v, p.d_o):
            t[b, n:] = float("nan")
    p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,Hq,Hk,Hv,dk,dv", [(2, 1600, 2, 2, 6, 48, 40), (1, 1500, 6, 1, 2, 64, 24), (2, 1700, 1, 3, 1, 5, 6)])
def test_shared_heads_in_segments(dtype, B, T, Hq, Hk, Hv, dk, dv):
    """Sums over shared heads of gradients that several workgroups have made, one after another along the tokens."""
    p = Problem(dtype, B, T, 6, dk, dv, Hq, Hk, Hv, lengths=[T - 90, T][:B])
    assert mdh.mdh_linattn_workspace_size(p.sizes, dtype, False) > 0  # the states between segments
    p.check()
