"""The selective state space scan: parity with the 64-bit oracle through the C ABI, at the sizes, groups, strides, lengths and values
where it can go wrong, and what it refuses.

Limits.  u = 2^-24; ``mag`` is the same sum over absolute values.  A step's factor e^(delta A) is off by 2 u (the exponential) and 2 u of
its exponent, products and sums by u each: a term that lives for n steps by 3 n u, and by 2 u of its whole exponent, which is 40 at
most where the term counts (e^-40 is below u^2).  delta is off by 8 u, which such an exponent multiplies again: 320 u.  Sums over N
states, the gate's 40 u (|gate| <= 8) and a few more products: (3 T + N + 500) u mag in all, and u for every term of sums over tokens
or channels.  Errors of random sign add as roots: 64 u of the root mean square.  A rounding to bf16 is 2^-8 of the value.
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
GRADS = ("d_x", "d_dt", "d_b", "d_c", "d_gate", "d_A", "d_skip", "d_dt_bias", "d_initial")
IN_TYPE = GRADS[:5]


def rand(seed, *shape, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def np64(t):
    return None if t is None else t.double().cpu().numpy()


def cuda(t):
    return None if t is None else t.cuda()


def close(got, ref, mag, half, n, what):
    got = np64(got)
    assert np.isfinite(got).all(), what
    limit = n * U * mag + (2.0 ** -8 * np.abs(ref) if half else 0) + 1e-37
    worst = np.max(np.abs(got - ref) / limit, initial=0)
    assert worst <= 1, "%s: %.2f times its limit" % (what, worst)
    rms, size = (np.sqrt(np.mean(v ** 2)) if got.size else 0.0 for v in (got - ref, mag))
    assert rms <= (2.0 ** -8 if half else 2.0 ** -18) * size, "%s: rms %.2g of %.2g" % (what, rms, size)


class Problem:
    def __init__(self, dtype, B, T, D, N, G=1, gate=True, softplus=True, skip=True, dt_bias=True, states=True, lengths=None, seed=0):
        self.dtype, self.B, self.T, self.D, self.N, self.G, self.softplus = dtype, B, T, D, N, G, softplus
        self.x, self.gate = rand(seed + 1, B, T, D, dtype=dtype), rand(seed + 2, B, T, D, dtype=dtype) if gate else None
        self.dt = rand(seed + 3, B, T, D, dtype=dtype) if softplus else (0.5 * rand(seed + 3, B, T, D).abs()).to(dtype)
        self.b, self.c = rand(seed + 4, B, T, G, N, dtype=dtype), rand(seed + 5, B, T, G, N, dtype=dtype)
        # memories of one to a hundred time steps
        self.A = -torch.exp(torch.linspace(-4, 1, N) + 0.3 * rand(seed + 6, D, N))
        self.skip, self.dt_bias = rand(seed + 7, D) if skip else None, 0.3 * rand(seed + 8, D) - 1 if dt_bias and softplus else None
        self.h0, self.dh = (rand(seed + i, B, D, N) if states else None for i in (9, 10))
        self.d_y = rand(seed + 11, B, T, D, dtype=dtype)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)

    def sizes(self):
        return self.B, self.T, self.D, self.N, self.G

    def empty(self, *shape, dtype=None):
        return torch.full(shape, NAN, dtype=dtype or self.dtype, device="cuda")

    def buffers(self, backward=True):
        n, k = mdh.mdh_selective_scan_workspace_size(self.sizes(), self.dtype, backward), mdh.mdh_selective_scan_checkpoints_size(self.sizes())
        return [torch.full((m,), 255, dtype=torch.uint8, device="cuda") if m else None for m in (n, k)]

    def rest(self, lay):
        return dict(skip=cuda(self.skip), gate=None if self.gate is None else lay(self.gate), dt_bias=cuda(self.dt_bias),
                    softplus=self.softplus, lengths=cuda(self.lengths))

    def forward(self, lay=cuda, y=None, checkpoints=None, workspace=None):
        y = self.empty(self.B, self.T, self.D) if y is None else y
        final = self.empty(self.B, self.D, self.N, dtype=F32)
        ws = self.buffers(False)[0] if workspace is None else workspace
        mdh.mdh_selective_scan(lay(self.x), lay(self.dt), self.A.cuda(), lay(self.b), lay(self.c), y, initial_state=cuda(self.h0),
                               final_state=final, checkpoints=checkpoints, workspace=ws, **self.rest(lay))
        return y, final

    def backward(self, lay=cuda, checkpoints=None, workspace=None, out=None):
        """Gradients in the order of GRADS (d_gate: None without a gate)."""
        if checkpoints is None:
            workspace, checkpoints = self.buffers()
            self.forward(lay, checkpoints=checkpoints, workspace=workspace)
        g = dict(d_x=self.empty(*self.x.shape), d_dt=self.empty(*self.x.shape), d_b=self.empty(*self.b.shape), d_c=self.empty(*self.b.shape),
                 d_gate=None if self.gate is None else self.empty(*self.x.shape), d_A=self.empty(self.D, self.N, dtype=F32),
                 d_skip=self.empty(self.D, dtype=F32), d_dt_bias=self.empty(self.D, dtype=F32),
                 d_initial=self.empty(self.B, self.D, self.N, dtype=F32))
        g.update(out or {})
        mdh.mdh_selective_scan_backward(lay(self.x), lay(self.dt), self.A.cuda(), lay(self.b), lay(self.c), lay(self.d_y), g["d_x"], g["d_dt"],
                                        g["d_A"], g["d_b"], g["d_c"], checkpoints, d_final_state=cuda(self.dh), d_skip=g["d_skip"],
                                        d_gate=g["d_gate"], d_dt_bias=g["d_dt_bias"], d_initial_state=g["d_initial"], workspace=workspace,
                                        **self.rest(lay))
        return [g[n] for n in GRADS]

    def oracle(self):
        return ((np64(self.x), np64(self.dt), np64(self.A), np64(self.b), np64(self.c)),
                dict(skip=np64(self.skip), gate=np64(self.gate), dt_bias=np64(self.dt_bias), softplus=self.softplus,
                     lengths=None if self.lengths is None else self.lengths.numpy(), initial=np64(self.h0)))

    def check(self, backward=True, **kw):
        a, k = self.oracle()
        n = 3 * self.T + self.N + 500
        half = self.dtype == BF16
        (ry, rf), (my, mf) = O.selective_scan(*a, **k), O.selective_scan(*a, **k, magnitude=True)
        y, final = self.forward(**kw)
        close(y, ry, my, half, n, "y")
        close(final, rf, mf, False, n, "final state")
        if not backward:
            return
        args = (*a, np64(self.d_y))
        ref, mag = (O.selective_scan_backward(*args, **k, d_final=np64(self.dh), magnitude=m) for m in (False, True))
        n = 2 * n + self.B * self.T + self.D
        for got, name in zip(self.backward(**kw), GRADS):
            if got is not None:
                close(got, ref[name], mag[name], half and name in IN_TYPE, n, name)


# T around the tiles of tokens, D around the channels of workgroups, N around the states of lanes
SHAPES = [(1, 1, 1, 1, 1), (2, 1, 16, 16, 1), (1, 2, 17, 16, 1), (3, 15, 5, 3, 1), (1, 16, 64, 16, 1), (2, 17, 65, 16, 1), (1, 33, 130, 8, 2),
          (2, 40, 36, 17, 4), (1, 50, 66, 24, 2), (2, 31, 20, 32, 1), (1, 64, 24, 33, 8), (2, 47, 40, 64, 1), (1, 70, 12, 48, 3), (4, 100, 96, 16, 1),
          (1, 200, 3, 5, 3), (1, 90, 200, 16, 1)]


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,D,N,G", SHAPES)
def test_parity(dtype, B, T, D, N, G):
    Problem(dtype, B, T, D, N, G, seed=T).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("left_out", [dict(gate=False), dict(softplus=False), dict(skip=False, dt_bias=False), dict(states=False),
                                      dict(gate=False, softplus=False, skip=False, states=False)])
def test_what_may_be_left_out(dtype, left_out):
    Problem(dtype, 2, 45, 40, 16, 2, **left_out).check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,lengths", [(70, [0, 70, 1, 16]), (70, [69, 33, 32, 17]), (70, [0, 0, 0, 0]), (70, [-3, 1000, 15, 48]),
                                       (900, [900, 130, 0, 513])])
def test_lengths_with_anything_behind_them(dtype, T, lengths):
    """Tokens past an entry's length hold NaN and infinities: nothing of them is read, their outputs and gradients are 0."""
    p = Problem(dtype, 4, T, 20, 16, 2, lengths=lengths)
    for i, n in enumerate(min(max(n, 0), T) for n in lengths):
        for t, bad in ((p.x, NAN), (p.dt, float("inf")), (p.b, NAN), (p.c, -float("inf")), (p.gate, NAN), (p.d_y, float("inf"))):
            t[i, n:] = bad
    p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_time_steps_of_zero_and_of_thousands(dtype):
    """Softplus far to both sides: a token that changes nothing, one that forgets everything; and states without decay."""
    p = Problem(dtype, 1, 40, 18, 16)
    p.dt[:, ::3], p.dt[:, 1::7], p.dt[:, 5] = -200.0, 40.0, 3000.0
    p.x[:, 5], p.dt[:, 8] = p.x[:, 5] * 1e-3, 21.0
    p.A[:, 0], p.A[3] = 0.0, -1e-3
    p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("mask", ["-inf", "lowest"])
@pytest.mark.parametrize("B,T,D,N,G", [(2, 50, 20, 16, 2), (1, 40, 18, 40, 1), (1, 1300, 20, 16, 1)])
def test_masked_time_steps(dtype, mask, B, T, D, N, G):
    """Tokens whose dt is -infinity or the type's lowest value, which softplus makes 0: the state stays, dt's gradient is 0."""
    low = -float("inf") if mask == "-inf" else torch.finfo(dtype).min
    p = Problem(dtype, B, T, D, N, G)
    p.dt[:, ::3], p.dt[:, 17:38, :5] = low, low
    p.check()
    assert not p.backward()[1][:, ::3].any()
    p.dt[:] = low
    p.check()
    assert torch.equal(p.forward()[1].cpu(), p.h0)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low", [-float("inf"), None])
@pytest.mark.parametrize("N", [16, 18])
def test_step_with_a_masked_time_step(dtype, low, N):
    p = Problem(dtype, 3, 1, 30, N)
    p.dt[1], p.dt[2, :, :7] = (torch.finfo(dtype).min if low is None else low,) * 2
    a, k = p.oracle()
    (ry, rf), (my, mf) = O.selective_scan(*a, **k), O.selective_scan(*a, **k, magnitude=True)
    state, y = p.h0.cuda(), p.empty(3, 30)
    mdh.mdh_selective_scan_step(*(t[:, 0].cuda() if t is not p.A else t.cuda() for t in (p.x, p.dt, p.A, p.b, p.c)), state, y, p.skip.cuda(),
                                p.gate[:, 0].cuda(), p.dt_bias.cuda(), True)
    close(y, ry[:, 0], my[:, 0], dtype == BF16, N + 503, "y")
    close(state, rf, mf, False, 503, "state")
    assert torch.equal(state[1].cpu(), p.h0[1]) and torch.equal(state[2, :7].cpu(), p.h0[2, :7])


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,D,N,G", [(2, 50, 20, 18, 2), (1, 40, 18, 40, 1), (1, 1300, 20, 16, 1), (3, 1, 30, 16, 1), (3, 1, 30, 18, 1)])
def test_largest_time_steps_and_decays(dtype, B, T, D, N, G):
    """Time steps and decays of the largest numbers: a token that resets all states but those without decay, states that live for one token
    only or for those with a time step of 0."""
    p = Problem(dtype, B, T, D, N, G)
    p.dt[:, 5::11], p.dt[:, ::4] = torch.finfo(dtype).max, -float("inf")
    p.x[:, 5::11] = 0
    p.A[:, 0], p.A[3] = 0.0, torch.finfo(F32).min
    p.check(backward=False)
    p.A[6, 1] = NAN  # (weights that are no numbers show)
    assert p.forward()[0][..., 6].isnan().all()
    p.A[6, 1] = -1.0
    if T == 1:
        a, k = p.oracle()
        (ry, rf), (my, mf) = O.selective_scan(*a, **k), O.selective_scan(*a, **k, magnitude=True)
        state, y = p.h0.cuda(), p.empty(B, D)
        mdh.mdh_selective_scan_step(*(t[:, 0].cuda() if t is not p.A else t.cuda() for t in (p.x, p.dt, p.A, p.b, p.c)), state, y, p.skip.cuda(),
                                    p.gate[:, 0].cuda(), p.dt_bias.cuda(), True)
        close(y, ry[:, 0], my[:, 0], dtype == BF16, N + 503, "y")
        close(state, rf, mf, False, 503, "state")


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,D,N,G", [(1, 2500, 8, 16, 1), (2, 1111, 20, 7, 2), (1, 1300, 33, 40, 1)])
def test_long_sequences(dtype, B, T, D, N, G):
    """Long enough that one channel's tokens are worked on in several places at once."""
    p = Problem(dtype, B, T, D, N, G, lengths=[T - 333, T][-B:], seed=T)
    assert mdh.mdh_selective_scan_workspace_size(p.sizes(), dtype, False) > 0
    p.check()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,D,N", [(1, 16384, 16, 16), (1, 16000, 4096, 16), (4, 8192, 4096, 8), (1, 9000, 4, 40)])
def test_slow_decays_add_up_no_bias(dtype, B, T, D, N):
    """Time steps of about 2^-13 that differ from token to token (with one for all of them a factor's rounding would be the same each time,
    up to T u / 2 in all): h_T = sum of delta_t a^(T-t), the gradient of what it began with a^T, the same for every channel.
    Factors and states are each rounded with half a step or so of random sign: 0.5 u of a token, sqrt(T / N) of that in the mean over N
    states, four times which are allowed.  What is of one sign adds up: less than a sixteenth of a step, T u / 16.  32 u for the rest."""
    delta = torch.rand(T, generator=torch.Generator().manual_seed(1)) * 2.0 ** -13 + 2.0 ** -14
    delta = delta.to(dtype).float()
    # (sixteenths of a bf16 step are on the grid of the factors: correctly rounded ones, too, would all be off to one side, by 1000 u)
    A = (-1 - (torch.arange(N) / 16.0 if dtype == F32 else torch.rand(N, generator=torch.Generator().manual_seed(2)))).expand(D, N).contiguous().cuda()
    x, dt = torch.ones(B, T, D, dtype=dtype, device="cuda"), delta.to(dtype).cuda()[None, :, None].expand(B, T, D).contiguous()
    b, c = torch.ones(B, T, 1, N, dtype=dtype, device="cuda"), torch.zeros(B, T, 1, N, dtype=dtype, device="cuda")
    y, end, begin = torch.empty_like(x), torch.empty(B, D, N, device="cuda"), torch.empty(B, D, N, device="cuda")
    sizes = (B, T, D, N, 1)
    kept = torch.empty(mdh.mdh_selective_scan_checkpoints_size(sizes), dtype=torch.uint8, device="cuda")
    ws = torch.empty(mdh.mdh_selective_scan_workspace_size(sizes, dtype, True), dtype=torch.uint8, device="cuda")
    mdh.mdh_selective_scan(x, dt, A, b, c, y, final_state=end, checkpoints=kept, workspace=ws)
    d_x, d_dt, d_b, d_c = (torch.empty_like(v) for v in (x, dt, b, c))
    mdh.mdh_selective_scan_backward(x, dt, A, b, c, 0 * x, d_x, d_dt, torch.empty_like(A), d_b, d_c, kept, d_final_state=torch.ones_like(end),
                                    d_initial_state=begin, workspace=ws)
    steps = np64(delta)
    after = steps.sum() - np.cumsum(steps)  # behind each token
    refs = np.exp(np.outer(after, np64(A)[0])).T @ steps, np.exp(np64(A)[0] * steps.sum())
    for got, ref, what in zip((end, begin), refs, ("end", "begin")):
        off = float(np.abs((np64(got) / ref - 1).mean(axis=-1)).max()) / U
        assert off <= T / 16 + 2 * np.sqrt(T / N) + 32, "%s: %.0f" % (what, off)


# in turn (two kinds), 4 tiles at once (two kinds), 8 at once, segments
FORMS = [(4, 8192, 4096, 8), (1, 8192, 8192, 40), (1, 5800, 4096, 16), (1, 5800, 4096, 24), (1, 2500, 2048, 16), (1, 32768, 64, 16), (1, 16000, 4096, 16)]


def _through(dtype, B, T, D, N, delta, A, h0):
    """What is left of the states h0 after T tokens that add nothing, and of such gradients of the final states."""
    x, dt = torch.zeros(B, T, D, dtype=dtype, device="cuda"), delta.to(dtype).cuda()[None, :, None].expand(B, T, D).contiguous()
    b, end, begin = torch.zeros(B, T, 1, N, dtype=dtype, device="cuda"), torch.empty_like(h0), torch.empty_like(h0)
    sizes = (B, T, D, N, 1)
    kept = torch.empty(mdh.mdh_selective_scan_checkpoints_size(sizes), dtype=torch.uint8, device="cuda")
    ws = torch.empty(mdh.mdh_selective_scan_workspace_size(sizes, dtype, True), dtype=torch.uint8, device="cuda")
    mdh.mdh_selective_scan(x, dt, A, b, b, torch.empty_like(x), initial_state=h0, final_state=end, checkpoints=kept, workspace=ws)
    mdh.mdh_selective_scan_backward(x, dt, A, b, b, x, torch.empty_like(x), torch.empty_like(x), torch.empty_like(A), torch.empty_like(b),
                                    torch.empty_like(b), kept, d_final_state=h0, d_initial_state=begin, workspace=ws)
    return (end, "end"), (begin, "begin")


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,D,N", FORMS)
def test_states_without_decay_stay(dtype, B, T, D, N):
    """A = 0: the factor is 1 whatever the time steps are, and the state's bits are those that came in."""
    h0 = rand(1, B, D, N).cuda()
    for got, what in _through(dtype, B, T, D, N, torch.rand(T, generator=torch.Generator().manual_seed(2)), torch.zeros(D, N, device="cuda"), h0):
        assert torch.equal(got, h0), what


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("steps", ["near 0", "one of sixteen"])
@pytest.mark.parametrize("B,T,D,N", FORMS)
def test_time_steps_near_zero(dtype, steps, B, T, D, N):
    """Tokens to be ignored: time steps of 2^-30 to 2^-28, whose factors are 1 in 32 bits, alone or around a token of about 2^-9 in every
    tile.  h_T = h_0 e^(A sum of delta), and its gradient is the same.  A tile of ignored tokens: the state is rounded by u at most, its factor by
    0.7 u, with 0.12 u of the exponent's shift.  Where one of sixteen moves it, errors are of random sign but for less than u a tile: in
    the mean over the states T u / 16, and four times the square root of T / 4 N."""
    r = torch.Generator().manual_seed(3)
    delta = torch.rand(T, generator=r) * 2.0 ** -29 + 2.0 ** -30
    if steps == "one of sixteen":
        delta = torch.where(torch.arange(T) % 16 == 5, torch.rand(T, generator=r) * 2.0 ** -9 + 2.0 ** -10, delta)
    A, h0 = -1 - torch.rand(D, N, generator=r), (1 + torch.rand(B, D, N, generator=r)).cuda()
    want = np.exp(np64(A) * np64(delta.to(dtype)).sum())
    for got, what in _through(dtype, B, T, D, N, delta, A.cuda(), h0):
        off = (np64(got) / np64(h0) / want - 1) / U
        worst = np.abs(off).max() if steps == "near 0" else np.abs(off.mean(axis=-1)).max()
        limit = 1.9 * T / 16 + 32 if steps == "near 0" else T / 16 + 2 * np.sqrt(T / N) + 32
        assert worst <= limit, "%s: %.0f of %.0f" % (what, worst, limit)


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    """Columns of one projection, at odd places; tokens before batch entries; one token's values for all tokens."""
    p = Problem(dtype, 2, 40, 22, 18, 2)

    def odd(t):
        wide = torch.full((*t.shape[:-1], t.shape[-1] + 5), NAN, dtype=dtype, device="cuda")
        wide[..., 3:-2] = t.cuda()
        return wide[..., 3:-2]

    p.check(lay=odd)
    p.check(lay=lambda t: t.cuda().transpose(0, 1).contiguous().transpose(0, 1))
    plain, grads = p.forward()[0], p.backward()
    wide = torch.full((2, 40, 25), 7.0, dtype=dtype, device="cuda")
    p.forward(y=wide[..., 1:23])
    assert torch.equal(wide[..., 1:23], plain) and (wide[..., 0] == 7).all() and (wide[..., 23:] == 7).all()
    out = {n: odd(torch.zeros(s, dtype=dtype)) for n, s in (("d_x", p.x.shape), ("d_dt", p.x.shape), ("d_gate", p.x.shape), ("d_b", p.b.shape),
                                                           ("d_c", p.b.shape))}
    for got, want in zip(p.backward(out=out), grads):
        assert torch.equal(got, want)
    p.b = p.b[:, :1].expand(p.b.shape)
    p.check(lay=lambda t: t[:, :1].cuda().expand(t.shape) if t.stride(1) == 0 else t.cuda())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_tokens(dtype):
    """T = 0: the state passes through."""
    p = Problem(dtype, 2, 0, 10, 16)
    assert torch.equal(p.forward()[1].cpu(), p.h0)
    g = dict(zip(GRADS, p.backward()))
    assert torch.equal(g["d_initial"].cpu(), p.dh) and not any(g[n].any() for n in ("d_A", "d_skip", "d_dt_bias"))
    p = Problem(dtype, 0, 5, 10, 16)
    p.forward()
    g = dict(zip(GRADS, p.backward()))
    assert not any(g[n].any() for n in ("d_A", "d_skip", "d_dt_bias"))


@gpu
@pytest.mark.parametrize("T", [70, 1300])
def test_states_in_place_and_in_slots(T):
    p = Problem(BF16, 3, T, 20, 16, 2)
    y, final = p.forward()
    a = [t.cuda() for t in (p.x, p.dt, p.A, p.b, p.c)]
    ws = p.buffers(False)[0]
    state, y2 = p.h0.cuda(), torch.empty_like(y)
    mdh.mdh_selective_scan(*a, y2, initial_state=state, final_state=state, workspace=ws, **p.rest(cuda))
    assert torch.equal(y, y2) and torch.equal(state, final)
    pool = rand(9, 7, 20, 16).cuda()
    before = pool.clone()
    pool[5], pool[2] = p.h0[0].cuda(), p.h0[2].cuda()
    slots = torch.tensor([5, -1, 2], dtype=torch.int32, device="cuda")
    mdh.mdh_selective_scan(*a, y2, initial_state=pool, final_state=pool, slots=slots, workspace=ws, **p.rest(cuda))
    assert torch.equal(pool[5], final[0]) and torch.equal(pool[2], final[2]) and torch.equal(y2[0], y[0]) and torch.equal(y2[2], y[2])
    rest = [0, 1, 3, 4, 6]
    assert torch.equal(pool[rest], before[rest])
    p.h0[1] = 0  # an entry without a slot begins with zeros
    assert torch.equal(p.forward()[0][1], y2[1])
    slots[1] = 7  # and one past the pool has none
    mdh.mdh_selective_scan(*a, y2, final_state=pool, slots=slots, workspace=ws, **p.rest(cuda))
    assert torch.equal(pool[rest], before[rest])


@gpu
def test_output_in_place():
    """y where dt or the gate was."""
    for T in (50, 1300):
        p = Problem(BF16, 2, T, 36, 16)
        y, _ = p.forward()
        for at in ("dt", "gate"):
            here = getattr(p, at).cuda()
            p.forward(lay=lambda t: here if t is getattr(p, at) else t.cuda(), y=here)
            assert torch.equal(here, y), at


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,D,N,G", [(1, 1, 1, 1), (3, 64, 16, 1), (2, 37, 16, 1), (5, 20, 4, 2), (2, 24, 64, 4), (300, 12, 8, 1), (2, 10, 3, 1),
                                     (2, 9, 17, 3), (1, 6, 50, 1), (3, 8, 36, 2), (1, 2048, 16, 1)])
def test_step(dtype, B, D, N, G):
    p = Problem(dtype, B, 1, D, N, G)
    a, k = p.oracle()
    (ry, rf), (my, mf) = O.selective_scan(*a, **k), O.selective_scan(*a, **k, magnitude=True)
    state, y = p.h0.cuda(), p.empty(B, D)
    mdh.mdh_selective_scan_step(*(t[:, 0].cuda() if t is not p.A else t.cuda() for t in (p.x, p.dt, p.A, p.b, p.c)), state, y, p.skip.cuda(),
                                p.gate[:, 0].cuda(), p.dt_bias.cuda(), True)
    close(y, ry[:, 0], my[:, 0], dtype == BF16, N + 503, "y")
    close(state, rf, mf, False, 503, "state")


@gpu
@pytest.mark.parametrize("N", [16, 18])
def test_step_in_slots_and_strides(N):
    p = Problem(BF16, 4, 1, 30, N, 2, gate=False, skip=False)
    x, dt, b, c = (t[:, 0].cuda() for t in (p.x, p.dt, p.b, p.c))
    A, bias = p.A.cuda(), p.dt_bias.cuda()
    y, state = p.empty(4, 30), p.h0.cuda()
    mdh.mdh_selective_scan_step(x, dt, A, b, c, state, y, dt_bias=bias, softplus=True)
    pool = rand(3, 9, 30, N).cuda()
    before = pool.clone()
    slots = torch.tensor([8, -1, 0, 9], dtype=torch.int32, device="cuda")
    pool[8], pool[0] = p.h0[0].cuda(), p.h0[2].cuda()
    wide, bc = p.empty(4, 50), p.empty(4, 2, 2 * N + 3)
    wide[:, 3:33] = x
    bc[..., 1:N + 1], bc[..., N + 2:2 * N + 2] = b, c
    y2 = p.empty(4, 2, 30)[:, 1]
    mdh.mdh_selective_scan_step(wide[:, 3:33], dt, A, bc[..., 1:N + 1], bc[..., N + 2:2 * N + 2], pool, y2, dt_bias=bias, softplus=True, slots=slots)
    assert torch.equal(y2[0], y[0]) and torch.equal(y2[2], y[2]) and not y2[1].any() and not y2[3].any()
    assert torch.equal(pool[8], state[0]) and torch.equal(pool[0], state[2]) and torch.equal(pool[1:8], before[1:8])


@gpu
def test_step_past_2_31_elements():
    """The last slot of a pool of 9 GB: its offset in elements does not fit 32 bits."""
    D, N, n = 4096, 16, 34000
    pool = torch.empty(n, D, N, device="cuda")
    assert pool.numel() > 1 << 31
    slots = torch.tensor([n - 1], dtype=torch.int32, device="cuda")
    p = Problem(F32, 1, 1, D, N)
    pool[n - 1] = p.h0[0].cuda()
    y, y2, state = torch.empty(1, D, device="cuda"), torch.empty(1, D, device="cuda"), p.h0.cuda()
    a = [t[:, 0].cuda() if t is not p.A else t.cuda() for t in (p.x, p.dt, p.A, p.b, p.c)]
    mdh.mdh_selective_scan_step(*a, pool, y, slots=slots)
    mdh.mdh_selective_scan_step(*a, state, y2)
    assert torch.equal(y, y2) and torch.equal(pool[n - 1], state[0])


@gpu
def test_activations_past_2_31_elements():
    """The last tokens of the last sequence, whose offsets in elements do not fit 32 bits: alone, from the state before them, they are
    the same sums in other segments."""
    B, T, D, N, tail = 2, 70000, 16384, 16, 160
    shape = (B, T, D)
    x, dt, y = (torch.zeros(shape, dtype=BF16, device="cuda") for _ in range(3))
    assert x.numel() > 1 << 31
    b, c = (rand(i, B, T, 1, N, dtype=BF16).cuda() for i in (1, 2))
    x[1, -tail:], dt[1, -tail:] = rand(3, tail, D, dtype=BF16).cuda(), rand(4, tail, D, dtype=BF16).abs().cuda()
    A = -torch.exp(0.3 * rand(5, D, N)).cuda()
    n = mdh.mdh_selective_scan_workspace_size((B, T, D, N, 1), BF16)
    mdh.mdh_selective_scan(x, dt, A, b, c, y, workspace=torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    few = torch.empty(1, tail, D, dtype=BF16, device="cuda")
    n = mdh.mdh_selective_scan_workspace_size((1, tail, D, N, 1), BF16)
    mdh.mdh_selective_scan(x[1:, -tail:], dt[1:, -tail:], A, b[1:, -tail:], c[1:, -tail:], few,
                           workspace=torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    # sums of 16 terms of size 16 at most, off by (3 tail + 500) u in either call, and one rounding each
    assert ((y[1, -tail:].float() - few[0].float()).abs() <= 2.0 ** -7 * few[0].float().abs() + 1e3 * U * 400).all()
    assert not y[0].any() and not y[1, :-tail].any()


@gpu
@pytest.mark.parametrize("T", [40, 700])
def test_gradients_past_2_31_elements(T):
    """All operands and gradients as columns of one buffer whose last tokens are past 2^31 elements: the bits of dense ones."""
    p = Problem(BF16, 2, T, 20, 16, 2, lengths=[T, T - 9])
    want = [*p.forward(), *p.backward()]
    wide = torch.empty(2, T, (1 << 31) // T + 4000, dtype=BF16, device="cuda")  # (the first sequence's last tokens are past it, too)
    assert wide[0].numel() > 1 << 31
    columns = iter(range(3, 5000, 47))

    def place(shape):
        at, n = next(columns), int(np.prod(shape[2:]))
        view = wide[:, :, at:at + n]
        return view if len(shape) == 3 else view.unflatten(2, shape[2:])

    def lay(t):
        return place(t.shape).copy_(t)

    y = place(p.x.shape)
    out = {n: place((p.b if n in ("d_b", "d_c") else p.x).shape) for n in GRADS[:5]}
    for got, ref in zip([*p.forward(lay, y), *p.backward(lay, out=out)], want):
        assert torch.equal(got, ref)


@gpu
def test_gradients_of_more_parameters_than_a_launch_has_lanes():
    """4 million channels with 64 states: d_A, d_skip and d_dt_bias are 277 million sums over the sequences.  A channel's are those of a
    call on some channels alone, bit for bit."""
    B, D, N = 2, 1 << 22, 64
    r = torch.Generator("cuda").manual_seed(1)
    new = lambda *shape: torch.randn(shape, generator=r, device="cuda")  # noqa: E731
    x, dt, d_y, b, c, A, dh = new(B, 1, D), new(B, 1, D), new(B, 1, D), new(B, 1, 1, N), new(B, 1, 1, N), -new(D, N).abs(), new(B, D, N)

    def grads(*channels):
        """[d_A, d_skip, d_dt_bias] of a range of channels"""
        p, q, w, a, g = (t[..., slice(*channels)].contiguous() for t in (x, dt, d_y, A.T, dh.transpose(1, 2)))
        a, g = a.T.contiguous(), g.transpose(1, 2).contiguous()
        n = a.shape[0]
        sizes = (B, 1, n, N, 1)
        kept = torch.empty(mdh.mdh_selective_scan_checkpoints_size(sizes), dtype=torch.uint8, device="cuda")
        ws = torch.empty(mdh.mdh_selective_scan_workspace_size(sizes, F32, True), dtype=torch.uint8, device="cuda")
        out = [torch.full(s, NAN, device="cuda") for s in ((n, N), (n,), (n,))]
        mdh.mdh_selective_scan(p, q, a, b, c, torch.empty_like(p), initial_state=g, checkpoints=kept, workspace=ws, softplus=True)
        mdh.mdh_selective_scan_backward(p, q, a, b, c, w, torch.empty_like(p), torch.empty_like(p), out[0], torch.empty_like(b), torch.empty_like(b),
                                        kept, d_final_state=g, d_skip=out[1], d_dt_bias=out[2], workspace=ws, softplus=True)
        return out

    got = grads(0, D)
    assert torch.equal(got[1], d_y[0, 0] * x[0, 0] + d_y[1, 0] * x[1, 0])
    for lo in (0, (1 << 21) - 50, D - 100):
        for whole, part in zip(got, grads(lo, lo + 100)):
            assert torch.equal(whole[lo:lo + 100], part), lo


@gpu
def test_prompt_then_tokens():
    """A prompt and the tokens after it, one at a time, are one sequence."""
    p = Problem(F32, 2, 60, 40, 16, 2)
    a, k = p.oracle()
    (ry, rf), (my, mf) = O.selective_scan(*a, **k), O.selective_scan(*a, **k, magnitude=True)
    x, dt, b, c, gate, A = (t.cuda() for t in (p.x, p.dt, p.b, p.c, p.gate, p.A))
    kw = dict(skip=p.skip.cuda(), dt_bias=p.dt_bias.cuda(), softplus=True)
    state, y = p.h0.cuda(), p.empty(2, 60, 40)
    ws = p.buffers(False)[0]
    mdh.mdh_selective_scan(x[:, :52], dt[:, :52], A, b[:, :52], c[:, :52], y[:, :52], gate=gate[:, :52], initial_state=state, final_state=state,
                           workspace=ws, **kw)
    for t in range(52, 60):
        mdh.mdh_selective_scan_step(x[:, t], dt[:, t], A, b[:, t], c[:, t], state, y[:, t], gate=gate[:, t], **kw)
    close(y, ry, my, False, 3 * 60 + 516, "y")
    close(state, rf, mf, False, 3 * 60 + 516, "state")


@gpu
def test_gradients_against_differences():
    """The kernels' gradients along random directions against differences of the oracle's forward function."""
    p = Problem(F32, 1, 60, 12, 8, 2, lengths=[57])
    grads = {n: np64(t) for n, t in zip(GRADS, p.backward())}
    names = ("d_x", "d_dt", "d_A", "d_b", "d_c", "d_skip", "d_gate", "d_dt_bias", "d_initial")
    at = [np64(t) for t in (p.x, p.dt, p.A, p.b, p.c, p.skip, p.gate, p.dt_bias, p.h0)]

    def loss(v):
        y, final = O.selective_scan(*v[:8], True, [57], v[8])
        return (y * np64(p.d_y)).sum() + (final * np64(p.dh)).sum()

    rng = np.random.default_rng(1)
    for i, name in enumerate(names):
        d, h = rng.standard_normal(at[i].shape), 1e-6
        up, down = ([v + s * d if j == i else v for j, v in enumerate(at)] for s in (h, -h))
        want = (loss(up) - loss(down)) / (2 * h)
        # curvature 1e-12 times a third derivative, 64-bit rounding 1e-16 / 1e-6 of the loss, and the kernels' own limit
        assert abs((grads[name] * d).sum() - want) <= 2e-5 * (np.abs(grads[name] * d).sum() + 1), name


def _states(A, delta, u, h0):
    h, all_ = h0, []
    for t in range(delta.shape[1]):
        h = torch.exp(delta[:, t, :, None] * A) * h + u[:, t]
        all_.append(h)
    return all_


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,T,D,N", [(4, 256, 2048, 16), (2, 300, 1000, 40), (1, 1200, 512, 16)])
def test_chip_full_of_work(dtype, B, T, D, N):
    """Every output with every compute unit busy, against 64 bits on the GPU; the same bits in three calls."""
    p = Problem(dtype, B, T, D, N, states=False)
    first = None
    for _ in range(3):
        got = [p.forward()[0], *p.backward()]
        first = first or got
        assert all(torch.equal(i, j) for i, j in zip(first, got))
    half, A = dtype == BF16, p.A.cuda().double()
    v = p.dt.cuda().double() + p.dt_bias.cuda().double()
    delta = torch.nn.functional.softplus(v, threshold=1000.0)
    n = 3 * T + N + 500
    out = []
    for f in (lambda t: t, torch.abs):
        x, b, c, skip, d_y, gate = (f(t.cuda().double()) for t in (p.x, p.b[:, :, 0], p.c[:, :, 0], p.skip, p.d_y, p.gate))
        w = torch.sigmoid(p.gate.cuda().double())
        zero = torch.zeros(B, D, N, dtype=torch.float64, device="cuda")
        hs = _states(A, delta, (delta * x)[..., None] * b[:, :, None], zero)
        pre = torch.stack([(h * c[:, t, None]).sum(-1) for t, h in enumerate(hs)], 1) + skip * x
        d_p = d_y * gate * w
        e, d_A = zero, torch.zeros_like(A)
        d_x, d_dt, d_b, d_c = [], [], [], []
        for t in reversed(range(T)):
            full = e + d_p[:, t, :, None] * c[:, t, None]
            r = (full * b[:, t, None]).sum(-1)
            e = torch.exp(delta[:, t, :, None] * A) * full
            q = e * (hs[t - 1] if t else zero)
            d_c.append((d_p[:, t, :, None] * hs[t]).sum(1)), d_b.append((full * (delta[:, t] * x[:, t])[..., None]).sum(1))
            d_A += (q * delta[:, t, :, None]).sum(0)
            d_x.append(delta[:, t] * r + skip * d_p[:, t])
            d_dt.append(((q * f(A)).sum(-1) + x[:, t] * r) * torch.sigmoid(v[:, t]))
        d_x, d_dt, d_b, d_c = (torch.stack(t[::-1], 1) for t in (d_x, d_dt, d_b, d_c))
        out.append([pre * gate * w, d_x, d_dt, d_b[:, :, None], d_c[:, :, None], d_y * pre * w * (1 + gate * (1 - w)), d_A,
                    (d_p * x).sum((0, 1)), d_dt.sum((0, 1))])
    for i, (g, r, m) in enumerate(zip(got, *out)):
        k = n if i == 0 else 2 * n + B * T + D
        limit = k * U * m + (2.0 ** -8 * r.abs() if half and i < 6 else 0) + 1e-37
        off = (g.double() - r).abs()
        assert (off <= limit).all(), "%s: %.2f" % (("y", *GRADS)[i], float((off / limit).max()))


@gpu
@pytest.mark.parametrize("T", [70, 1100])
def test_same_bits_on_another_stream_and_in_a_graph(T):
    p = Problem(BF16, 2, T, 40, 16, 2, lengths=[T, T - 40])
    want = [*p.forward(), *p.backward()]
    got = [torch.empty_like(t) for t in want]
    x, dt, A, b, c, d_y, h0, dh = (t.cuda() for t in (p.x, p.dt, p.A, p.b, p.c, p.d_y, p.h0, p.dh))
    rest, (ws, kept) = p.rest(cuda), p.buffers()
    g = dict(zip(GRADS, got[2:]))

    def call():
        mdh.mdh_selective_scan(x, dt, A, b, c, got[0], initial_state=h0, final_state=got[1], checkpoints=kept, workspace=ws, **rest)
        mdh.mdh_selective_scan_backward(x, dt, A, b, c, d_y, g["d_x"], g["d_dt"], g["d_A"], g["d_b"], g["d_c"], kept, d_final_state=dh,
                                        d_skip=g["d_skip"], d_gate=g["d_gate"], d_dt_bias=g["d_dt_bias"], d_initial_state=g["d_initial"],
                                        workspace=ws, **rest)

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


def _raw(sizes, dtype=0, x=64, dt=64, b=64, c=64, A=64, y=64, strides=None, slots=None, n=0, final=None, kept=None, nkept=0, ws=1 << 20,
         nws=1 << 50):
    S = mdh.binding._sizes
    return mdh.lib().mdh_selective_scan(S(sizes), dtype, x, dt, None, b, c, None if strides is None else S(strides), A, None, None, 1, None,
                                        None, final, slots, n, y, kept, nkept, ws, nws, None)


def _back(sizes, strides=None, gate=None, kept=1 << 20, nkept=1 << 50, ws=1 << 20, nws=1 << 50, dh=None, dh0=None, **p):
    S = mdh.binding._sizes
    g = lambda n: p.get(n, 64)  # noqa: E731
    return mdh.lib().mdh_selective_scan_backward(S(sizes), 0, g("x"), g("dt"), gate, g("b"), g("c"), g("d_y"), None if strides is None else S(strides),
                                                 g("A"), None, None, 1, None, dh, kept, nkept, g("d_x"), g("d_dt"), None, g("d_b"), g("d_c"), None,
                                                 None, None, dh0, ws, nws, None)


def test_refusals():
    ok = (2, 40, 8, 16, 2)
    for sizes in ((-1, *ok[1:]), (2, -1, 8, 16, 2), (2, 40, 0, 16, 2), (2, 40, 8, 0, 2), (2, 40, 8, 16, 0), (2, 40, 8, 16, 3), (1 << 16, 1 << 16, 8, 16, 2),
                  (1, 40, 1 << 24, 16, 1), (1, 1 << 27, 8, 32, 1), (1 << 24, 2, 8, 16, 1)):
        assert _raw(sizes) == E_SIZE
    assert _raw((2, 40, 8, 65, 2)) == E_UNSUP and _raw(ok, dtype=2) == E_UNSUP
    for name in ("x", "dt", "b", "c", "A", "y"):
        assert _raw(ok, **{name: None}) == E_NULL and _raw(ok, **{name: 66}) == E_UNSUP
    assert _raw(ok, slots=64, n=-1) == E_SIZE and _raw(ok, final=62) == E_UNSUP
    dense = [320, 8, 320, 8, 320, 8, 320, 8, 1280, 32, 16, 1280, 32, 16]
    assert _raw(ok, strides=dense[:7] + [0] + dense[8:]) == E_SIZE  # outputs on one another
    assert _raw((0, *ok[1:]), x=None, y=None) == 0 and _raw((2, 0, 8, 16, 2), x=None, y=None) == 0  # nothing to do
    kept = mdh.mdh_selective_scan_checkpoints_size(ok)
    assert kept > 0 and _raw(ok, kept=64, nkept=kept - 1) == E_WS and _raw(ok, kept=72, nkept=kept) == E_WS
    long = (1, 4096, 8, 16, 2)
    need = mdh.mdh_selective_scan_workspace_size(long, F32)
    assert need > 0 and _raw(long, ws=None) == E_WS and _raw(long, nws=need - 1) == E_WS and _raw(long, ws=(1 << 20) + 8) == E_WS
    need = mdh.mdh_selective_scan_workspace_size(ok, F32, True)
    assert need > 0 and _back(ok, ws=None) == E_WS and _back(ok, nws=need - 1) == E_WS and _back(ok, ws=(1 << 20) + 8) == E_WS
    assert _back(ok, kept=None) == E_WS and _back(ok, nkept=kept - 1) == E_WS
    for name in ("x", "dt", "b", "c", "A", "d_y", "d_x", "d_dt", "d_b", "d_c"):
        assert _back(ok, **{name: None}) == E_NULL
    assert _back(ok, gate=64) == E_NULL  # a gate without room for its gradient
    assert _back(ok, dh=64, dh0=64) == E_UNSUP
    strides = [320, 8] * 7 + [1280, 32, 16] * 4
    for i in (9, 11, 21, 22, 25):
        assert _back(ok, strides=strides[:i] + [0] + strides[i + 1:]) == E_SIZE
    step = lambda sizes, x=64, state=64: mdh.lib().mdh_selective_scan_step(mdh.binding._sizes(sizes), 0, x, 64, None, 64, 64, None, 64, None, None, 1,  # noqa: E731
                                                                           state, None, 0, 64, None)
    assert step((2, 8, 16, 3)) == E_SIZE and step((2, 8, 65, 1)) == E_UNSUP and step((1 << 22, 8, 16, 1)) == E_SIZE
    assert step((2, 8, 16, 1), x=None) == E_NULL and step((2, 8, 16, 1), state=None) == E_NULL and step((0, 8, 16, 1)) == 0


@pytest.mark.parametrize("T", [0, 313, 314, 1024, 100000])
@pytest.mark.parametrize("N", [16, 17, 33, 64])
def test_an_empty_batch_wants_no_workspace(T, N):
    for dtype in (F32, BF16):
        for D, G in ((256, 1), (16, 16)):
            sizes = (0, T, D, N, G)
            assert mdh.mdh_selective_scan_workspace_size(sizes, dtype) == 0 == mdh.mdh_selective_scan_workspace_size(sizes, dtype, True)
            assert mdh.mdh_selective_scan_checkpoints_size(sizes) == 0


def test_refuses_gradients_of_b_and_c_past_2_31_elements():
    assert _back((1, 17, 3900000, 64, 3900000)) == E_SIZE and _back((1, 1 << 21, 64, 64, 16)) == E_SIZE


def test_refuses_outputs_whose_rows_overlap():
    ok = (2, 40, 8, 16, 2)
    dense = [320, 8, 320, 8, 320, 8, 320, 8, 1280, 32, 16, 1280, 32, 16]
    for i, n in ((6, 7), (6, -7), (7, 7)):
        assert _raw(ok, strides=dense[:i] + [n] + dense[i + 1:]) == E_SIZE
    strides = [320, 8] * 7 + [1280, 32, 16] * 4
    for i in (8, 9, 10, 11):
        assert _back(ok, strides=strides[:i] + [7] + strides[i + 1:]) == E_SIZE
    for i in range(20, 26):
        assert _back(ok, strides=strides[:i] + [15] + strides[i + 1:]) == E_SIZE


def test_binding_refuses_what_does_not_fit():
    x, A, b = torch.zeros(2, 5, 8), torch.zeros(8, 4), torch.zeros(2, 5, 2, 4)
    with pytest.raises(TypeError):
        mdh.mdh_selective_scan(x, x, A, b, b, x)  # not on the GPU
    for bad in ((x[:, :3], x, A, b, b, x), (x, x[:, :3], A, b, b, x), (x, x, A[:4], b, b, x), (x, x, A, b[:, :3], b, x), (x, x, A, b, b[..., :2], x),
                (x, x, A, b, b, x[:1]), (x, x, A, b[:, :, 0], b, x)):
        with pytest.raises(ValueError):
            mdh.mdh_selective_scan(*bad)
    with pytest.raises(ValueError):
        mdh.mdh_selective_scan_backward(x, x, A, b, b, x, x, x, None, b, b, None, gate=x)
    with pytest.raises(ValueError):
        mdh.mdh_selective_scan_step(x[:, 0], x[:, 0], A, b[:, 0], b[:, 0], torch.zeros(2, 8, 5), x[:, 0])
    with pytest.raises(TypeError):
        mdh.mdh_selective_scan_workspace_size((2, 5, 8, 4, 2), torch.float64)


def test_binding_refuses_steps_that_do_not_fit():
    x, A, b, h = torch.zeros(2, 8), torch.zeros(8, 4), torch.zeros(2, 2, 4), torch.zeros(2, 8, 4)
    with pytest.raises(TypeError):
        mdh.mdh_selective_scan_step(x, x, A, b, b, h, x)  # not on the GPU
    for bad in ((x[:1], x, A, b, b, h, x), (x, x[:1], A, b, b, h, x), (x, x, A[:4], b, b, h, x), (x, x, A[..., None], b, b, h, x),
                (x, x, A[0], b, b, h, x), (x, x, A, b[0], b, h, x), (x, x, A, b[..., :2], b, h, x), (x, x, A, b, b[:, :1], h, x),
                (x, x, A, b, b, h, x[:, :4]), (x[None], x, A, b, b, h, x)):
        with pytest.raises(ValueError):
            mdh.mdh_selective_scan_step(*bad)
    with pytest.raises(ValueError):
        mdh.mdh_selective_scan_step(x, x, A, b, b, h, x, gate=x[:1])
