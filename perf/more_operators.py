"""The selective state space scan, the short causal convolution before it, and layer norm on a residual stream: work to be
timed and checked.

``own`` chooses between the operators' plain forms (elementary torch operations in 32 bits) and this library's entry points.
A case names the operator, its sizes and its types; ``prepare`` makes what a program has in hand before the call, ``run`` is
one pass, ``exact`` the same from the definitions in 64 bits.

Layouts: activations are (batch, token, channel), what the channels of a group share (batch, token, group, state), states
(batch or slot, channel, state) in fp32, the convolution's windows (batch or slot, taps - 1, channel) in the activations' type.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ----------------------------------------------------------------------------------------------- the cases


def _scan(kind, dtype, B, T, D, N, G=1, gate=True, ragged=False, state=False, fused=False):
    return {"kind": kind, "dtype": dtype, "B": B, "T": T, "D": D, "N": N, "G": G, "gate": gate, "ragged": ragged, "state": state,
            "fused": fused}


def _scan_step(dtype, B, D, N, G=1, slots=0, gate=True):
    return {"kind": "scan_step", "dtype": dtype, "B": B, "D": D, "N": N, "G": G, "slots": slots, "gate": gate}


def _conv(kind, dtype, B, T, C, W, act="silu", ragged=False, state=False, fused=False):
    return {"kind": kind, "dtype": dtype, "B": B, "T": T, "C": C, "W": W, "act": act, "ragged": ragged, "state": state, "fused": fused}


def _conv_step(dtype, B, C, W, slots=0):
    return {"kind": "conv_step", "dtype": dtype, "B": B, "C": C, "W": W, "slots": slots, "act": "silu"}


def _norm(kind, dtype, rows, C, residual=True):
    return {"kind": kind, "dtype": dtype, "rows": rows, "C": C, "residual": residual}


def _named(name, case):
    return dict(case, name=name)


def listed():
    return [
        # one request's prompt; the state goes on to the generation of tokens, the gate lies beside x in a projection's output
        _named("scan_prompt", _scan("scan", "bf16", 1, 2048, 4096, 16, state=True, fused=True)),
        # prompts of several requests padded to the longest, one of them empty, that go on from states; groups of odd widths
        _named("scan_ragged", _scan("scan", "bf16", 6, 1021, 1250, 24, G=2, ragged=True, state=True)),
        # one long document through a narrow layer: the work has to be split along the tokens
        _named("scan_long", _scan("scan", "bf16", 1, 32768, 1536, 16)),
        # a training step's layer: outputs and all gradients
        _named("scan_train", _scan("scan_train", "bf16", 4, 2048, 4096, 16)),
        # the same in fp32 on pieces of a longer text: a state comes in and its gradient goes on; an odd number of tokens
        _named("scan_train_f32", _scan("scan_train", "f32", 2, 1001, 768, 16, G=4, state=True)),
        # the next token of many requests, their states in a pool of which some slots are not in use
        _named("scan_step_many", _scan_step("bf16", 250, 4096, 16, slots=300)),
        # the next token of one request, with wider states
        _named("scan_step_one", _scan_step("bf16", 1, 2048, 64)),
        # prompts padded to the longest, with the windows that the next tokens go on from; x is a part of wider rows
        _named("conv_ragged", _conv("conv", "bf16", 6, 1021, 2500, 4, ragged=True, state=True, fused=True)),
        # a training step's convolution: outputs and all gradients
        _named("conv_train", _conv("conv_train", "bf16", 4, 2048, 4096, 4)),
        # the next token of some requests: latency alone
        _named("conv_step", _conv_step("bf16", 8, 2048, 4, slots=20)),
        # the norm before a layer, in training: the residual stream's sum, outputs and all gradients
        _named("norm_train", _norm("norm_train", "bf16", 16384, 4096)),
        # rows that divide nothing, in fp32, of a prompt
        _named("norm_odd", _norm("norm", "f32", 1021, 2501)),
    ]


def _log(rng, lo, hi):
    """Whole number, uniform over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _channels(rng, lo, hi, groups=1):
    """Mostly what vector loads like, else any; a multiple of the groups."""
    n = _log(rng, lo, hi)
    return groups * max(1, (n + 31) // 64 * 64 // groups if rng.random() < 0.6 else n // groups)


def _draw_scan(rng):
    kind = rng.choice(["scan", "scan_train"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    G = rng.choice([1, 1, 1, 2, 4, 8])
    D = _channels(rng, 64, 8192, G)
    N = 16 if rng.random() < 0.6 else rng.randint(1, 64)
    # steps of the recurrence: half of the largest listed training step's, all of the long document's in a forward call
    most = 4 * 2048 * 4096 * 16 // 2 if kind == "scan_train" else 32768 * 1536 * 16
    T, B = _log(rng, 1, 4096 if kind == "scan_train" else 32768), _log(rng, 1, 32)
    wide = D * max(N, 16) * (2 if dtype == "f32" else 1)
    while B > 1 and B * T * wide > most:
        B -= 1
    return _scan(kind, dtype, B, max(1, min(T, most // (B * wide))), D, N, G, gate=rng.random() < 0.7, ragged=rng.random() < 0.4,
                 state=rng.random() < 0.5, fused=rng.random() < 0.3)


def _draw_scan_step(rng):
    G = rng.choice([1, 1, 1, 2, 4])
    D = _channels(rng, 64, 8192, G)
    N = 16 if rng.random() < 0.6 else rng.randint(1, 64)
    B = max(1, min(_log(rng, 1, 400), 250 * 4096 * 16 // (D * N)))
    return _scan_step("f32" if rng.random() < 0.3 else "bf16", B, D, N, G, B + rng.randint(1, 20) if rng.random() < 0.5 else 0,
                      gate=rng.random() < 0.7)


def _draw_conv(rng):
    if rng.random() < 0.3:
        B = _log(rng, 1, 400)
        return _conv_step("f32" if rng.random() < 0.3 else "bf16", B, _channels(rng, 64, 8192), rng.choice([2, 3, 4, 4, 4]),
                          B + rng.randint(1, 20) if rng.random() < 0.5 else 0)
    kind = rng.choice(["conv", "conv_train"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    C = _channels(rng, 64, 12288)
    most = 4 * 2048 * 4096 // (2 if dtype == "f32" else 1)
    T, B = _log(rng, 1, 32768), _log(rng, 1, 32)
    while B > 1 and B * T * C > most:
        B -= 1
    return _conv(kind, dtype, B, max(1, min(T, most // (B * C))), C, rng.choice([2, 3, 4, 4, 4]), act=rng.choice(["silu", "silu", "none"]),
                 ragged=rng.random() < 0.4, state=rng.random() < 0.5, fused=rng.random() < 0.3)


def _draw_norm(rng):
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    C = _channels(rng, 64, 16384)
    most = 16384 * 4096 // (2 if dtype == "f32" else 1)
    return _norm(rng.choice(["norm", "norm_train"]), dtype, max(1, min(_log(rng, 1, 65536), most // C)), C, residual=rng.random() < 0.7)


def draw(rng):
    u = rng.random()
    return _draw_scan(rng) if u < 0.4 else _draw_scan_step(rng) if u < 0.5 else _draw_conv(rng) if u < 0.75 else _draw_norm(rng)


# ----------------------------------------------------------------------------------------------- the inputs


def _normal(gen, *shape, dtype=torch.float32, times=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * times).to(dtype)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda")


def _lengths(case, gen):
    """Any from nothing to all of it, with the first the longest and the second empty."""
    at = torch.randint(0, case["T"] + 1, (case["B"],), generator=gen, device="cuda")
    at[0] = case["T"]
    if case["B"] > 1:
        at[1] = 0
    return at.to(torch.int32)


def _slots(case, gen):
    n = case["slots"]
    return torch.randperm(n, generator=gen, device="cuda")[: case["B"]].to(torch.int32) if n else None


def _pair(gen, fused, lead, wide, dt):
    """Two tensors of rows, of their own or side by side in one."""
    if not fused:
        return _normal(gen, *lead, wide, dtype=dt), _normal(gen, *lead, wide, dtype=dt)
    return _normal(gen, *lead, 2 * wide, dtype=dt).split(wide, dim=-1)


def _prepare_scan(case, gen, dt, s):
    B, D, N, G = (case[n] for n in ("B", "D", "N", "G"))
    step = case["kind"] == "scan_step"
    lead = (B,) if step else (B, case["T"])
    s["x"], s["gate"] = _pair(gen, case.get("fused"), lead, D, dt)
    if not case["gate"]:
        s["gate"] = None
    s["dt"] = _normal(gen, *lead, D, dtype=dt, times=0.5)
    s["b"], s["c"] = _normal(gen, *lead, G, N, dtype=dt), _normal(gen, *lead, G, N, dtype=dt)
    # decays of 1, 2, .. N a unit of time, learned a little away from there; time steps of 0.001 to 0.1 through the softplus
    s["A"] = -torch.arange(1, N + 1, device="cuda") * torch.exp(_normal(gen, D, N, times=0.1))
    s["dt_bias"] = torch.log(torch.expm1(torch.exp(_uniform(gen, D) * math.log(100.0) + math.log(1e-3))))
    s["skip"] = 1 + _normal(gen, D, times=0.2)
    s["y"] = torch.empty(*lead, D, dtype=dt, device="cuda")
    if step:
        s["slots"] = _slots(case, gen)
        s["state"] = _normal(gen, case["slots"] or B, D, N)
        return s
    s["lengths"] = _lengths(case, gen) if case["ragged"] else None
    s["initial"] = _normal(gen, B, D, N) if case["state"] else None
    s["final"] = torch.empty(B, D, N, device="cuda") if case["state"] else None
    if case["kind"] == "scan_train":
        s["d_y"] = _normal(gen, *lead, D, dtype=dt)
        for n in ("x", "dt", "b", "c"):
            s["d_" + n] = torch.empty(s[n].shape, dtype=dt, device="cuda")
        s["d_gate"] = torch.empty(*lead, D, dtype=dt, device="cuda") if case["gate"] else None
        for n in ("A", "skip", "dt_bias"):
            s["d_" + n] = torch.empty_like(s[n])
        s["d_final"] = _normal(gen, B, D, N) if case["state"] else None
        s["d_initial"] = torch.empty(B, D, N, device="cuda") if case["state"] else None
    return s


def _prepare_conv(case, gen, dt, s):
    B, C, W = (case[n] for n in ("B", "C", "W"))
    step = case["kind"] == "conv_step"
    lead = (B,) if step else (B, case["T"])
    s["x"], _ = _pair(gen, case.get("fused"), lead, C, dt)
    s["weight"], s["bias"] = _normal(gen, C, W, times=W ** -0.5), _normal(gen, C, times=0.2)
    s["y"] = torch.empty(*lead, C, dtype=dt, device="cuda")
    if step:
        s["slots"] = _slots(case, gen)
        s["state"] = _normal(gen, case["slots"] or B, W - 1, C, dtype=dt)
        return s
    s["lengths"] = _lengths(case, gen) if case["ragged"] else None
    s["initial"] = _normal(gen, B, W - 1, C, dtype=dt) if case["state"] else None
    s["final"] = torch.empty(B, W - 1, C, dtype=dt, device="cuda") if case["state"] else None
    if case["kind"] == "conv_train":
        s["d_y"] = _normal(gen, *lead, C, dtype=dt)
        s["d_x"] = torch.empty(*lead, C, dtype=dt, device="cuda")
        s["d_weight"], s["d_bias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
        s["d_final"] = _normal(gen, B, W - 1, C, dtype=dt) if case["state"] else None
        s["d_initial"] = torch.empty(B, W - 1, C, dtype=dt, device="cuda") if case["state"] else None
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"].startswith("scan"):
        return _prepare_scan(case, gen, dt, s)
    if case["kind"].startswith("conv"):
        return _prepare_conv(case, gen, dt, s)
    rows, C = case["rows"], case["C"]
    s["x"] = _normal(gen, rows, C, dtype=dt)
    s["residual"] = (_normal(gen, rows, C, times=3.0) + _normal(gen, C)).to(dt) if case["residual"] else None
    s["total"] = torch.empty_like(s["x"]) if case["residual"] else None
    s["weight"], s["bias"], s["eps"] = 1 + _normal(gen, C, times=0.2), _normal(gen, C, times=0.2), 1e-5
    s["y"] = torch.empty_like(s["x"])
    if case["kind"] == "norm_train":
        s["d_y"] = _normal(gen, rows, C, dtype=dt)
        s["d_total"] = _normal(gen, rows, C, dtype=dt) if case["residual"] else None
        s["mean"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        s["d_x"] = torch.empty_like(s["x"])
        s["d_weight"], s["d_bias"] = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    return s


# ----------------------------------------------------------------------------------------------- the plain forms


def _valid(s):
    """(batch, token, 1): tokens before their sequence's length."""
    B, T = s["case"]["B"], s["case"]["T"]
    if s["lengths"] is None:
        return torch.ones(B, T, 1, dtype=torch.bool, device="cuda")
    return (torch.arange(T, device="cuda") < s["lengths"][:, None])[..., None]


def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _softplus(v):
    return v.clamp_min(0) + torch.log1p(torch.exp(-v.abs()))


def _plain_scan(s):
    """In chunks of tokens, all chunks a token at a time side by side: first what each leaves from a state of zeros, then the
    states that they begin with, then the chunks again from these."""
    c = s["case"]
    B, T, D, N, G = (c[n] for n in ("B", "T", "D", "N", "G"))
    dt_, E = s["x"].dtype, D // G
    valid = _valid(s)
    C = min(T, 64)
    n = -(-T // C)

    def cut(t):  # (token of a chunk, batch, chunk, ...)
        t = torch.nn.functional.pad(t, (0, 0) * (t.dim() - 2) + (0, n * C - T))
        return t.reshape(B, n, C, *t.shape[2:]).permute(2, 0, 1, *range(3, t.dim() + 1))

    v = s["dt"].float() + s["dt_bias"]
    x = torch.where(valid, s["x"].float(), 0.0)
    delta = torch.where(valid, _softplus(v), 0.0)
    b, cc = (torch.where(valid[..., None], s[m].float(), 0.0) for m in ("b", "c"))
    A = s["A"].reshape(G, E, N)
    xs, ds, bs, cs = cut(x.reshape(B, T, G, E)), cut(delta.reshape(B, T, G, E)), cut(b), cut(cc)
    whole = torch.exp(ds.sum(0)[..., None] * A)  # of a chunk

    def step(i, h):
        return torch.exp(ds[i][..., None] * A) * h + (ds[i] * xs[i])[..., None] * bs[i][:, :, :, None, :]

    h = torch.zeros(B, n, G, E, N, device="cuda")
    for i in range(C):
        h = step(i, h)
    starts = [s["initial"].reshape(B, G, E, N) if s["initial"] is not None else torch.zeros(B, G, E, N, device="cuda")]
    for m in range(n):
        starts.append(whole[:, m] * starts[-1] + h[:, m])
    end, h = starts.pop(), torch.stack(starts, 1)
    train = c["kind"] == "scan_train"
    kept, p = [h], []
    for i in range(C):
        h = step(i, h)
        p.append((h * cs[i][:, :, :, None, :]).sum(-1))
        if train:
            kept.append(h)

    def join(ts):
        t = torch.stack(ts, 2)
        return t.reshape(B, n * C, *t.shape[3:])[:, :T]

    p = join(p).reshape(B, T, D) + s["skip"] * x
    gate = None if s["gate"] is None else torch.where(valid, s["gate"].float(), 0.0)
    y = p if gate is None else p * gate * _sigmoid(gate)
    got = {"y": torch.where(valid, y, 0.0).to(dt_)}
    if s["final"] is not None:
        got["final"] = end.reshape(B, D, N)
    if not train:
        return got
    d_y = torch.where(valid, s["d_y"].float(), 0.0)
    d_p = d_y
    if gate is not None:
        w = _sigmoid(gate)
        d_p = d_y * gate * w
        got["d_gate"] = (d_y * p * w * (1 + gate * (1 - w))).to(dt_)
    dp = cut(d_p.reshape(B, T, G, E))

    def back(i, e):  # (the gradient of the state behind token i, and of the state before it)
        g = e + dp[i][..., None] * cs[i][:, :, :, None, :]
        return g, torch.exp(ds[i][..., None] * A) * g

    e = torch.zeros(B, n, G, E, N, device="cuda")
    for i in reversed(range(C)):
        e = back(i, e)[1]
    ends = [s["d_final"].reshape(B, G, E, N) if s["d_final"] is not None else torch.zeros(B, G, E, N, device="cuda")]
    for m in reversed(range(n)):
        ends.append(whole[:, m] * ends[-1] + e[:, m])
    d_initial, e = ends.pop(), torch.stack(ends[::-1], 1)
    d_A = torch.zeros(G, E, N, device="cuda")
    d_b, d_c, d_in, d_delta = [], [], [], []
    for i in reversed(range(C)):
        g, e = back(i, e)
        d_c.append((dp[i][..., None] * kept[i + 1]).sum(3))
        d_b.append((g * (ds[i] * xs[i])[..., None]).sum(3))
        r = (g * bs[i][:, :, :, None, :]).sum(-1)
        q = e * kept[i]
        d_A += (q * ds[i][..., None]).sum((0, 1))
        d_in.append(ds[i] * r)
        d_delta.append((q * A).sum(-1) + xs[i] * r)
    d_b, d_c, d_in, d_delta = (join(t[::-1]) for t in (d_b, d_c, d_in, d_delta))
    d_dt = torch.where(valid, d_delta.reshape(B, T, D) * _sigmoid(v), 0.0)
    got.update(d_x=(d_in.reshape(B, T, D) + s["skip"] * d_p).to(dt_), d_dt=d_dt.to(dt_), d_b=d_b.to(dt_), d_c=d_c.to(dt_),
               d_A=d_A.reshape(D, N), d_skip=(d_p * x).sum((0, 1)), d_dt_bias=d_dt.sum((0, 1)))
    if s["d_initial"] is not None:
        got["d_initial"] = d_initial.reshape(B, D, N)
    return got


def _plain_scan_step(s):
    c = s["case"]
    B, D, N, G = (c[n] for n in ("B", "D", "N", "G"))
    x, delta = s["x"].float(), _softplus(s["dt"].float() + s["dt_bias"])
    b, cc = (s[n].float().repeat_interleave(D // G, dim=1) for n in ("b", "c"))
    a, u = torch.exp(delta[..., None] * s["A"]), (delta * x)[..., None] * b
    if s["slots"] is None:
        h = s["state"].mul_(a).add_(u)
    else:
        at = s["slots"].long()
        h = s["state"][at] * a + u
        s["state"][at] = h
    y = (h * cc).sum(-1) + s["skip"] * x
    if s["gate"] is not None:
        gate = s["gate"].float()
        y = y * gate * _sigmoid(gate)
    return {"y": y.to(s["x"].dtype), "state": s["state"]}


def _plain_conv(s):
    c = s["case"]
    B, T, C, W = (c[n] for n in ("B", "T", "C", "W"))
    dt, valid = s["x"].dtype, _valid(s)
    before = s["initial"] if s["initial"] is not None else torch.zeros(B, W - 1, C, dtype=dt, device="cuda")
    line = torch.cat((before, torch.where(valid, s["x"], 0.0)), 1)
    at = (s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device="cuda"))[:, None] + torch.arange(W - 1, device="cuda")
    at = at[..., None].expand(B, W - 1, C)
    w = s["weight"]
    z = sum(w[:, j] * line[:, j:j + T].float() for j in range(W)) + s["bias"]
    p = _sigmoid(z)
    y = z * p if c["act"] == "silu" else z
    got = {"y": torch.where(valid, y, 0.0).to(dt)}
    if s["final"] is not None:
        got["final"] = line.gather(1, at)
    if c["kind"] == "conv":
        return got
    d_z = torch.where(valid, s["d_y"].float() * (p * (1 + z * (1 - p)) if c["act"] == "silu" else 1.0), 0.0)
    d_line = torch.zeros(B, T + W - 1, C, device="cuda")
    if s["d_final"] is not None:
        d_line.scatter_add_(1, at, s["d_final"].float())
    for j in range(W):
        d_line[:, j:j + T] += w[:, j] * d_z
    got.update(d_x=torch.where(valid, d_line[:, W - 1:], 0.0).to(dt), d_bias=d_z.sum((0, 1)),
               d_weight=torch.stack([(d_z * line[:, j:j + T].float()).sum((0, 1)) for j in range(W)], 1))
    if s["d_initial"] is not None:
        got["d_initial"] = d_line[:, :W - 1].to(dt)
    return got


def _plain_conv_step(s):
    at = s["slots"].long() if s["slots"] is not None else torch.arange(s["case"]["B"], device="cuda")
    line = torch.cat((s["state"][at], s["x"][:, None]), 1)
    s["state"][at] = line[:, 1:]
    z = (line.float() * s["weight"].t()).sum(1) + s["bias"]
    return {"y": (z * _sigmoid(z)).to(s["x"].dtype), "state": s["state"]}


def _plain_norm(s):
    dt, got = s["x"].dtype, {}
    x = s["x"].float()
    if s["residual"] is not None:  # the stream is stored in its type, and read from there
        got["total"] = (x + s["residual"].float()).to(dt)
        x = got["total"].float()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + s["eps"])
    xh = (x - mean) * rstd
    got["y"] = (xh * s["weight"] + s["bias"]).to(dt)
    if s["case"]["kind"] == "norm":
        return got
    d_y = s["d_y"].float()
    t = d_y * s["weight"]
    d_x = rstd * (t - t.mean(1, keepdim=True) - xh * (t * xh).mean(1, keepdim=True))
    if s["d_total"] is not None:
        d_x = d_x + s["d_total"].float()
    got.update(mean=mean[:, 0], rstd=rstd[:, 0], d_x=d_x.to(dt), d_weight=(d_y * xh).sum(0), d_bias=d_y.sum(0))
    return got


# ----------------------------------------------------------------------------------------------- the library's


def _workspace(s, bytes_):
    """What the caller keeps between calls."""
    if "workspace" not in s:
        n = bytes_()
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return s["workspace"]


def _own_scan(s):
    import paper_2405_05118_amd as mdh

    c = s["case"]
    train = c["kind"] == "scan_train"
    sizes = tuple(c[n] for n in ("B", "T", "D", "N", "G"))
    ws = _workspace(s, lambda: mdh.mdh_selective_scan_workspace_size(sizes, s["x"].dtype, backward=train))
    if train and "checkpoints" not in s:  # what the forward call leaves for the backward call: states along the tokens
        s["checkpoints"] = torch.empty(mdh.mdh_selective_scan_checkpoints_size(sizes), dtype=torch.uint8, device="cuda")
    kept = s.get("checkpoints")
    mdh.mdh_selective_scan(s["x"], s["dt"], s["A"], s["b"], s["c"], s["y"], skip=s["skip"], gate=s["gate"], dt_bias=s["dt_bias"],
                           softplus=True, lengths=s["lengths"], initial_state=s["initial"], final_state=s["final"], checkpoints=kept,
                           workspace=ws)
    got = {"y": s["y"]}
    if s["final"] is not None:
        got["final"] = s["final"]
    if not train:
        return got
    mdh.mdh_selective_scan_backward(s["x"], s["dt"], s["A"], s["b"], s["c"], s["d_y"], s["d_x"], s["d_dt"], s["d_A"], s["d_b"], s["d_c"],
                                    kept, skip=s["skip"], gate=s["gate"], dt_bias=s["dt_bias"], softplus=True, lengths=s["lengths"],
                                    d_final_state=s["d_final"], d_skip=s["d_skip"], d_gate=s["d_gate"], d_dt_bias=s["d_dt_bias"],
                                    d_initial_state=s["d_initial"], workspace=ws)
    got.update((n, s[n]) for n in ("d_x", "d_dt", "d_b", "d_c", "d_A", "d_skip", "d_dt_bias"))
    got.update((n, s[n]) for n in ("d_gate", "d_initial") if s[n] is not None)
    return got


def _own_scan_step(s):
    import paper_2405_05118_amd as mdh

    mdh.mdh_selective_scan_step(s["x"], s["dt"], s["A"], s["b"], s["c"], s["state"], s["y"], skip=s["skip"], gate=s["gate"],
                                dt_bias=s["dt_bias"], softplus=True, slots=s["slots"])
    return {"y": s["y"], "state": s["state"]}


def _own_conv(s):
    import paper_2405_05118_amd as mdh

    c = s["case"]
    act = getattr(mdh, "MDH_ACT_" + c["act"].upper())
    mdh.mdh_causal_conv(s["x"], s["weight"], s["bias"], s["y"], act, lengths=s["lengths"], initial_window=s["initial"],
                        final_window=s["final"])
    got = {"y": s["y"]}
    if s["final"] is not None:
        got["final"] = s["final"]
    if c["kind"] == "conv":
        return got
    ws = _workspace(s, lambda: mdh.mdh_causal_conv_workspace_size(tuple(c[n] for n in ("B", "T", "C", "W")), s["x"].dtype))
    mdh.mdh_causal_conv_backward(s["x"], s["weight"], s["bias"], s["d_y"], s["d_x"], s["d_weight"], s["d_bias"], act,
                                 lengths=s["lengths"], initial_window=s["initial"], d_final_window=s["d_final"],
                                 d_initial_window=s["d_initial"], workspace=ws)
    got.update((n, s[n]) for n in ("d_x", "d_weight", "d_bias"))
    if s["d_initial"] is not None:
        got["d_initial"] = s["d_initial"]
    return got


def _own_conv_step(s):
    import paper_2405_05118_amd as mdh

    mdh.mdh_causal_conv_step(s["x"], s["weight"], s["bias"], s["state"], s["y"], mdh.MDH_ACT_SILU, slots=s["slots"])
    return {"y": s["y"], "state": s["state"]}


def _own_norm(s):
    import paper_2405_05118_amd as mdh

    c = s["case"]
    mdh.mdh_layer_norm(s["x"], s["weight"], s["bias"], s["y"], s["eps"], residual=s["residual"], total=s["total"], mean=s.get("mean"),
                       rstd=s.get("rstd"))
    got = {"y": s["y"]}
    if s["total"] is not None:
        got["total"] = s["total"]
    if c["kind"] == "norm":
        return got
    ws = _workspace(s, lambda: mdh.mdh_layer_norm_workspace_size((c["rows"], c["C"]), s["x"].dtype))
    mdh.mdh_layer_norm_backward(s["x"] if s["total"] is None else s["total"], s["weight"], s["mean"], s["rstd"], s["d_y"], s["d_x"],
                                s["d_weight"], s["d_bias"], d_total=s["d_total"], workspace=ws)
    got.update((n, s[n]) for n in ("mean", "rstd", "d_x", "d_weight", "d_bias"))
    return got


_FORMS = {"scan": (_plain_scan, _own_scan), "scan_train": (_plain_scan, _own_scan), "scan_step": (_plain_scan_step, _own_scan_step),
          "conv": (_plain_conv, _own_conv), "conv_train": (_plain_conv, _own_conv), "conv_step": (_plain_conv_step, _own_conv_step),
          "norm": (_plain_norm, _own_norm), "norm_train": (_plain_norm, _own_norm)}


def run(state):
    return _FORMS[state["case"]["kind"]][bool(own)](state)


# ----------------------------------------------------------------------------------------------- what a pass needs


def work(case):
    e, kind = 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind.startswith("scan"):
        B, D, N, G = (case[n] for n in ("B", "D", "N", "G"))
        tokens, gate = B * case.get("T", 1), 1 if case["gate"] else 0
        shared, params, states = 2 * e * tokens * G * N, 4 * D * (N + 2), 4 * B * D * N
        steps = tokens * D * N  # of the recurrence: a product, an exponential, two products and sums for h, one for y
        if kind == "scan_step":
            return {"bytes": e * tokens * D * (3 + gate) + shared + params + 2 * states, "flops": 7 * steps}
        ends = 2 * states if case["state"] else 0
        forward = e * tokens * D * (3 + gate) + shared + params + ends
        if kind == "scan":
            return {"bytes": forward, "flops": 7 * steps}
        # the recurrence again, its gradient, five sums of products
        return {"bytes": forward + e * tokens * D * (5 + 2 * gate) + 2 * shared + 2 * params + 2 * ends, "flops": (7 + 5 + 3 + 12) * steps}
    if kind.startswith("conv"):
        B, C, W = (case[n] for n in ("B", "C", "W"))
        n, params, windows = B * case.get("T", 1) * C, 4 * C * (W + 1), e * B * (W - 1) * C
        if kind == "conv_step":
            return {"bytes": 2 * e * n + params + 2 * windows, "flops": (2 * W + 5) * n}
        ends = 2 * windows if case["state"] else 0
        if kind == "conv":
            return {"bytes": 2 * e * n + params + ends, "flops": (2 * W + 5) * n}
        return {"bytes": 5 * e * n + 3 * params + 2 * ends, "flops": (8 * W + 15) * n}
    n, extra = case["rows"] * case["C"], 1 if case["residual"] else 0
    if kind == "norm":
        return {"bytes": e * n * (2 + 2 * extra), "flops": 8 * n}
    return {"bytes": e * n * (5 + 3 * extra), "flops": 24 * n}


# ----------------------------------------------------------------------------------------------- in 64 bits


def _exact_scan(s):
    """Token by token as the recurrence says; gradients by differentiating that."""
    c = s["case"]
    B, T, D, N, G = (c[n] for n in ("B", "T", "D", "N", "G"))
    train = c["kind"] == "scan_train"
    leaf = {n: s[n].double().requires_grad_(train) for n in ("x", "dt", "A", "b", "c", "skip", "dt_bias")}
    if s["gate"] is not None:
        leaf["gate"] = s["gate"].double().requires_grad_(train)
    zero = torch.zeros(B, D, N, dtype=torch.float64, device="cuda")
    start = (s["initial"].double() if s["initial"] is not None else zero).requires_grad_(train)
    live = None if s["lengths"] is None else [(s["lengths"] > t)[:, None, None] for t in range(T)]
    h, p = start, []
    delta = torch.nn.functional.softplus(leaf["dt"] + leaf["dt_bias"], threshold=1000.0)
    for t, (xt, dl, bt, ct) in enumerate(zip(leaf["x"].unbind(1), delta.unbind(1), leaf["b"].unbind(1), leaf["c"].unbind(1))):
        u = ((dl * xt).view(B, G, -1, 1) * bt[:, :, None, :]).view(B, D, N)
        new = torch.exp(dl[..., None] * leaf["A"]) * h + u
        h = new if live is None else torch.where(live[t], new, h)
        p.append((h.view(B, G, -1, N) @ ct[..., None]).view(B, D))
    y = torch.stack(p, 1) + leaf["skip"] * leaf["x"]
    if "gate" in leaf:
        y = y * leaf["gate"] * torch.sigmoid(leaf["gate"])
    if live is not None:
        y = torch.where((torch.arange(T, device="cuda") < s["lengths"][:, None])[..., None], y, 0.0)
    got = {"y": y.detach()}
    if s["final"] is not None:
        got["final"] = h.detach()
    if train:
        loss = (y * s["d_y"].double()).sum()
        if s["d_final"] is not None:
            loss = loss + (h * s["d_final"].double()).sum()
        names = list(leaf)
        grads = torch.autograd.grad(loss, [leaf[n] for n in names] + [start])
        got.update(("d_" + n, g) for n, g in zip(names, grads))
        if s["d_initial"] is not None:
            got["d_initial"] = grads[-1]
    return got


def _exact_scan_step(s):
    c = s["case"]
    B, D, N, G = (c[n] for n in ("B", "D", "N", "G"))
    pool = s["state"].double()
    at = s["slots"].long() if s["slots"] is not None else torch.arange(B, device="cuda")
    delta, x = torch.nn.functional.softplus(s["dt"].double() + s["dt_bias"].double(), threshold=1000.0), s["x"].double()
    u = torch.einsum("bge,bgn->bgen", (delta * x).view(B, G, -1), s["b"].double()).reshape(B, D, N)
    new = pool[at] * torch.exp(delta[..., None] * s["A"].double()) + u
    pool[at] = new
    y = torch.einsum("bgen,bgn->bge", new.view(B, G, -1, N), s["c"].double()).reshape(B, D) + s["skip"].double() * x
    if s["gate"] is not None:
        y = y * torch.nn.functional.silu(s["gate"].double())
    return {"y": y, "state": pool}


def _exact_conv(s):
    """The definition over windows of the line of tokens; gradients by differentiating it."""
    c = s["case"]
    B, T, C, W = (c[n] for n in ("B", "T", "C", "W"))
    train = c["kind"] == "conv_train"
    x, w, bias = (s[n].double().requires_grad_(train) for n in ("x", "weight", "bias"))
    before = s["initial"].double() if s["initial"] is not None else torch.zeros(B, W - 1, C, dtype=torch.float64, device="cuda")
    before.requires_grad_(train)
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device="cuda")
    live = (torch.arange(T, device="cuda") < n[:, None])[..., None]
    line = torch.cat((before, x), 1)
    z = (line.unfold(1, W, 1) * w).sum(-1) + bias
    y = torch.where(live, torch.nn.functional.silu(z) if c["act"] == "silu" else z, 0.0)
    final = torch.stack([line[i, int(m):int(m) + W - 1] for i, m in enumerate(n.tolist())])
    got = {"y": y.detach()}
    if s["final"] is not None:
        got["final"] = final.detach()
    if train:
        loss = (y * s["d_y"].double()).sum()
        if s["d_final"] is not None:
            loss = loss + (final * s["d_final"].double()).sum()
        grads = torch.autograd.grad(loss, (x, w, bias, before))
        got.update(d_x=grads[0], d_weight=grads[1], d_bias=grads[2])
        if s["d_initial"] is not None:
            got["d_initial"] = grads[3]
    return got


def _exact_conv_step(s):
    at = s["slots"].long() if s["slots"] is not None else torch.arange(s["case"]["B"], device="cuda")
    pool = s["state"].double()
    now = torch.cat((pool[at], s["x"].double()[:, None]), 1)
    pool[at] = now[:, 1:]
    return {"y": torch.nn.functional.silu(torch.einsum("bwc,cw->bc", now, s["weight"].double()) + s["bias"].double()), "state": pool}


def _exact_norm(s):
    train = s["case"]["kind"] == "norm_train"
    got, x = {}, s["x"].double()
    if s["residual"] is not None:
        got["total"] = x + s["residual"].double()
        x = got["total"].to(s["x"].dtype).double()  # what is normalised is the stream as it is stored
    x, w, b = x.requires_grad_(train), s["weight"].double().requires_grad_(train), s["bias"].double().requires_grad_(train)
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    rstd = (var + s["eps"]) ** -0.5
    y = (x - mean) * rstd * w + b
    got["y"] = y.detach()
    if train:
        d_x, d_w, d_b = torch.autograd.grad((y * s["d_y"].double()).sum(), (x, w, b))
        got.update(mean=mean[:, 0].detach(), rstd=rstd[:, 0].detach(), d_weight=d_w, d_bias=d_b,
                   d_x=d_x if s["d_total"] is None else d_x + s["d_total"].double())
    return got


def exact(case, seed):
    kind = case["kind"]
    if kind in ("scan", "scan_train"):
        # a loop over the tokens, each some ten launches over all states, three times as much with gradients
        train = kind == "scan_train"
        one = case["B"] * case["D"] * case["N"] * 8
        if case["T"] * (3 if train else 1) * (150e-6 + one * 16 / 3e12) > 15 or (train and case["T"] * one * 8 > 60e9):
            return None
    s = prepare(case, seed)
    return {"scan": _exact_scan, "scan_train": _exact_scan, "scan_step": _exact_scan_step, "conv": _exact_conv, "conv_train": _exact_conv,
            "conv_step": _exact_conv_step, "norm": _exact_norm, "norm_train": _exact_norm}[kind](s)
