"""Linear attention with a decay for each head, and group norm with an activation: work to be timed and checked.

``own`` chooses between the operators' plain forms (elementary torch operations in 32 bits) and this library's
entry points.  A case names the operator, its sizes and its types; ``prepare`` makes what a program has in hand before
the call, ``run`` is one pass, ``exact`` the same from the definitions in 64 bits.

Layouts: q, k, v and o are (batch, token, head, channel), states (batch or slot, head, dk, dv) in fp32, images and rows
of activations (N, positions, channels).  ``decay`` is given as its natural logarithm, one for each head.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ----------------------------------------------------------------------------------------------- the cases


def _la(kind, dtype, B, T, H, dk, dv, Hq=None, Hk=None, Hv=None, ragged=False, state=False, fused=False):
    return {"kind": kind, "dtype": dtype, "B": B, "T": T, "H": H, "Hq": Hq or H, "Hk": Hk or H, "Hv": Hv or H, "dk": dk, "dv": dv,
            "ragged": ragged, "state": state, "fused": fused}


def _step(dtype, B, H, dk, dv, slots=0, Hq=None, Hk=None, Hv=None):
    return {"kind": "linattn_step", "dtype": dtype, "B": B, "H": H, "Hq": Hq or H, "Hk": Hk or H, "Hv": Hv or H, "dk": dk, "dv": dv,
            "slots": slots}


def _gn(kind, dtype, N, S, C, G, act, gate=False):
    return {"kind": kind, "dtype": dtype, "N": N, "S": S, "C": C, "G": G, "act": act, "gate": gate}


def _named(name, case):
    return dict(case, name=name)


def listed():
    return [
        # one request's prompt, its projections in one buffer; the state goes on to the generation of tokens
        _named("la_prompt", _la("linattn", "bf16", 1, 2048, 32, 128, 128, state=True, fused=True)),
        # prompts of several requests padded to the longest, one of them empty, queries and keys shared by three heads each
        _named("la_ragged", _la("linattn", "bf16", 6, 1021, 12, 80, 96, Hq=4, Hk=4, ragged=True, state=True)),
        # one long document, few heads: the work has to be split along the tokens
        _named("la_long", _la("linattn", "bf16", 1, 65536, 16, 128, 128)),
        # a training step's layer: outputs and all gradients
        _named("la_train", _la("linattn_train", "bf16", 8, 4096, 16, 128, 128)),
        # the same in fp32 on pieces of a longer text: a state comes in and its gradient goes on; an odd number of tokens
        _named("la_train_f32", _la("linattn_train", "f32", 2, 2001, 8, 64, 128, state=True)),
        # the next token of one request
        _named("la_step_one", _step("bf16", 1, 32, 128, 128)),
        # the next token of many requests, their states in a pool of which some slots are not in use
        _named("la_step_many", _step("bf16", 250, 16, 128, 128, slots=300)),
        # the heads of one request's next token, normalised and gated
        _named("gn_token", _gn("group_norm", "bf16", 1, 1, 4096, 32, "silu", gate=True)),
        # the same over a training batch's tokens, with all gradients
        _named("gn_rows_train", _gn("group_norm_train", "bf16", 16384, 1, 4096, 32, "silu", gate=True)),
        # what follows an ordinary 3 x 3 convolution layer: images of 56 x 56, two channels a group
        _named("gn_image", _gn("group_norm", "f32", 16, 56 * 56, 64, 32, "relu")),
        # larger images in training
        _named("gn_image_train", _gn("group_norm_train", "bf16", 8, 128 * 128, 256, 32, "silu")),
        # sizes that divide nothing: five channels a group
        _named("gn_ragged", _gn("group_norm_train", "f32", 3, 1021, 120, 24, "gelu")),
    ]


def _log(rng, lo, hi):
    """Whole number, uniform over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng):
    """Channels of a head: mostly what vector loads like, else any."""
    return 8 * rng.randint(3, 20) if rng.random() < 0.7 else rng.randint(17, 160)


def _heads(rng):
    """(H, Hq, Hk, Hv): mostly as many of each, else queries and keys shared, or keys and values."""
    H = rng.choice([4, 6, 8, 12, 16, 24, 32])
    u, few = rng.random(), H // 2
    return (H, H, H, H) if u < 0.6 else (H, few, few, H) if u < 0.8 else (H, H, few, few)


def _draw_la(rng):
    kind = rng.choice(["linattn", "linattn_train"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    H, Hq, Hk, Hv = _heads(rng)
    dk, dv = _width(rng), _width(rng)
    # values of one operand: at most those of the largest listed training step, a quarter of that in fp32
    most = (8 * 4096 * 16 * 128) // (4 if dtype == "f32" else 1)
    T = _log(rng, 1, 8192 if kind == "linattn_train" else 32768)
    B = _log(rng, 1, 32)
    wide = H * max(dk, dv) * max(128, min(dk, dv)) // 128
    while B > 1 and B * T * wide > most:
        B -= 1
    T = max(1, min(T, most // (B * wide)))
    return _la(kind, dtype, B, T, H, dk, dv, Hq, Hk, Hv, ragged=rng.random() < 0.4, state=rng.random() < 0.5, fused=rng.random() < 0.3)


def _draw_step(rng):
    H, Hq, Hk, Hv = _heads(rng)
    dk, dv = _width(rng), _width(rng)
    B = max(1, min(_log(rng, 1, 400), (250 * 16 * 128 * 128) // (H * dk * dv)))
    return _step("f32" if rng.random() < 0.3 else "bf16", B, H, dk, dv, B + rng.randint(1, 20) if rng.random() < 0.5 else 0, Hq, Hk, Hv)


def _draw_gn(rng):
    kind = rng.choice(["group_norm", "group_norm_train"])
    dtype = "f32" if rng.random() < 0.4 else "bf16"
    # (no relu in training: its slope jumps where z is 0, and a z within rounding of 0 has either)
    act = rng.choice(["none", "silu", "gelu", "relu" if kind == "group_norm" else "silu"])
    most = 8 * 128 * 128 * 256
    if rng.random() < 0.5:  # rows of heads
        G = rng.choice([4, 8, 12, 16, 32])
        C = G * _width(rng)
        return _gn(kind, dtype, max(1, min(_log(rng, 1, 32768), most // C)), 1, C, G, act, gate=rng.random() < 0.7)
    G = rng.choice([4, 8, 16, 24, 32])
    C = G * _log(rng, 1, 24)
    N = _log(rng, 1, 32)
    return _gn(kind, dtype, N, max(1, min(_log(rng, 4, 40000), most // (C * N))), C, G, act, gate=rng.random() < 0.2)


def draw(rng):
    u = rng.random()
    return _draw_la(rng) if u < 0.45 else _draw_step(rng) if u < 0.6 else _draw_gn(rng)


# ----------------------------------------------------------------------------------------------- the inputs


def _normal(gen, *shape, dtype=torch.float32, times=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * times).to(dtype)


def _log_decay(H):
    """Memories from 8 to 2000 tokens, one for each head: ln(1 - 2^-x), x from 3 to 11."""
    x = torch.linspace(3, 11, H, dtype=torch.float64) if H > 1 else torch.full((1,), 6.0, dtype=torch.float64)
    return torch.log1p(-torch.exp2(-x)).to(torch.float32).cuda()


def _lengths(case, gen):
    """Any from nothing to all of it, with the first the longest and the second empty."""
    at = torch.randint(0, case["T"] + 1, (case["B"],), generator=gen, device="cuda")
    at[0] = case["T"]
    if case["B"] > 1:
        at[1] = 0
    return at.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = _TYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"].startswith("linattn"):
        H, Hq, Hk, Hv, dk, dv, B = (case[n] for n in ("H", "Hq", "Hk", "Hv", "dk", "dv", "B"))
        s["log_decay"], s["scale"] = _log_decay(H), dk ** -0.5
        lead = (B,) if case["kind"] == "linattn_step" else (B, case["T"])
        if case.get("fused"):  # one projection makes all three
            qkv = _normal(gen, *lead, Hq * dk + Hk * dk + Hv * dv, dtype=dt)
            q, k, v = qkv.split((Hq * dk, Hk * dk, Hv * dv), dim=-1)
        else:
            q, k, v = (_normal(gen, *lead, n, dtype=dt) for n in (Hq * dk, Hk * dk, Hv * dv))
        s["q"], s["k"], s["v"] = q.unflatten(-1, (Hq, dk)), k.unflatten(-1, (Hk, dk)), v.unflatten(-1, (Hv, dv))
        s["o"] = torch.empty(*lead, H, dv, dtype=dt, device="cuda")
        if case["kind"] == "linattn_step":
            n = case["slots"]
            s["state"] = _normal(gen, n or B, H, dk, dv, times=2.0)
            s["slots"] = torch.randperm(n, generator=gen, device="cuda")[:B].to(torch.int32) if n else None
            return s
        s["lengths"] = _lengths(case, gen) if case["ragged"] else None
        s["initial"] = _normal(gen, B, H, dk, dv, times=2.0) if case["state"] else None
        s["final"] = torch.empty(B, H, dk, dv, device="cuda") if case["state"] else None
        if case["kind"] == "linattn_train":
            s["d_o"] = _normal(gen, *lead, H, dv, dtype=dt)
            for n in ("q", "k", "v"):
                s["d_" + n] = torch.empty(s[n].shape, dtype=dt, device="cuda")
            s["d_final"] = _normal(gen, B, H, dk, dv) if case["state"] else None
            s["d_initial"] = torch.empty(B, H, dk, dv, device="cuda") if case["state"] else None
        return s
    N, S, C, G = (case[n] for n in "NSCG")
    s["x"] = (_normal(gen, N, S, C) * (0.5 + torch.rand(C, generator=gen, device="cuda")) + _normal(gen, C)).to(dt)
    s["gate"] = _normal(gen, N, S, C, dtype=dt) if case["gate"] else None
    s["weight"], s["bias"] = 1 + _normal(gen, C, times=0.2), _normal(gen, C, times=0.2)
    s["eps"] = 1e-5
    s["y"] = torch.empty_like(s["x"])
    if case["kind"] == "group_norm_train":
        s["d_y"] = _normal(gen, N, S, C, dtype=dt)
        s["mean"], s["rstd"] = (torch.empty(N, G, device="cuda") for _ in range(2))
        s["d_x"] = torch.empty_like(s["x"])
        s["d_gate"] = torch.empty_like(s["x"]) if case["gate"] else None
        s["d_weight"], s["d_bias"] = (torch.empty(C, device="cuda") for _ in range(2))
    return s


# ----------------------------------------------------------------------------------------------- the plain forms


def _per_head(x, H):
    """(batch, token, heads that may be shared, channel) as (batch, H, token, channel) in 32 bits."""
    return x.float().repeat_interleave(H // x.shape[2], dim=2).transpose(1, 2)


def _shared(x, n, dtype):
    """The other way: gradients of every head, summed for each that shares an operand."""
    B, H, T, d = x.shape
    return x.transpose(1, 2).reshape(B, T, n, H // n, d).sum(3).to(dtype)


def _turned(x, lengths):
    """Every sequence's valid tokens in reverse order."""
    B, H, T, d = x.shape
    at = (lengths[:, None] - 1 - torch.arange(T, device="cuda")).clamp_min(0)
    return x.gather(2, at[:, None, :, None].expand(B, H, T, d))


def _plain_pass(a, b, c, g, lengths, state, scale, first, scale_state):
    """out_i = scale sum_{j<=i} l^{i-j} (a_i.b_j) c_j + l^{i+first} a_i state, and the state behind the last valid token,
    in chunks: products within them, and of every chunk with the sums of those before it.  `first` is 1 where a token
    reads the state after its own decay, else 0; what enters the state is multiplied by scale_state."""
    B, H, T, da = a.shape
    dc, C = c.shape[-1], min(T, 128 if T <= 8192 else 256)
    n = -(-T // C)
    valid = (torch.arange(T, device="cuda") < lengths[:, None])[:, None, :, None]
    a, b, c = (torch.where(valid, x, 0.0) for x in (a, b, c))
    g = g[:, None]
    left = (lengths[:, None] - 1 - torch.arange(T, device="cuda")).clamp_min(0) + (1 - first)
    end = (scale_state * b * torch.exp(g * left[:, None, :])[..., None]).transpose(2, 3) @ c
    if state is not None:
        end = end + torch.exp(g[:, 0] * lengths[:, None])[..., None, None] * state
    a, b, c = (torch.nn.functional.pad(x, (0, 0, 0, n * C - T)).reshape(B, H, n, C, x.shape[-1]) for x in (a, b, c))
    i = torch.arange(C, device="cuda")
    near = torch.where(i[:, None] >= i, torch.exp(g[..., None] * (i[:, None] - i).clamp_min(0)), 0.0) * scale
    out = ((a @ b.transpose(3, 4)) * near[:, None]) @ c
    part = (scale_state * b * torch.exp(g * (C - first - i))[:, None, :, None]).transpose(3, 4) @ c
    m = torch.arange(n, device="cuda")
    far = torch.where(m[:, None] > m, torch.exp(g[..., None] * C * (m[:, None] - 1 - m).clamp_min(0)), 0.0)
    before = (far @ part.reshape(B, H, n, da * dc)).reshape(B, H, n, da, dc)
    if state is not None:
        before = before + torch.exp(g * C * m)[:, :, None, None] * state[:, :, None]
    read = scale / scale_state
    out = out + (read * a * torch.exp(g * (i + first))[:, None, :, None]) @ before
    return out.reshape(B, H, n * C, dc)[:, :, :T], end


def _plain_linattn(s):
    H, T, B, dt = s["case"]["H"], s["case"]["T"], s["case"]["B"], s["q"].dtype
    lengths = s["lengths"] if s["lengths"] is not None else torch.full((B,), T, device="cuda")
    q, k, v = (_per_head(s[n], H) for n in ("q", "k", "v"))
    g, scale, state = s["log_decay"], s["scale"], s["initial"]
    o, end = _plain_pass(q, k, v, g, lengths, state, scale, 1, 1.0)
    got = {"o": o.transpose(1, 2).to(dt)}
    if s["final"] is not None:
        got["final"] = end
    if s["case"]["kind"] == "linattn":
        return got
    d_o = _per_head(s["d_o"], H)
    d_q, _ = _plain_pass(d_o, v, k, g, lengths, None if state is None else state.transpose(2, 3), scale, 1, 1.0)
    q, k, v, d_o = (_turned(x, lengths) for x in (q, k, v, d_o))
    d_end = s["d_final"]
    d_k, _ = _plain_pass(v, d_o, q, g, lengths, None if d_end is None else d_end.transpose(2, 3), scale, 0, scale)
    d_v, d_initial = _plain_pass(k, q, d_o, g, lengths, d_end, scale, 0, scale)
    valid = (torch.arange(T, device="cuda") < lengths[:, None])[:, None, :, None]
    d_k, d_v = (torch.where(valid, _turned(x, lengths), 0.0) for x in (d_k, d_v))
    got.update(d_q=_shared(d_q, s["case"]["Hq"], dt), d_k=_shared(d_k, s["case"]["Hk"], dt), d_v=_shared(d_v, s["case"]["Hv"], dt))
    if d_end is not None:
        got["d_initial"] = d_initial
    return got


def _plain_step(s):
    H = s["case"]["H"]
    q, k, v = (s[n].float().repeat_interleave(H // s[n].shape[1], dim=1) for n in ("q", "k", "v"))
    l = torch.exp(s["log_decay"])[:, None, None]
    if s["slots"] is None:
        now = s["state"].mul_(l).add_(k[..., :, None] * v[..., None, :])
    else:
        at = s["slots"].long()
        now = s["state"][at] * l + k[..., :, None] * v[..., None, :]
        s["state"][at] = now
    return {"o": (s["scale"] * (q[..., None, :] @ now)[..., 0, :]).to(s["q"].dtype), "state": s["state"]}


def _act(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5))) if name == "gelu" else z


def _slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _plain_group_norm(s):
    c = s["case"]
    N, S, C, G, act = c["N"], c["S"], c["C"], c["G"], c["act"]
    dt = s["x"].dtype
    x = s["x"].float().reshape(N, S, G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean((1, 3), keepdim=True) + s["eps"])
    xh = (x - mean) * rstd
    w = s["weight"].reshape(G, -1)
    z = xh * w + s["bias"].reshape(G, -1)
    gate = None if s["gate"] is None else s["gate"].float().reshape(x.shape)
    y = _act(z, act) if gate is None else z * _act(gate, act)
    got = {"y": y.reshape(N, S, C).to(dt)}
    if c["kind"] == "group_norm":
        return got
    d_y = s["d_y"].float().reshape(x.shape)
    d_z = d_y * (_slope(z, act) if gate is None else _act(gate, act))
    if gate is not None:
        got["d_gate"] = (d_y * z * _slope(gate, act)).reshape(N, S, C).to(dt)
    t = d_z * w
    d_x = rstd * (t - t.mean((1, 3), keepdim=True) - xh * (t * xh).mean((1, 3), keepdim=True))
    got.update(mean=mean.reshape(N, G), rstd=rstd.reshape(N, G), d_x=d_x.reshape(N, S, C).to(dt),
               d_weight=(d_z * xh).sum((0, 1)).reshape(C), d_bias=d_z.sum((0, 1)).reshape(C))
    return got


# ----------------------------------------------------------------------------------------------- the library's


def _workspace(s, bytes_):
    """What the caller keeps between calls."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(bytes_, dtype=torch.uint8, device="cuda") if bytes_ else None
    return s["workspace"]


def _own_linattn(s):
    import paper_2405_05118_amd as mdh

    c = s["case"]
    if "workspace" not in s:
        sizes = tuple(c[n] for n in ("B", "T", "H", "Hq", "Hk", "Hv", "dk", "dv"))
        _workspace(s, mdh.mdh_linattn_workspace_size(sizes, s["q"].dtype, backward=c["kind"] == "linattn_train"))
    mdh.mdh_linattn(s["q"], s["k"], s["v"], s["log_decay"], s["o"], s["scale"], lengths=s["lengths"], initial_state=s["initial"],
                    final_state=s["final"], workspace=s["workspace"])
    got = {"o": s["o"]}
    if s["final"] is not None:
        got["final"] = s["final"]
    if c["kind"] == "linattn":
        return got
    mdh.mdh_linattn_backward(s["q"], s["k"], s["v"], s["log_decay"], s["d_o"], s["d_q"], s["d_k"], s["d_v"], s["scale"],
                             lengths=s["lengths"], initial_state=s["initial"], d_final_state=s["d_final"],
                             d_initial_state=s["d_initial"], workspace=s["workspace"])
    got.update(d_q=s["d_q"], d_k=s["d_k"], d_v=s["d_v"])
    if s["d_initial"] is not None:
        got["d_initial"] = s["d_initial"]
    return got


def _own_step(s):
    import paper_2405_05118_amd as mdh

    mdh.mdh_linattn_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["o"], s["scale"], slots=s["slots"])
    return {"o": s["o"], "state": s["state"]}


def _own_group_norm(s):
    import paper_2405_05118_amd as mdh

    c = s["case"]
    train = c["kind"] == "group_norm_train"
    if "workspace" not in s:
        _workspace(s, mdh.mdh_group_norm_workspace_size((c["N"], c["S"], c["C"], c["G"]), s["x"].dtype, backward=train))
    act = getattr(mdh, "MDH_ACT_" + c["act"].upper())
    mdh.mdh_group_norm(s["x"], s["weight"], s["bias"], s["y"], c["G"], s["eps"], act, gate=s["gate"], mean=s.get("mean"),
                       rstd=s.get("rstd"), workspace=s["workspace"])
    got = {"y": s["y"]}
    if not train:
        return got
    mdh.mdh_group_norm_backward(s["x"], s["weight"], s["bias"], s["mean"], s["rstd"], s["d_y"], s["d_x"], s["d_weight"], s["d_bias"],
                                c["G"], act, gate=s["gate"], d_gate=s["d_gate"], workspace=s["workspace"])
    if s["d_gate"] is not None:
        got["d_gate"] = s["d_gate"]
    got.update((n, s[n]) for n in ("mean", "rstd", "d_x", "d_weight", "d_bias"))
    return got


def run(state):
    kind = state["case"]["kind"]
    if kind == "linattn_step":
        return (_own_step if own else _plain_step)(state)
    if kind.startswith("linattn"):
        return (_own_linattn if own else _plain_linattn)(state)
    return (_own_group_norm if own else _plain_group_norm)(state)


# ----------------------------------------------------------------------------------------------- what a pass needs


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"].startswith("linattn"):
        B, H, Hq, Hk, Hv, dk, dv = (case[n] for n in ("B", "H", "Hq", "Hk", "Hv", "dk", "dv"))
        T = case.get("T", 1)
        states, tokens = 4 * B * H * dk * dv, B * T
        inputs, outputs = e * tokens * (Hq * dk + Hk * dk + Hv * dv), e * tokens * H * dv
        flops = 4 * tokens * H * dk * dv  # a state's update and its product with q
        if case["kind"] == "linattn_step":
            return {"bytes": inputs + outputs + 2 * states, "flops": flops}
        if case["kind"] == "linattn":
            return {"bytes": inputs + outputs + (2 * states if case["state"] else 0), "flops": flops}
        # and the other state's update, and three products with states
        return {"bytes": 2 * inputs + 2 * outputs + (4 * states if case["state"] else 0), "flops": 3 * flops}
    n = case["N"] * case["S"] * case["C"]
    if case["kind"] == "group_norm":
        return {"bytes": e * n * (3 if case["gate"] else 2), "flops": 10 * n}
    return {"bytes": e * n * (6 if case["gate"] else 4), "flops": 30 * n}


# ----------------------------------------------------------------------------------------------- in 64 bits


def _exact_linattn(s):
    """Token by token, as the recurrence says."""
    c = s["case"]
    H, T, B = c["H"], c["T"], c["B"]
    q, k, v = (s[n].double().repeat_interleave(H // s[n].shape[2], dim=2) for n in ("q", "k", "v"))
    l = torch.exp(s["log_decay"].double())[:, None, None]
    length = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device="cuda")
    start = s["initial"].double() if s["initial"] is not None else torch.zeros(B, H, c["dk"], c["dv"], dtype=torch.float64, device="cuda")
    train, scale = c["kind"] == "linattn_train", s["scale"]
    d_o = s["d_o"].double() if train else None
    live = (torch.arange(T, device="cuda") < length[:, None])[:, :, None, None]
    o, d_q, at = [], [], start
    for t in range(T):
        new = l * at + k[:, t, :, :, None] * v[:, t, :, None, :]
        o.append((q[:, t, :, None, :] @ new)[:, :, 0])
        if train:
            d_q.append((new @ d_o[:, t, :, :, None])[..., 0])
        at = new if c["T"] == 1 or not c["ragged"] else torch.where(live[:, t, :, :, None], new, at)
    got = {"o": torch.where(live, scale * torch.stack(o, 1), 0.0)}
    if s["final"] is not None:
        got["final"] = torch.where((length > 0)[:, None, None, None], at, start)
    if not train:
        return got
    d_k, d_v = [], []
    grad = s["d_final"].double() if s["d_final"] is not None else torch.zeros_like(start)
    for t in reversed(range(T)):
        full = grad + scale * q[:, t, :, :, None] * d_o[:, t, :, None, :]
        d_k.append((full @ v[:, t, :, :, None])[..., 0])
        d_v.append((k[:, t, :, None, :] @ full)[:, :, 0])
        grad = torch.where(live[:, t, :, :, None], l * full, grad)
    for name, x, n in (("d_q", scale * torch.stack(d_q, 1), c["Hq"]), ("d_k", torch.stack(d_k[::-1], 1), c["Hk"]),
                       ("d_v", torch.stack(d_v[::-1], 1), c["Hv"])):
        got[name] = torch.where(live, x, 0.0).reshape(B, T, n, H // n, -1).sum(3)
    if s["d_initial"] is not None:
        got["d_initial"] = grad
    return got


def _exact_step(s):
    H = s["case"]["H"]
    q, k, v = (s[n].double().repeat_interleave(H // s[n].shape[1], dim=1) for n in ("q", "k", "v"))
    all_states = s["state"].double()
    at = s["slots"].long() if s["slots"] is not None else torch.arange(q.shape[0], device="cuda")
    new = all_states[at] * torch.exp(s["log_decay"].double())[:, None, None] + torch.einsum("bhi,bhj->bhij", k, v)
    all_states[at] = new
    return {"o": s["scale"] * torch.einsum("bhi,bhij->bhj", q, new), "state": all_states}


def _exact_group_norm(s):
    """Forward by the definition, gradients by differentiating it."""
    c = s["case"]
    train, act = c["kind"] == "group_norm_train", c["act"]
    x, w, b = (s[n].double().requires_grad_(train) for n in ("x", "weight", "bias"))
    gate = s["gate"].double().requires_grad_(train) if s["gate"] is not None else None
    f = {"none": lambda u: u, "relu": torch.relu, "silu": lambda u: u * torch.sigmoid(u),
         "gelu": lambda u: u * (1 - 0.5 * torch.special.erfc(u / math.sqrt(2)))}[act]
    grouped = x.unflatten(2, (c["G"], -1))
    var, mean = torch.var_mean(grouped, (1, 3), correction=0, keepdim=True)
    rstd = (var + s["eps"]) ** -0.5
    z = ((grouped - mean) * rstd).flatten(2) * w + b
    y = f(z) if gate is None else z * f(gate)
    if not train:
        return {"y": y}
    inputs = [x, w, b] + ([gate] if gate is not None else [])
    grads = torch.autograd.grad(y, inputs, s["d_y"].double())
    got = {"y": y, "mean": mean.flatten(1), "rstd": rstd.flatten(1), "d_x": grads[0], "d_weight": grads[1], "d_bias": grads[2]}
    if gate is not None:
        got["d_gate"] = grads[3]
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "linattn_step":
        return _exact_step(s)
    if case["kind"].startswith("linattn"):
        # two loops over the tokens, each token some ten launches over all states
        cost = case["T"] * (3 if case["kind"] == "linattn_train" else 1) * (120e-6 + case["B"] * case["H"] * case["dk"] * case["dv"] * 8 * 8 / 3e12)
        return _exact_linattn(s) if cost < 15 else None
    return _exact_group_norm(s)
