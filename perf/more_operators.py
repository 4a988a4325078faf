"""What is timed of the layers of policies whose memory is of constant size and chooses what it keeps: the selective scan, the short
causal convolution in front of it, and the norms of queries and keys with the position rotation, as they stand in front of
decay attention.

Each operator is here in its plain form (elementary torch operations in 32 bits, angles and long sums in 64) and as the call a
user makes of the library (`own`).  The kinds:

  conv, conv_bwd, conv_step   convolution along the steps of each env, its gradients, one decision with the state in place
  scan, scan_bwd, scan_step   selective scan, its gradients, one decision with the state in place
  heads, heads_bwd            norms of queries and keys with the rotation, and their gradients
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------------------- cases --


def _conv(kind, T, Be, C, width, act, dtype, done=0.0, state=True):
    return {"kind": kind, "T": T, "Be": Be, "C": C, "width": width, "act": act, "dtype": dtype, "done": done, "state": state}


def _scan(kind, T, Be, C, N, groups, dtype, done=0.0, state=True, gate=True):
    return {"kind": kind, "T": T, "Be": Be, "C": C, "N": N, "groups": groups, "dtype": dtype, "done": done, "state": state, "gate": gate}


def _heads(kind, rows, heads, kv, d, rot, interleaved, dtype, first=0, base=10000.0):
    return {"kind": kind, "rows": rows, "heads": heads, "kv": kv, "d": d, "rot": rot, "interleaved": interleaved, "dtype": dtype, "first": first,
            "base": base}


def listed():
    named = [
        # one decision of a simulator GPU's envs
        ("conv_step", _conv("conv_step", 1, 512, 4096, 4, "silu", "bf16", 0.01)),
        # one long prompt, several documents packed behind one another
        ("conv_prompt", _conv("conv", 8192, 1, 4096, 4, "silu", "bf16", 0.0005)),
        # gradients of a training minibatch of the recurrent policy's shape: 16 steps of 256 envs
        ("conv_bwd", _conv("conv_bwd", 16, 256, 2048, 4, "silu", "bf16", 0.01)),
        # one decision of a handful of envs (evaluation, the deployed gripper): latency
        ("scan_step_16", _scan("scan_step", 1, 16, 1024, 16, 1, "bf16")),
        # one decision of a simulator GPU's envs: the states go through once
        ("scan_step_512", _scan("scan_step", 1, 512, 4096, 16, 1, "bf16", 0.01)),
        # outputs of the training minibatch, state carried in and out
        ("scan_rollout", _scan("scan", 16, 256, 2048, 16, 1, "bf16", 0.01)),
        # the long prompt
        ("scan_prompt", _scan("scan", 8192, 1, 4096, 16, 1, "bf16", 0.0005)),
        # gradients of the training minibatch
        ("scan_bwd_rollout", _scan("scan_bwd", 16, 256, 2048, 16, 1, "bf16", 0.01)),
        # gradients in 32 bits, odd sizes everywhere, no gate
        ("scan_bwd_odd_f32", _scan("scan_bwd", 119, 37, 202, 12, 2, "f32", 0.01, True, False)),
        # gradients of a few long sequences
        ("scan_bwd_long", _scan("scan_bwd", 2048, 2, 2048, 16, 1, "bf16", 0.001, False)),
        # queries and keys of a batch of prompts, late in a long context, key heads shared by four
        ("heads_prompt", _heads("heads", 16384, 16, 4, 128, 128, False, "bf16", 200000, 500000.0)),
        # gradients of a training minibatch, half of each head turned
        ("heads_bwd", _heads("heads_bwd", 4096, 16, 16, 64, 32, True, "bf16")),
    ]
    return [dict(case, name=name) for name, case in named]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("conv", "conv_bwd", "conv_step", "scan", "scan", "scan_bwd", "scan_bwd", "scan_step", "heads", "heads_bwd"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    size = 2 if dtype == "f32" else 1  # 32-bit cases of half the elements: no more bytes than the listed ones
    done = rng.choice((0.0, 0.002, 0.02))
    if kind in ("heads", "heads_bwd"):
        kv = rng.choice((1, 2, 3, 4, 8))
        heads = kv * rng.choice((1, 2, 4))
        d = rng.choice((64, 128, 128)) if rng.random() < 0.6 else 2 * rng.randint(8, 128)
        rot = d if rng.random() < 0.6 else 2 * rng.randint(0, d // 2)
        most = (40000000 if kind == "heads" else 8000000) // size // (heads + kv) // d
        return _heads(kind, _log(rng, 1, min(most, 65536)), heads, kv, d, rot, rng.random() < 0.5, dtype, rng.choice((0, 5000, 1000000)),
                      rng.choice((10000.0, 500000.0)))
    if kind in ("conv", "conv_bwd", "conv_step"):
        C = rng.choice((512, 1024, 2048, 4096)) if rng.random() < 0.6 else _log(rng, 3, 8192)
        width, act = rng.choice((2, 3, 4, 4, 4, 8)), rng.choice(("silu", "silu", "none"))
        if kind == "conv_step":
            return _conv(kind, 1, _log(rng, 1, min(2048, 2000000 // size // C)), C, width, act, dtype, done)
        most = (32000000 if kind == "conv" else 8000000) // size // C
        T = _log(rng, 1, min(8192, most))
        return _conv(kind, T, _log(rng, 1, most // T), C, width, act, dtype, done, rng.random() < 0.7)
    groups = rng.choice((1, 1, 2, 4))
    C = rng.choice((512, 1024, 2048, 4096)) if rng.random() < 0.6 else groups * _log(rng, 3, 8192 // groups)
    N = rng.choice((16, 16, 16, 8, 32, 64, rng.randint(1, 64)))
    if kind == "scan_step":
        return _scan(kind, 1, _log(rng, 1, min(2048, 32000000 // C // N)), C, N, groups, dtype, done, True, rng.random() < 0.7)
    # states of all steps, padded to 16, stay below those of the largest listed cases
    most = (500000000 if kind == "scan" else 130000000) // size // C // max(N, 16)
    T = _log(rng, 1, min(8192 if kind == "scan" else 2048, most))
    return _scan(kind, T, _log(rng, 1, min(2048, most // T)), C, N, groups, dtype, done, rng.random() < 0.7, rng.random() < 0.7)


# ------------------------------------------------------------------------------------------------------------ inputs --


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _TYPES[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    kind, f32 = case["kind"], torch.float32
    s = {"case": dict(case)}
    if kind in ("heads", "heads_bwd"):
        rows, heads, kv, d, rot = (case[n] for n in ("rows", "heads", "kv", "d", "rot"))
        # projections whose heads differ in size
        s["q"] = (normal(rows, heads, d, dtype=f32) * (0.5 + 2 * uniform(heads, 1))).to(dt)
        s["k"] = (normal(rows, kv, d, dtype=f32) * (0.5 + 2 * uniform(kv, 1))).to(dt)
        s["gamma_q"], s["gamma_k"] = 1 + 0.2 * normal(d, dtype=f32), 1 + 0.2 * normal(d, dtype=f32)
        s["freq"] = case["base"] ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / max(rot, 1))
        # documents that start anywhere: positions count up from each start
        start = torch.randint(0, 1 + rows, (), generator=g, device="cuda")
        row = torch.arange(rows, device="cuda")
        s["pos"] = (case["first"] + torch.where(row < start, row, row - start)).to(torch.int32)
        if kind == "heads":
            s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        else:
            s["dq_out"], s["dk_out"] = normal(rows, heads, d), normal(rows, kv, d)
            s["dq"], s["dk"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
            s["dgamma_q"], s["dgamma_k"] = torch.empty_like(s["gamma_q"]), torch.empty_like(s["gamma_k"])
        return s
    T, Be, C = case["T"], case["Be"], case["C"]
    # a set flag ends an episode, or a document, at that step; a decision is given the flags of the step before
    s["done"] = (uniform(T, Be) < case["done"]).to(torch.uint8)
    if kind in ("conv", "conv_bwd", "conv_step"):
        W = case["width"]
        s["x"] = normal(T, Be, C)
        s["weight"], s["bias"] = normal(C, W, dtype=f32) * W ** -0.5, 0.2 * normal(C, dtype=f32)
        s["state_in"] = normal(Be, W - 1, C) if case["state"] else None
        if kind == "conv_bwd":
            s["dy"], s["dx"] = normal(T, Be, C), torch.empty_like(s["x"])
            s["dstate_out"] = normal(Be, W - 1, C) if case["state"] else None
            s["dstate_in"] = torch.empty_like(s["state_in"]) if case["state"] else None
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
        else:
            s["y"] = torch.empty_like(s["x"])
            s["state_out"] = torch.empty_like(s["state_in"]) if case["state"] else None
        return s
    N, groups = case["N"], case["groups"]
    x = normal(T, Be, C, dtype=f32)
    s["x"] = (x * torch.sigmoid(x)).to(dt)  # behind the convolution's activation
    # step sizes from some thousandths to a few tenths, that the data moves about
    step = torch.exp(math.log(1e-3) + math.log(100.0) * uniform(C))
    s["dt"], s["dt_bias"] = normal(T, Be, C), step + torch.log(-torch.expm1(-step))
    s["A"] = -torch.arange(1, N + 1, device="cuda", dtype=f32) * torch.exp(0.1 * normal(C, N, dtype=f32))
    s["B"], s["C"] = normal(T, Be, groups, N), normal(T, Be, groups, N)
    s["D"] = 1 + 0.2 * normal(C, dtype=f32)
    s["z"] = normal(T, Be, C) if case["gate"] else None
    s["state_in"] = 0.3 * normal(Be, C, N, dtype=f32) if case["state"] else None
    if kind == "scan_bwd":
        s["dy"] = normal(T, Be, C)
        s["dstate_out"] = normal(Be, C, N, dtype=f32) if case["state"] else None
        s["dstate_in"] = torch.empty_like(s["state_in"]) if case["state"] else None
        for n in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias"):
            s["d" + n] = torch.empty_like(s[n]) if s[n] is not None else None
    else:
        s["y"] = torch.empty_like(s["x"])
        s["state_out"] = torch.empty_like(s["state_in"]) if case["state"] else None
    return s


# ------------------------------------------------------------------------------------------------------- plain forms --


def _history(s):
    """x in 32 bits with the width - 1 inputs in front of the sequence, [T + width - 1, Be, C]; and for each step and tap whether
    no flag lies between them, [width, T, Be, 1]: tap i reads row t + i."""
    c = s["case"]
    T, Be, W = c["T"], c["Be"], c["width"]
    old = torch.zeros((W - 1, Be, c["C"]), device="cuda") if s["state_in"] is None else s["state_in"].float().transpose(0, 1)
    flags = torch.zeros((W - 1 + T + 1, Be), device="cuda", dtype=torch.int32)
    flags[W:] = s["done"].int()  # flag of step t at row t + W, so that ...
    count = torch.cumsum(flags, 0)  # ... row t + W - 1 counts the flags in front of step t
    reach = torch.stack([count[i:i + T] == count[W - 1:W - 1 + T] for i in range(W)]).float()[..., None]
    return torch.cat([old, s["x"].float()]), reach, (count[T:T + W - 1] == count[T + W - 1]).float()[..., None]


def _silu(v):
    return v / (1 + torch.exp(-v))


def _dsilu(v):
    p = 1 / (1 + torch.exp(-v))
    return p * (1 + v * (1 - p))


def _plain_conv(s):
    c = s["case"]
    T = c["T"]
    x, reach, left = _history(s)
    v = s["bias"] + sum(reach[i] * x[i:i + T] * s["weight"][:, i] for i in range(c["width"]))
    out = {"y": (_silu(v) if c["act"] == "silu" else v).to(s["y"].dtype)}
    if s["state_in"] is not None:
        out["state"] = (left * x[T:]).transpose(0, 1).to(s["x"].dtype)
    return out


def _plain_conv_step(s):
    c = s["case"]
    old = s["state_in"].float() * (1 - s["done"][0].float())[:, None, None]
    x = torch.cat([old, s["x"][0].float()[:, None]], 1)  # [Be, width, C]
    v = s["bias"] + (x * s["weight"].t()).sum(1)
    s["state_in"].copy_(x[:, 1:])
    return {"y": (_silu(v) if c["act"] == "silu" else v)[None].to(s["y"].dtype), "state": s["state_in"]}


def _plain_conv_bwd(s):
    c = s["case"]
    T, W = c["T"], c["width"]
    x, reach, left = _history(s)
    v = s["bias"] + sum(reach[i] * x[i:i + T] * s["weight"][:, i] for i in range(W))
    g = s["dy"].float() * (_dsilu(v) if c["act"] == "silu" else 1)
    dx = torch.zeros_like(x)
    for i in range(W):
        dx[i:i + T] += reach[i] * g * s["weight"][:, i]
    if s["dstate_out"] is not None:
        dx[T:] += left * s["dstate_out"].float().transpose(0, 1)
    dw = torch.stack([(reach[i] * g * x[i:i + T]).double().sum((0, 1)) for i in range(W)], 1).float()
    out = {"dx": dx[W - 1:].to(s["x"].dtype), "dweight": dw, "dbias": g.double().sum((0, 1)).float()}
    if s["state_in"] is not None:
        out["dstate"] = dx[:W - 1].transpose(0, 1).to(s["x"].dtype)
    return out


def _wide(s, x):
    """[..., groups, N] -> [..., C, N] in 32 bits."""
    return x.float().repeat_interleave(s["case"]["C"] // s["case"]["groups"], -2)


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _linear(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis, by doubling."""
    T, k = a.shape[0], 1
    while k < T:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        if 2 * k < T:
            a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _steps(s):
    """Step sizes; factors of the state of the step before, with the flags in them; what each step adds."""
    d = _softplus(s["dt"].float() + s["dt_bias"])
    a = torch.exp(d[..., None] * s["A"])
    a[1:] *= (1 - s["done"][:-1].float())[..., None, None]
    return d, a, (d * s["x"].float())[..., None] * _wide(s, s["B"])


def _plain_scan(s):
    x, (d, a, b) = s["x"].float(), _steps(s)
    if s["state_in"] is not None:
        b[0] += a[0] * s["state_in"]
    h = _linear(a, b)
    y = (h * _wide(s, s["C"])).sum(-1) + s["D"] * x
    out = {"y": (y if s["z"] is None else y * _silu(s["z"].float())).to(s["y"].dtype)}
    if s["state_in"] is not None:
        out["state"] = h[-1] * (1 - s["done"][-1].float())[:, None, None]
    return out


def _plain_scan_step(s):
    x = s["x"][0].float()
    d = _softplus(s["dt"][0].float() + s["dt_bias"])
    state = s["state_in"] * (1 - s["done"][0].float())[:, None, None]
    state = torch.exp(d[..., None] * s["A"]) * state + (d * x)[..., None] * _wide(s, s["B"][0])
    s["state_in"].copy_(state)
    y = (state * _wide(s, s["C"][0])).sum(-1) + s["D"] * x
    return {"y": (y if s["z"] is None else y * _silu(s["z"][0].float()))[None].to(s["y"].dtype), "state": s["state_in"]}


def _plain_scan_bwd(s):
    c = s["case"]
    x, z, (d, a, b) = s["x"].float(), None if s["z"] is None else s["z"].float(), _steps(s)
    if s["state_in"] is not None:
        b[0] += a[0] * s["state_in"]
    h = _linear(a, b)
    dout = s["dy"].float()
    dy = dout if z is None else dout * _silu(z)
    wc = _wide(s, s["C"])
    g = wc * dy[..., None]
    if s["dstate_out"] is not None:
        g[-1] += s["dstate_out"] * (1 - s["done"][-1].float())[:, None, None]
    g = _linear(torch.cat([a[1:], a[:1]]).flip(0), g.flip(0)).flip(0)
    before = torch.cat([torch.zeros_like(h[:1]) if s["state_in"] is None else s["state_in"][None], h[:-1]])
    q = g * a * before
    gb = (g * _wide(s, s["B"])).sum(-1)
    dd = x * gb + (q * s["A"]).sum(-1)
    raw = dd / (1 + torch.exp(-(s["dt"].float() + s["dt_bias"])))
    fold = lambda t: t.unflatten(2, (c["groups"], -1)).sum(3).to(s["x"].dtype)  # noqa: E731
    out = {"dx": (s["D"] * dy + d * gb).to(s["x"].dtype), "ddt": raw.to(s["x"].dtype),
           "dA": (q * d[..., None]).double().sum((0, 1)).float() if q.numel() < 1 << 26 else
           torch.stack([(qi * di[..., None]).sum(0, dtype=torch.float64) for qi, di in zip(q, d)]).sum(0).float(),
           "dB": fold(g * (d * x)[..., None]), "dC": fold(h * dy[..., None]),
           "dD": (dy * x).double().sum((0, 1)).float(), "ddt_bias": raw.double().sum((0, 1)).float()}
    if z is not None:
        out["dz"] = (dout * ((h * wc).sum(-1) + s["D"] * x) * _dsilu(z)).to(s["x"].dtype)
    if s["state_in"] is not None:
        out["dstate"] = a[0] * g[0]
    return out


def _turns(s):
    """cos and sin of every row's angles, [rows, 1, rot / 2]: the angles in 64 bits."""
    angle = s["pos"].double()[:, None] * s["freq"]
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _pairs(s, x):
    """The first and second elements of the pairs that are turned, and the rest."""
    rot = s["case"]["rot"]
    if s["case"]["interleaved"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _join(s, a, b, rest):
    if s["case"]["interleaved"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _rms(x):
    return 1 / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)


def _plain_heads(s):
    cos, sin = _turns(s)
    out = {}
    for n in "qk":
        x = s[n].float()
        a, b, rest = _pairs(s, x * _rms(x) * s["gamma_" + n])
        out[n] = _join(s, a * cos - b * sin, a * sin + b * cos, rest).to(s[n].dtype)
    return out


def _plain_heads_bwd(s):
    cos, sin = _turns(s)
    out = {}
    for n in "qk":
        a, b, rest = _pairs(s, s["d" + n + "_out"].float())
        dy = _join(s, a * cos + b * sin, b * cos - a * sin, rest)
        x = s[n].float()
        r = _rms(x)
        xhat, g = x * r, dy * s["gamma_" + n]
        out["d" + n] = (r * (g - xhat * ((g * xhat).sum(-1, keepdim=True) / x.shape[-1]))).to(s[n].dtype)
        out["dgamma_" + n] = (dy * xhat).double().sum((0, 1)).float()
    return out


# --------------------------------------------------------------------------------------------------- the library's calls --


def _workspace(s, need):
    """Made by the first pass of a state and kept, as a program keeps it."""
    if "workspace" not in s:
        need = need()
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s["workspace"]


def _own(s):
    from paper_2509_16434_b200 import binding as ppo
    c, kind = s["case"], s["case"]["kind"]
    if kind == "conv":
        ppo.ppo_causal_conv_fwd(s["x"], s["weight"], s["bias"], s["y"], done=s["done"], state_in=s["state_in"], state_out=s["state_out"], act=c["act"])
        return {"y": s["y"]} if s["state_out"] is None else {"y": s["y"], "state": s["state_out"]}
    if kind == "conv_step":
        ppo.ppo_causal_conv_step(s["x"][0], s["weight"], s["bias"], s["state_in"], s["y"][0], start=s["done"][0], act=c["act"])
        return {"y": s["y"], "state": s["state_in"]}
    if kind == "conv_bwd":
        ws = _workspace(s, lambda: ppo.ppo_causal_conv_workspace_bytes(s["x"], c["width"]))
        ppo.ppo_causal_conv_bwd(s["x"], s["weight"], s["bias"], s["dy"], s["dx"], s["dweight"], s["dbias"], done=s["done"], state_in=s["state_in"],
                                dstate_out=s["dstate_out"], dstate_in=s["dstate_in"], act=c["act"], workspace=ws)
        out = {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}
        return out if s["dstate_in"] is None else {**out, "dstate": s["dstate_in"]}
    if kind == "scan":
        ws = _workspace(s, lambda: ppo.ppo_selective_scan_workspace_bytes(s["x"], s["B"], backward=False))
        ppo.ppo_selective_scan_fwd(s["x"], s["dt"], s["A"], s["B"], s["C"], s["y"], D=s["D"], z=s["z"], dt_bias=s["dt_bias"], softplus=True,
                                   done=s["done"], state_in=s["state_in"], state_out=s["state_out"], workspace=ws)
        return {"y": s["y"]} if s["state_out"] is None else {"y": s["y"], "state": s["state_out"]}
    if kind == "scan_step":
        ppo.ppo_selective_scan_step(s["x"][0], s["dt"][0], s["A"], s["B"][0], s["C"][0], s["state_in"], s["y"][0], D=s["D"],
                                    z=None if s["z"] is None else s["z"][0], dt_bias=s["dt_bias"], softplus=True, start=s["done"][0])
        return {"y": s["y"], "state": s["state_in"]}
    if kind == "scan_bwd":
        ws = _workspace(s, lambda: ppo.ppo_selective_scan_workspace_bytes(s["x"], s["B"], backward=True))
        ppo.ppo_selective_scan_bwd(s["x"], s["dt"], s["A"], s["B"], s["C"], s["dy"], s["dx"], s["ddt"], s["dA"], s["dB"], s["dC"], D=s["D"], z=s["z"],
                                   dt_bias=s["dt_bias"], softplus=True, done=s["done"], state_in=s["state_in"], dstate_out=s["dstate_out"], dD=s["dD"],
                                   dz=s["dz"], ddt_bias=s["ddt_bias"], dstate_in=s["dstate_in"], workspace=ws)
        out = {n: s[n] for n in ("dx", "ddt", "dA", "dB", "dC", "dD", "ddt_bias")}
        if s["dz"] is not None:
            out["dz"] = s["dz"]
        return out if s["dstate_in"] is None else {**out, "dstate": s["dstate_in"]}
    if kind == "heads":
        ppo.ppo_qk_norm_rotate_fwd(s["q"], s["k"], s["gamma_q"], s["gamma_k"], s["pos"], s["freq"], s["q_out"], s["k_out"], eps=EPS,
                                   interleaved=c["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"]}
    ws = _workspace(s, lambda: ppo.ppo_qk_norm_rotate_workspace_bytes(s["q"], s["k"]))
    ppo.ppo_qk_norm_rotate_bwd(s["q"], s["k"], s["gamma_q"], s["gamma_k"], s["pos"], s["freq"], s["dq_out"], s["dk_out"], s["dq"], s["dk"],
                               s["dgamma_q"], s["dgamma_k"], eps=EPS, interleaved=c["interleaved"], workspace=ws)
    return {n: s[n] for n in ("dq", "dk", "dgamma_q", "dgamma_k")}


_PLAIN = {"conv": _plain_conv, "conv_bwd": _plain_conv_bwd, "conv_step": _plain_conv_step, "scan": _plain_scan, "scan_bwd": _plain_scan_bwd,
          "scan_step": _plain_scan_step, "heads": _plain_heads, "heads_bwd": _plain_heads_bwd}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# -------------------------------------------------------------------------------------------------------------- work --


def work(case):
    size, kind = _TYPES[case["dtype"]].itemsize, case["kind"]
    if kind in ("heads", "heads_bwd"):
        n = case["rows"] * (case["heads"] + case["kv"]) * case["d"]
        small = 4 * case["rows"] + 4 * case["rot"] + 8 * case["d"]
        return {"bytes": 2 * size * n + small, "flops": 7 * n} if kind == "heads" else {"bytes": 3 * size * n + small + 8 * case["d"], "flops": 16 * n}
    rows, C = case["T"] * case["Be"], case["C"]
    if kind in ("conv", "conv_bwd", "conv_step"):
        W, n = case["width"], rows * C
        states = size * case["Be"] * (W - 1) * C if case["state"] else 0
        if kind == "conv_bwd":
            return {"bytes": 3 * size * n + rows + 3 * states + 8 * (W + 1) * C, "flops": n * (6 * W + 8)}
        return {"bytes": 2 * size * n + rows + 2 * states + 4 * (W + 1) * C, "flops": n * (2 * W + 4)}
    N, G, gate = case["N"], case["groups"], int(case["gate"])
    states, params, n = 4 * case["Be"] * C * N if case["state"] else 0, 4 * C * (N + 2), rows * C
    # x, dt, z, y and B, C; gradients of all of them from dy
    if kind == "scan_bwd":
        return {"bytes": size * (n * (5 + 2 * gate) + 4 * rows * G * N) + rows + 3 * states + 2 * params, "flops": n * (16 * N + 30)}
    return {"bytes": size * (n * (3 + gate) + 2 * rows * G * N) + rows + 2 * states + params, "flops": n * (6 * N + 12)}


# ------------------------------------------------------------------------------------------------------------- 64 bits --


def _alive(s):
    return (s["done"] == 0).double()


def _exact_conv(s):
    """Step by step, with the inputs that a step sees kept in a window that a flag empties; gradients by automatic differentiation."""
    c = s["case"]
    T, Be, C, W = c["T"], c["Be"], c["C"], c["width"]
    bwd, live = c["kind"] == "conv_bwd", _alive(s)
    leaf = lambda t: t.double().requires_grad_(bwd)  # noqa: E731
    x, weight, bias = leaf(s["x"]), leaf(s["weight"]), leaf(s["bias"])
    state = None if s["state_in"] is None else leaf(s["state_in"])
    window = [torch.zeros((Be, C), dtype=torch.float64, device="cuda") if state is None else state[:, i] for i in range(W - 1)]
    if c["kind"] == "conv_step":
        window, live = [w * live[0][:, None] for w in window], torch.ones_like(live)
    taps, out = weight.unbind(1), []
    for t, xt in enumerate(x.unbind(0)):
        window.append(xt)
        v = bias
        for w, tap in zip(window, taps):
            v = torch.addcmul(v, w, tap)
        out.append(v)
        window = [w * live[t][:, None] for w in window[1:]] if c["done"] else window[1:]
    y = torch.stack(out)
    if c["act"] == "silu":
        y = y * torch.sigmoid(y)
    last = torch.stack(window, 1)
    if not bwd:
        return {"y": y, **({} if state is None else {"state": last})}
    total = (y * s["dy"].double()).sum()
    if state is not None:
        total = total + (last * s["dstate_out"].double()).sum()
    grads = torch.autograd.grad(total, [x, weight, bias] + ([] if state is None else [state]))
    return dict(zip(("dx", "dweight", "dbias", "dstate"), grads))


def _exact_scan(s):
    """Step by step, from the recurrence; gradients by automatic differentiation."""
    c = s["case"]
    bwd, live = c["kind"] == "scan_bwd", _alive(s)
    names = [n for n in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias") if s[n] is not None]
    v = {n: s[n].double().requires_grad_(bwd) for n in names}
    h = torch.zeros((c["Be"], c["C"], c["N"]), dtype=torch.float64, device="cuda") if s["state_in"] is None else s["state_in"].double()
    start = h.requires_grad_(bwd)
    if c["kind"] == "scan_step":
        h, live = h * live[0][:, None, None], torch.ones_like(live)
    d = torch.nn.functional.softplus(v["dt"] + v["dt_bias"], threshold=1e6)
    share, per = lambda m: m.repeat_interleave(c["C"] // c["groups"], 1), []  # noqa: E731
    flags = s["done"].any(1).tolist()
    for t, (dt, ut, bt, ct) in enumerate(zip(d.unbind(0), (d * v["x"]).unbind(0), v["B"].unbind(0), v["C"].unbind(0))):
        h = torch.addcmul(torch.exp(dt[..., None] * v["A"]) * h, ut[..., None], share(bt))
        per.append((h * share(ct)).sum(2))
        if flags[t]:
            h = h * live[t][:, None, None]
    y = torch.stack(per) + v["D"] * v["x"]
    if "z" in v:
        y = y * torch.nn.functional.silu(v["z"])
    if not bwd:
        return {"y": y, **({} if s["state_in"] is None else {"state": h})}
    total = (y * s["dy"].double()).sum()
    if s["dstate_out"] is not None:
        total = total + (h * s["dstate_out"].double()).sum()
    grads = torch.autograd.grad(total, [v[n] for n in names] + [start])
    out = {"d" + n: g for n, g in zip(names, grads)}
    return out if s["state_in"] is None else {**out, "dstate": grads[-1]}


def _exact_heads(s):
    """The pairs as complex numbers; gradients by automatic differentiation."""
    c = s["case"]
    bwd, out, rot = c["kind"] == "heads_bwd", {}, c["rot"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), (s["pos"].double()[:, None] * s["freq"])[:, None])
    at = torch.arange(rot, device="cuda")
    at = at.view(-1, 2) if c["interleaved"] else at.view(2, -1).t()
    for n in "qk":
        x, gamma = s[n].double().requires_grad_(bwd), s["gamma_" + n].double().requires_grad_(bwd)
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gamma
        if rot:
            z = torch.complex(y[..., at[:, 0]], y[..., at[:, 1]]) * turn
            whole = torch.empty_like(y[..., :rot])
            whole[..., at[:, 0]], whole[..., at[:, 1]] = z.real, z.imag
            y = torch.cat([whole, y[..., rot:]], -1)
        if bwd:
            out["d" + n], out["dgamma_" + n] = torch.autograd.grad(y, (x, gamma), s["d" + n + "_out"].double())
        else:
            out[n] = y
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_heads if "rows" in case else _exact_conv if "width" in case else _exact_scan)(s)
