"""What is timed of the operators for policies that answer in tokens: linear attention with a decay per head, group
normalisation with an activation, and the clipped policy loss over a vocabulary.

Each operator is here in its plain form (elementary torch operations in 32 bits, angles and long sums in 64) and as the call a
user makes of the library (`own`).  The kinds:

  fwd, bwd, step   decay attention over a sequence minibatch, its gradients, one decision with the state in place
  norm, norm_bwd   group norm with activation, channels last, and its gradients
  loss, logp       clipped token loss with its gradient; log-probabilities and entropies alone
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ACTS = ("none", "relu", "silu")


# ------------------------------------------------------------------------------------------------------------- cases --


def _attn(kind, T, Be, heads, kv, dk, dv, dtype, done=0.0, state=True):
    return {"kind": kind, "T": T, "Be": Be, "heads": heads, "kv": kv, "dk": dk, "dv": dv, "dtype": dtype, "done": done, "state": state}


def _norm(kind, B, HW, C, groups, act, dtype):
    return {"kind": kind, "B": B, "HW": HW, "C": C, "groups": groups, "act": act, "dtype": dtype}


def _loss(kind, rows, vocab, dtype, kl=0.0, ent=0.0, left_out=0.0):
    return {"kind": kind, "rows": rows, "vocab": vocab, "dtype": dtype, "kl": kl, "ent": ent, "left_out": left_out}


def listed():
    named = [
        # one decision of a handful of envs (evaluation, the deployed gripper): latency; 1024 units as 16 heads
        ("step_16", _attn("step", 1, 16, 16, 16, 64, 64, "bf16")),
        # one decision of a simulator GPU's envs, key and value heads shared by four: the states go through once
        ("step_512", _attn("step", 1, 512, 8, 2, 128, 128, "bf16", 0.01)),
        # training minibatch of the recurrent policy's shape: 16 steps of 256 envs with resets, state carried in and out
        ("fwd_rollout", _attn("fwd", 16, 256, 16, 16, 64, 64, "bf16", 0.01)),
        # one long prompt, several documents packed behind one another
        ("fwd_long", _attn("fwd", 8192, 1, 16, 16, 128, 128, "bf16", 0.0005)),
        # gradients in 32 bits, odd sizes everywhere
        ("bwd_odd_f32", _attn("bwd", 119, 37, 6, 2, 48, 80, "f32", 0.01)),
        # gradients of a few long sequences with shared key and value heads
        ("bwd_long", _attn("bwd", 2048, 4, 16, 4, 64, 64, "bf16", 0.001, False)),
        # convolution outputs of a minibatch, 40 x 30 pixels of 64 channels
        ("norm_frames", _norm("norm", 1024, 1200, 64, 8, "relu", "bf16")),
        # their gradients one layer earlier, 80 x 60 pixels of 32 channels
        ("norm_bwd_frames", _norm("norm_bwd", 512, 4800, 32, 4, "relu", "bf16")),
        # the attention's output normalised per head, as it stands behind fwd_rollout, its gradients
        ("norm_bwd_heads", _norm("norm_bwd", 4096, 1, 1024, 16, "silu", "f32")),
        # a policy over a few dozen discrete actions: latency
        ("loss_actions", _loss("loss", 1024, 37, "f32", 0.0, 0.01)),
        # a minibatch of 4096 tokens over a usual vocabulary, padded rows among them
        ("loss_vocab", _loss("loss", 4096, 32000, "bf16", 0.05, 0.01, 0.1)),
        # a few answers scored under the reference policy, large odd vocabulary
        ("logp_few", _loss("logp", 40, 100003, "bf16")),
    ]
    return [dict(case, name=name) for name, case in named]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("step", "fwd", "bwd", "norm", "norm_bwd", "loss", "logp"))
    if kind in ("step", "fwd", "bwd"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        dk, dv = (8 * rng.randint(2, 16) for _ in range(2)) if rng.random() < 0.4 else (rng.choice((64, 128)),) * 2
        kv = rng.choice((1, 2, 4, 8))
        heads = kv * rng.choice((1, 2, 4)) if kv < 8 else kv * rng.choice((1, 2))
        if kind == "step":
            return _attn("step", 1, _log(rng, 1, 4000 // heads), heads, kv, dk, dv, dtype, rng.choice((0.0, 0.02)))
        T = _log(rng, 1, 8192 if kind == "fwd" and dtype == "bf16" else 2048)
        # rows and states of all heads, and the T x T products of the plain form, stay below those of the largest listed cases
        most = min((131072 if dtype == "bf16" else 32768) // T, (1 << 30) // (T * T), 1500) // heads
        return _attn(kind, T, _log(rng, 1, max(1, most)), heads, kv, dk, dv, dtype, rng.choice((0.0, 0.002, 0.02)), rng.random() < 0.7)
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if kind in ("norm", "norm_bwd"):
        groups = rng.choice((1, 2, 3, 4, 8, 16, 32))
        HW = 1 if rng.random() < 0.25 else _log(rng, 2, 19200)
        C = groups * rng.choice((8, 16, 24, 32, 64) if HW < 4 else (2, 4, 6, 8, 16, 24, 32, 64))
        return _norm(kind, max(1, _log(rng, 1, max(1, 64000000 // (HW * C)))), HW, C, groups, rng.choice(_ACTS), dtype)
    vocab = _log(rng, 2, 160000)
    rows = _log(rng, 1, max(1, min(16384, 60000000 // vocab)))
    if kind == "logp":
        return _loss("logp", rows, vocab, dtype)
    return _loss("loss", rows, vocab, dtype, rng.choice((0.0, 0.05)), rng.choice((0.0, 0.01)), rng.choice((0.0, 0.2)))


# ------------------------------------------------------------------------------------------------------------ inputs --


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _TYPES[case["dtype"]]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = {"case": dict(case)}
    if case["kind"] in ("step", "fwd", "bwd"):
        T, Be, heads, kv, dk, dv = (case[n] for n in ("T", "Be", "heads", "kv", "dk", "dv"))
        s.update(q=normal(T, Be, heads, dk), k=normal(T, Be, kv, dk), v=normal(T, Be, kv, dv), scale=dk ** -0.5)
        # memories from some ten to some thousand steps long
        s["decay"] = 1 - torch.exp2(-torch.linspace(3, 11, heads, device="cuda") - uniform(heads))
        # a set flag ends an episode, or a document, at that step; a decision is given the flags of the step before
        s["done"] = (uniform(T, Be) < case["done"]).to(torch.uint8)
        s["state_in"] = normal(Be, heads, dk, dv, dtype=torch.float32) if case["state"] else None
        if case["kind"] == "bwd":
            s["do"] = normal(T, Be, heads, dv)
            s["dstate_out"] = normal(Be, heads, dk, dv, dtype=torch.float32) if case["state"] else None
            s.update(dq=torch.empty_like(s["q"]), dk=torch.empty_like(s["k"]), dv=torch.empty_like(s["v"]))
            s["dstate_in"] = torch.empty_like(s["state_in"]) if case["state"] else None
        else:
            s["o"] = torch.empty((T, Be, heads, dv), dtype=dt, device="cuda")
            s["state_out"] = torch.empty_like(s["state_in"]) if case["state"] else None
    elif case["kind"] in ("norm", "norm_bwd"):
        B, HW, C, groups = (case[n] for n in ("B", "HW", "C", "groups"))
        # channels of unlike level and spread, as convolutions leave them
        s["x"] = (normal(B, HW, C, dtype=torch.float32) * (0.5 + uniform(C)) + normal(C, dtype=torch.float32) + 0.5).to(dt)
        s["gamma"], s["beta"] = 1 + 0.2 * normal(C, dtype=torch.float32), 0.2 * normal(C, dtype=torch.float32)
        s["mean"], s["rstd"] = (torch.empty((B, groups), device="cuda") for _ in range(2))
        s["eps"] = 1e-5
        if case["kind"] == "norm":
            s["y"] = torch.empty_like(s["x"])
        else:
            # what the forward pass left
            xg = s["x"].double().view(B, HW, groups, C // groups)
            mean, var = xg.mean((1, 3)), xg.var((1, 3), unbiased=False)
            s["mean"], s["rstd"] = mean.float(), (var + s["eps"]).rsqrt().float()
            s["dy"] = normal(B, HW, C)
            s["dx"], s["dgamma"], s["dbeta"] = torch.empty_like(s["x"]), torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    else:
        rows, vocab = case["rows"], case["vocab"]
        logits = normal(rows, vocab, dtype=torch.float32) * 3
        if vocab >= 8:  # tokens that are not allowed, and the columns that fill a vocabulary up
            logits = logits.masked_fill(uniform(rows, vocab) < 0.01, -math.inf)
            logits[:, vocab - vocab // 64:] = -math.inf
            logits[:, 0] = 1.0
        s["logits"] = logits.to(dt)
        x = s["logits"].float()
        s["tokens"] = (x - torch.log(-torch.log(uniform(rows, vocab).clamp(1e-20, 0.9999999)))).argmax(1).to(torch.int32)
        logp = x.gather(1, s["tokens"].long()[:, None])[:, 0] - x.logsumexp(1)
        s["logp"], s["entropy"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        if case["kind"] == "loss":
            s["logp_old"] = logp + 0.2 * normal(rows, dtype=torch.float32)
            s["logp_ref"] = logp + 0.3 * normal(rows, dtype=torch.float32) if case["kl"] else None
            s["adv"] = normal(rows, dtype=torch.float32)
            s["weight"] = (uniform(rows) >= case["left_out"]).float() if case["left_out"] else None
            s["B_total"] = rows
            s["clip_low"], s["clip_high"] = 0.2, 0.28
            s["grad_scale"] = 512.0 * rows if case["dtype"] == "f16" else 1.0  # 16-bit floats of the short range have their loss scaled
            # a ratio that 32 bits put on one side of a border and 64 bits on the other has no gradient to compare
            ratio = torch.exp(logp - s["logp_old"])
            near = ((ratio - 0.8).abs() < 1e-4) | ((ratio - 1.28).abs() < 1e-4)
            s["logp_old"] = torch.where(near, s["logp_old"] + 0.001, s["logp_old"])
            s["dlogits"], s["loss"] = torch.empty_like(s["logits"]), torch.empty(5, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------- plain forms --


def _weights(s):
    """decay ** (i - j) where step j reaches step i, [Be, heads, T, T]; the same for the state in (into each step) and for the
    state out (from each step), [Be, heads, T]; and from one to the other, [Be, heads]."""
    c, done = s["case"], s["done"].double()
    T = c["T"]
    lam = s["decay"].double()
    before = torch.cumsum(done, 0) - done  # resets in front of each step
    total = done.sum(0)
    t = torch.arange(T, device="cuda", dtype=torch.float64)
    n = t[:, None] - t[None, :]
    same = (before.t()[:, :, None] == before.t()[:, None, :]) & (n >= 0)
    # step to step: one power per head, masked per env
    w = torch.pow(lam[:, None, None], n.clamp(min=0)[None]).float()[None] * same[:, None].float()
    w_in = (torch.pow(lam[:, None], t + 1)[None] * (before.t() == 0)[:, None]).float()
    w_out = (torch.pow(lam[:, None], T - 1 - t)[None] * (before == total).t()[:, None]).float()
    w_end = (torch.pow(lam, T)[None] * (total == 0)[:, None]).float()
    return w, w_in, w_out, w_end


def _heads(s, x):
    """[T, Be, kv, d] -> [Be, heads, T, d] in 32 bits."""
    return x.float().repeat_interleave(s["case"]["heads"] // x.shape[2], 2).permute(1, 2, 0, 3)


def _rows(x, like):
    """[Be, heads, T, d] -> [T, Be, kv, d] in the type of `like`, heads that share one summed."""
    T, Be, kv, d = like.shape
    return x.permute(2, 0, 1, 3).reshape(T, Be, kv, -1, d).sum(3).to(like.dtype)


def _plain_fwd(s):
    q, k, v = (_heads(s, s[n]) for n in "qkv")
    w, w_in, w_out, w_end = _weights(s)
    q = q * s["scale"]
    o = (q @ k.transpose(2, 3) * w) @ v
    if s["state_in"] is None:
        return {"o": o.permute(2, 0, 1, 3).to(s["o"].dtype)}
    o = o + w_in[..., None] * (q @ s["state_in"])
    state = (k * w_out[..., None]).transpose(2, 3) @ v + w_end[..., None, None] * s["state_in"]
    return {"o": o.permute(2, 0, 1, 3).to(s["o"].dtype), "state": state}


def _plain_step(s):
    q, k, v = (_heads(s, s[n])[:, :, 0] for n in "qkv")
    keep = s["decay"][None, :] * (1 - s["done"][0].float())[:, None]
    state = keep[..., None, None] * s["state_in"] + k[..., :, None] * v[..., None, :]
    s["state_in"].copy_(state)
    o = (q[..., None, :] @ state)[..., 0, :] * s["scale"]
    return {"o": o[None].to(s["o"].dtype), "state": s["state_in"]}


def _plain_bwd(s):
    q, k, v, do = (_heads(s, s[n]) for n in ("q", "k", "v", "do"))
    w, w_in, w_out, w_end = _weights(s)
    do = do * s["scale"]
    a = q @ k.transpose(2, 3) * w
    da = do @ v.transpose(2, 3) * w
    dq, dk, dv = da @ k, da.transpose(2, 3) @ q, a.transpose(2, 3) @ do
    out = {}
    if s["state_in"] is not None:
        dS = s["dstate_out"]
        dq = dq + w_in[..., None] * (do @ s["state_in"].transpose(2, 3))
        dk = dk + w_out[..., None] * (v @ dS.transpose(2, 3))
        dv = dv + w_out[..., None] * (k @ dS)
        out["dstate"] = (q * w_in[..., None]).transpose(2, 3) @ do + w_end[..., None, None] * dS
    return {"dq": dq.permute(2, 0, 1, 3).to(s["q"].dtype), "dk": _rows(dk, s["k"]), "dv": _rows(dv, s["v"]), **out}


def _grouped(s, x):
    c = s["case"]
    return x.float().reshape(c["B"], c["HW"], c["groups"], c["C"] // c["groups"])


def _act(z, act):
    return z.clamp(min=0) if act == "relu" else z / (1 + torch.exp(-z)) if act == "silu" else z


def _dact(z, act):
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _open(s):
    """The values that the ReLU lets through, given the statistics of the forward pass: which side of 0 they are on, in 64 bits."""
    c = s["case"]
    mean, rstd = (s[n].double()[:, None, :, None] for n in ("mean", "rstd"))
    xhat = (s["x"].double().reshape(c["B"], c["HW"], c["groups"], -1) - mean) * rstd
    return xhat.reshape(s["x"].shape) * s["gamma"].double() + s["beta"].double() > 0


def _plain_norm(s):
    c = s["case"]
    x = _grouped(s, s["x"])
    n = x.shape[1] * x.shape[3]
    mean = (x.double().sum((1, 3)) / n).float()
    d = x - mean[:, None, :, None]
    rstd = (d.square().double().sum((1, 3)) / n + s["eps"]).rsqrt().float()
    z = (d * rstd[:, None, :, None]).reshape(s["x"].shape) * s["gamma"] + s["beta"]
    return {"y": _act(z, c["act"]).to(s["y"].dtype), "mean": mean, "rstd": rstd}


def _plain_norm_bwd(s):
    c = s["case"]
    x = _grouped(s, s["x"])
    xhat = (x - s["mean"][:, None, :, None]) * s["rstd"][:, None, :, None]
    flat = xhat.reshape(s["x"].shape)
    dz = s["dy"].float() * (_open(s).float() if c["act"] == "relu" else _dact(flat * s["gamma"] + s["beta"], c["act"]))
    dgamma, dbeta = (dz * flat).double().sum((0, 1)).float(), dz.double().sum((0, 1)).float()
    g = _grouped(s, dz * s["gamma"])
    n = x.shape[1] * x.shape[3]
    m1, m2 = (g.double().sum((1, 3), keepdim=True) / n).float(), ((g * xhat).double().sum((1, 3), keepdim=True) / n).float()
    dx = s["rstd"][:, None, :, None] * (g - m1 - xhat * m2)
    return {"dx": dx.reshape(s["x"].shape).to(s["x"].dtype), "dgamma": dgamma, "dbeta": dbeta}


def _plain_distribution(s):
    x = s["logits"].float()
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    logq = x - top - torch.log(total)  # log-probabilities of all tokens
    p = e / total
    plogq = torch.where(p > 0, p * logq, torch.zeros_like(p))
    return logq, p, plogq, logq.gather(1, s["tokens"].long()[:, None])[:, 0], -plogq.sum(1)


def _plain_logp(s):
    _, _, _, logp, entropy = _plain_distribution(s)
    return {"logp": logp, "entropy": entropy}


def _plain_loss(s):
    c = s["case"]
    _, p, plogq, logp, entropy = _plain_distribution(s)
    w = (s["weight"] if s["weight"] is not None else torch.ones_like(logp)) / s["B_total"]
    ratio = torch.exp(logp - s["logp_old"])
    free, held = ratio * s["adv"], ratio.clamp(1 - s["clip_low"], 1 + s["clip_high"]) * s["adv"]
    g = -torch.where(free <= held, free, torch.zeros_like(free))
    kl = torch.zeros_like(logp)
    if s["logp_ref"] is not None:
        d = s["logp_ref"] - logp
        kl = torch.exp(d) - d - 1
        g = g + c["kl"] * (1 - torch.exp(d))
    clipped = ((ratio < 1 - s["clip_low"]) | (ratio > 1 + s["clip_high"])).float()
    on = w != 0
    grad = -g[:, None] * p
    grad.scatter_add_(1, s["tokens"].long()[:, None], g[:, None])
    grad = w[:, None] * (grad + c["ent"] * (plogq + p * entropy[:, None]))
    terms = torch.stack([-torch.minimum(free, held), kl, entropy, s["logp_old"] - logp, clipped])
    terms = (terms.double() * w).sum(1).float()
    grad = torch.where(on[:, None], grad * s["grad_scale"], torch.zeros_like(grad))
    return {"dlogits": grad.to(s["logits"].dtype), "logp": torch.where(on, logp, torch.zeros_like(logp)),
            "loss": terms}


# --------------------------------------------------------------------------------------------------- the library's calls --


def _workspace(s, need):
    """Made by the first pass of a state and kept, as a program keeps it."""
    if need and s.get("workspace") is None:
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return s.get("workspace")


def _own(s):
    from paper_2509_16434_b200 import binding as ppo
    c, kind = s["case"], s["case"]["kind"]
    if kind == "step":
        ppo.ppo_decay_attention_step(s["q"][0], s["k"][0], s["v"][0], s["decay"], s["state_in"], s["o"][0], start=s["done"][0], scale=s["scale"])
        return {"o": s["o"], "state": s["state_in"]}
    if kind in ("fwd", "bwd"):
        if "workspace" not in s:
            s["workspace"] = _workspace(s, ppo.ppo_decay_attention_workspace_bytes(s["q"], s["k"], s["v"], backward=kind == "bwd"))
        if kind == "fwd":
            ppo.ppo_decay_attention_fwd(s["q"], s["k"], s["v"], s["decay"], s["o"], done=s["done"], state_in=s["state_in"], state_out=s["state_out"],
                                        scale=s["scale"], workspace=s["workspace"])
            return {"o": s["o"], "state": s["state_out"]} if s["state_out"] is not None else {"o": s["o"]}
        ppo.ppo_decay_attention_bwd(s["q"], s["k"], s["v"], s["decay"], s["do"], s["dq"], s["dk"], s["dv"], done=s["done"], state_in=s["state_in"],
                                    dstate_out=s["dstate_out"], dstate_in=s["dstate_in"], scale=s["scale"], workspace=s["workspace"])
        out = {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
        return out if s["dstate_in"] is None else {**out, "dstate": s["dstate_in"]}
    if kind in ("norm", "norm_bwd"):
        if "workspace" not in s:
            s["workspace"] = _workspace(s, ppo.ppo_group_norm_workspace_bytes(s["x"], c["groups"], backward=kind == "norm_bwd"))
        if kind == "norm":
            ppo.ppo_group_norm_fwd(s["x"], c["groups"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], act=c["act"], eps=s["eps"],
                                   workspace=s["workspace"])
            return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        ppo.ppo_group_norm_bwd(s["x"], c["groups"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dy"], s["dx"], s["dgamma"], s["dbeta"],
                               act=c["act"], workspace=s["workspace"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if kind == "logp":
        ppo.ppo_token_logp(s["logits"], s["tokens"], s["logp"], s["entropy"])
        return {"logp": s["logp"], "entropy": s["entropy"]}
    if "workspace" not in s:
        s["workspace"] = _workspace(s, ppo.ppo_token_loss_workspace_bytes(s["logits"]))
    ppo.ppo_token_loss_fwd_bwd(s["logits"], s["tokens"], s["logp_old"], s["adv"], s["B_total"], s["dlogits"], s["loss"], logp_ref=s["logp_ref"],
                               weight=s["weight"], clip_low=s["clip_low"], clip_high=s["clip_high"], kl_coef=c["kl"], ent_coef=c["ent"],
                               grad_scale=s["grad_scale"], logp_out=s["logp"], workspace=s["workspace"])
    return {"dlogits": s["dlogits"], "logp": s["logp"], "loss": s["loss"]}


_PLAIN = {"fwd": _plain_fwd, "bwd": _plain_bwd, "step": _plain_step, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "loss": _plain_loss,
          "logp": _plain_logp}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# -------------------------------------------------------------------------------------------------------------- work --


def work(case):
    size = _TYPES[case["dtype"]].itemsize
    if case["kind"] in ("step", "fwd", "bwd"):
        T, rows, heads, kv, dk, dv = case["T"], case["T"] * case["Be"], case["heads"], case["kv"], case["dk"], case["dv"]
        inputs, states = rows * size * (heads * dk + kv * (dk + dv)), 4 * case["Be"] * heads * dk * dv if case["state"] else 0
        # the recurrence, or for short sequences the products of all pairs of steps
        flops = rows * heads * min(4 * dk * dv, (T + 1) * (dk + dv) + (4 * dk * dv if case["state"] else 0))
        if case["kind"] == "bwd":  # states in, their gradients in and out
            return {"bytes": 2 * inputs + rows * (size * heads * dv + 1) + 3 * states + 4 * heads, "flops": 2.5 * flops}
        return {"bytes": inputs + rows * (size * heads * dv + 1) + 2 * states + 4 * heads, "flops": flops}
    if case["kind"] in ("norm", "norm_bwd"):
        n, stats = case["B"] * case["HW"] * case["C"], 8 * case["B"] * case["groups"]
        if case["kind"] == "norm":
            return {"bytes": 2 * size * n + stats + 8 * case["C"], "flops": 9 * n}
        return {"bytes": 3 * size * n + stats + 16 * case["C"], "flops": 18 * n}
    n, rows = case["rows"] * case["vocab"], case["rows"]
    if case["kind"] == "logp":
        return {"bytes": size * n + 12 * rows, "flops": 5 * n}
    read = n * (1 - case["left_out"])  # rows that are left out are not read; their gradient is written
    return {"bytes": size * (read + n) + (16 + (4 if case["kl"] else 0) + (4 if case["left_out"] else 0)) * rows + 20, "flops": 9 * read}


# ------------------------------------------------------------------------------------------------------------- 64 bits --


def _exact_attention(s):
    """Step by step, from the recurrence."""
    c = s["case"]
    share = c["heads"] // c["kv"]
    q = s["q"].double() * s["scale"]
    k, v = (s[n].double().repeat_interleave(share, 2) for n in "kv")
    lam = s["decay"].double()[None, :, None, None]
    Be, heads, dk, dv = c["Be"], c["heads"], c["dk"], c["dv"]
    zero = torch.zeros((Be, heads, dk, dv), dtype=torch.float64, device="cuda")
    S = zero if s["state_in"] is None else s["state_in"].double()
    live = (s["done"] == 0).double()[..., None, None, None]
    if c["kind"] == "step":
        S = torch.addcmul(lam * live[0] * S, k[0][..., None], v[0][..., None, :])
        return {"o": torch.einsum("bhk,bhkv->bhv", q[0], S)[None], "state": S}
    o = torch.empty((c["T"], Be, heads, dv), dtype=torch.float64, device="cuda")
    dq = torch.empty_like(q)
    do = s["do"].double() if c["kind"] == "bwd" else None
    for t in range(c["T"]):
        S = torch.addcmul(lam * S, k[t][..., None], v[t][..., None, :])
        if do is None:
            o[t] = (q[t][..., None, :] @ S)[..., 0, :]
        else:
            dq[t] = (S @ do[t][..., None])[..., 0]
        S = S * live[t]
    if do is None:
        return {"o": o, **({} if s["state_in"] is None else {"state": S})}
    dk_, dv_ = torch.empty_like(k), torch.empty_like(v)
    dS = zero if s["dstate_out"] is None else s["dstate_out"].double()
    for t in range(c["T"] - 1, -1, -1):
        dS = torch.addcmul(live[t] * dS, q[t][..., None], do[t][..., None, :])
        dk_[t] = (dS @ v[t][..., None])[..., 0]
        dv_[t] = (k[t][..., None, :] @ dS)[..., 0, :]
        dS = lam * dS
    fold = lambda x: x.reshape(c["T"], Be, c["kv"], share, -1).sum(3)  # noqa: E731
    return {"dq": dq * s["scale"], "dk": fold(dk_), "dv": fold(dv_), **({} if s["state_in"] is None else {"dstate": dS})}


def _exact_norm(s):
    """Values and gradients of the definition, the latter by automatic differentiation."""
    c = s["case"]
    x, gamma, beta = (s[n].double().requires_grad_(c["kind"] == "norm_bwd") for n in ("x", "gamma", "beta"))
    per = x.view(c["B"], c["HW"], c["groups"], -1).transpose(1, 2).flatten(2)
    mean, var = per.mean(2), per.var(2, unbiased=False)
    rstd = 1 / torch.sqrt(var + s["eps"])
    per = (per - mean[..., None]) * rstd[..., None]
    z = per.view(c["B"], c["groups"], c["HW"], -1).transpose(1, 2).reshape(x.shape) * gamma + beta
    if c["act"] == "relu" and c["kind"] == "norm_bwd":  # the gate goes by the statistics that were handed over
        saved = [s[n].double().repeat_interleave(c["C"] // c["groups"], 1)[:, None] for n in ("mean", "rstd")]
        y = z * torch.addcmul(beta, (x - saved[0]) * saved[1], gamma).detach().gt(0)
    else:
        y = z.relu() if c["act"] == "relu" else z * z.sigmoid() if c["act"] == "silu" else z
    if c["kind"] == "norm":
        return {"y": y, "mean": mean, "rstd": rstd}
    dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def _exact_loss(s):
    c = s["case"]
    x = s["logits"].double()
    lse = x.logsumexp(1)
    logp = x.gather(1, s["tokens"].long()[:, None])[:, 0] - lse
    prob = torch.exp(x - lse[:, None])
    entropy = lse - (prob * x.clamp(min=-1e30)).sum(1)
    if c["kind"] == "logp":
        return {"logp": logp, "entropy": entropy}
    # each term as a function of the log-probability and the entropy of its row
    lp, en = logp.clone().requires_grad_(), entropy.clone().requires_grad_()
    w = (torch.ones_like(logp) if s["weight"] is None else s["weight"].double()) / s["B_total"]
    ratio, adv = torch.exp(lp - s["logp_old"].double()), s["adv"].double()
    bounded = ratio.clamp(1 - s["clip_low"], 1 + s["clip_high"])
    policy = -torch.minimum(ratio * adv, bounded * adv)
    kl = torch.zeros_like(lp)
    if s["logp_ref"] is not None:
        d = s["logp_ref"].double() - lp
        kl = torch.expm1(d) - d
    total = (w * (policy + c["kl"] * kl - c["ent"] * en)).sum()
    g_lp, g_en = torch.autograd.grad(total, (lp, en))
    # d logp / d x_j = [j = token] - p_j,  d H / d x_j = -p_j (log p_j + H)
    grad = -prob * (g_lp[:, None] + g_en[:, None] * ((x - lse[:, None]).clamp(min=-1e30) + entropy[:, None]))
    grad.scatter_add_(1, s["tokens"].long()[:, None], g_lp[:, None])
    outside = (ratio < 1 - s["clip_low"]) | (ratio > 1 + s["clip_high"])
    loss = torch.stack([(w * t).sum() for t in (policy, kl, en, s["logp_old"].double() - lp, outside.double())])
    return {"dlogits": grad * s["grad_scale"], "logp": torch.where(w != 0, logp, 0.0), "loss": loss.detach()}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm_bwd") and case["B"] * case["HW"] * case["C"] > 1 << 28:
        return None
    return _exact_attention(s) if kind in ("step", "fwd", "bwd") else _exact_norm(s) if kind in ("norm", "norm_bwd") else _exact_loss(s)
