"""A policy in tokens whose memory is a layer of causal convolution and selective scan and a layer of decay attention over normed, rotated queries and
keys: projection -> convolution -> projections of step sizes, B, C -> gated scan -> projection -> norms with rotation -> decay attention ->
vocabulary -> clipped loss, and all gradients back to the weights, against automatic differentiation in 64 bits; decisions one by one against
the sequence.

In 32 bits every stage is within some 3e-6 (2-norm) of its own formula (their own tests); nine stages in a row, none of which has a
condition above 10 on these inputs (convolutions and projections of random matrices, states that remember some tens of steps,
normalisation of heads that vary by about 1), stay below 9 x 10 x 3e-6 = 2.7e-4."""
import pytest
import torch

from paper_2509_16434_b200 import binding as ppo
from helpers import rel_l2

pytestmark = pytest.mark.gpu
DEV = "cuda"
BOUND = 2.7e-4

T, Be, D, C, W, N, G, HEADS, KV, DK, DV, V = 40, 6, 24, 32, 4, 8, 2, 4, 2, 16, 12, 50
PAIRS, ENT = 4, 0.02


def _problem():
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    p = dict(x=n(T, Be, D), w_in=n(D, 2 * C) / D ** 0.5, conv_w=n(C, W) / 2, conv_b=0.2 * n(C), w_dt=n(C, C) / C ** 0.5, w_bc=n(C, 2 * G * N) / C ** 0.5,
             A=-torch.exp(0.5 * n(C, N)), Dskip=n(C), dt_bias=n(C) - 2, w_qkv=n(C, HEADS * DK + KV * (DK + DV)) / C ** 0.5, gq=1 + 0.2 * n(DK), gk=1 + 0.2 * n(DK),
             w_out=n(HEADS * DV, V) * 0.2, conv_s=n(Be, W - 1, C), scan_s=n(Be, C, N), attn_s=n(Be, HEADS, DK, DV))
    p["lam"] = torch.tensor([0.5, 0.8, 0.95, 0.99], device=DEV)
    p["done"] = (torch.rand(T, Be, generator=g, device=DEV) < 0.05).to(torch.uint8)
    # positions count up from the start of each episode
    pos, at = torch.zeros(T, Be, dtype=torch.int32, device=DEV), torch.full((Be,), 3, dtype=torch.int32, device=DEV)
    for t in range(T):
        pos[t] = at
        at = torch.where(p["done"][t] == 0, at + 1, torch.zeros_like(at))
    p["pos"], p["freq"] = pos, 100.0 ** (-torch.arange(PAIRS, device=DEV, dtype=torch.float64) / PAIRS)
    p["tokens"], p["adv"], p["noise"] = torch.randint(0, V, (T * Be,), generator=g, device=DEV, dtype=torch.int32), n(T * Be), n(T * Be)
    return p


LEAVES = ("x", "w_in", "conv_w", "conv_b", "w_dt", "w_bc", "A", "Dskip", "dt_bias", "w_qkv", "gq", "gk", "w_out", "conv_s", "scan_s", "attn_s")


def _ws(n):
    return torch.empty(n, dtype=torch.uint8, device=DEV) if n else None


def _qkv(rows):
    q, k, v = rows.split([HEADS * DK, KV * DK, KV * DV], -1)
    return q.unflatten(-1, (HEADS, DK)), k.unflatten(-1, (KV, DK)), v.unflatten(-1, (KV, DV))


def _bc(rows):
    b, c = rows.split([G * N, G * N], -1)
    return b.unflatten(-1, (G, N)), c.unflatten(-1, (G, N))


def _forward(p):
    s = {"rows": p["x"] @ p["w_in"]}
    s["u"], s["z"] = s["rows"].split([C, C], -1)  # parts of wider rows, as they are
    e = lambda *sh: torch.full(sh, float("nan"), device=DEV)  # noqa: E731
    s["h"], s["conv_s"] = e(T, Be, C), e(Be, W - 1, C)
    ppo.ppo_causal_conv_fwd(s["u"], p["conv_w"], p["conv_b"], s["h"], p["done"], p["conv_s"], s["conv_s"], "silu")
    s["dt"], s["bc"] = s["h"] @ p["w_dt"], s["h"] @ p["w_bc"]
    B, Cm = _bc(s["bc"])
    s["y"], s["scan_s"] = e(T, Be, C), e(Be, C, N)
    ppo.ppo_selective_scan_fwd(s["h"], s["dt"], p["A"], B, Cm, s["y"], p["Dskip"], s["z"], p["dt_bias"], True, p["done"], p["scan_s"], s["scan_s"],
                               _ws(ppo.ppo_selective_scan_workspace_bytes(s["h"], B, False)))
    s["qkv"] = s["y"] @ p["w_qkv"]
    q, k, v = _qkv(s["qkv"])
    s["q"], s["k"] = e(T * Be, HEADS, DK), e(T * Be, KV, DK)
    ppo.ppo_qk_norm_rotate_fwd(q.flatten(0, 1), k.flatten(0, 1), p["gq"], p["gk"], p["pos"].flatten(), p["freq"], s["q"], s["k"])
    s["o"], s["attn_s"] = e(T, Be, HEADS, DV), e(Be, HEADS, DK, DV)
    ppo.ppo_decay_attention_fwd(s["q"].view(T, Be, HEADS, DK), s["k"].view(T, Be, KV, DK), v, p["lam"], s["o"], p["done"], p["attn_s"], s["attn_s"], 0.25)
    s["logits"] = s["o"].view(T * Be, -1) @ p["w_out"]
    return s


def _reference(leaves, p):
    live = (1 - p["done"].double())[..., None]
    rows = leaves["x"] @ leaves["w_in"]
    u, z = rows.split([C, C], -1)
    window, h = list(leaves["conv_s"].unbind(1)), []
    for t in range(T):
        window = window + [u[t]]
        a = leaves["conv_b"] + sum(w * leaves["conv_w"][:, i] for i, w in enumerate(window))
        h.append(a * torch.sigmoid(a))
        window = [w * live[t] for w in window[1:]]
    h = torch.stack(h)
    d = torch.nn.functional.softplus(h @ leaves["w_dt"] + leaves["dt_bias"])
    B, Cm = (m.repeat_interleave(C // G, 2) for m in _bc(h @ leaves["w_bc"]))
    S, y = leaves["scan_s"], []
    for t in range(T):
        S = torch.exp(d[t][..., None] * leaves["A"]) * S + (d[t] * h[t])[..., None] * B[t]
        y.append((S * Cm[t]).sum(-1) + leaves["Dskip"] * h[t])
        S = S * live[t][..., None]
    y = torch.stack(y) * z * torch.sigmoid(z)
    q, k, v = _qkv(y @ leaves["w_qkv"])
    angle = (p["pos"].double()[..., None] * p["freq"])[:, :, None]

    def turned(m, gamma):
        m = m / torch.sqrt((m * m).mean(-1, keepdim=True) + 1e-6) * gamma
        a, b, rest = m[..., :PAIRS], m[..., PAIRS:2 * PAIRS], m[..., 2 * PAIRS:]
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos(), rest], -1)
    q, k = turned(q, leaves["gq"]), turned(k, leaves["gk"])
    M, o = leaves["attn_s"], []
    for t in range(T):
        M = p["lam"].double()[None, :, None, None] * M + k[t].repeat_interleave(HEADS // KV, 1)[..., None] * v[t].repeat_interleave(HEADS // KV, 1)[..., None, :]
        o.append((q[t][..., None, :] @ M)[..., 0, :] * 0.25)
        M = M * live[t][..., None, None]
    return torch.stack(o).reshape(T * Be, -1) @ leaves["w_out"], torch.stack(window, 1), S, M


def test_forward_and_backward():
    p = _problem()
    s = _forward(p)
    old = torch.empty(T * Be, device=DEV)
    ppo.ppo_token_logp(s["logits"], p["tokens"], old)
    old = old + 0.05 * p["noise"]
    dlogits, loss = torch.empty_like(s["logits"]), torch.empty(5, device=DEV)
    ppo.ppo_token_loss_fwd_bwd(s["logits"], p["tokens"], old, p["adv"], T * Be, dlogits, loss, ent_coef=ENT, workspace=_ws(ppo.ppo_token_loss_workspace_bytes(s["logits"])))
    got = {"w_out": s["o"].view(T * Be, -1).t() @ dlogits}
    do = (dlogits @ p["w_out"].t()).view(T, Be, HEADS, DV)
    dqkv = torch.empty_like(s["qkv"])
    (q, k, v), (dq, dk, dv) = _qkv(s["qkv"]), _qkv(dqkv)
    gq, gk = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    Q, K = s["q"].view(T, Be, HEADS, DK), s["k"].view(T, Be, KV, DK)
    got["attn_s"] = torch.empty_like(p["attn_s"])
    # the attention's gradients lie as its operands do: v's in its row of dqkv
    ppo.ppo_decay_attention_bwd(Q, K, v, p["lam"], do, gq.view(T, Be, HEADS, DK), gk.view(T, Be, KV, DK), dv, p["done"], p["attn_s"], None, got["attn_s"], 0.25,
                                _ws(ppo.ppo_decay_attention_workspace_bytes(Q, K, v, True)))
    got["gq"], got["gk"] = torch.empty_like(p["gq"]), torch.empty_like(p["gk"])
    ppo.ppo_qk_norm_rotate_bwd(q.flatten(0, 1), k.flatten(0, 1), p["gq"], p["gk"], p["pos"].flatten(), p["freq"], gq, gk, dq.flatten(0, 1), dk.flatten(0, 1),
                               got["gq"], got["gk"], workspace=_ws(ppo.ppo_qk_norm_rotate_workspace_bytes(q.flatten(0, 1), k.flatten(0, 1))))
    got["w_qkv"] = s["y"].flatten(0, 1).t() @ dqkv.flatten(0, 1)
    dy = dqkv @ p["w_qkv"].t()
    drows, dh, ddt, dbc = torch.empty_like(s["rows"]), torch.empty_like(s["h"]), torch.empty_like(s["dt"]), torch.empty_like(s["bc"])
    (B, Cm), (dB, dC), (du, dz) = _bc(s["bc"]), _bc(dbc), drows.split([C, C], -1)
    for name, src in (("A", "A"), ("Dskip", "Dskip"), ("dt_bias", "dt_bias"), ("scan_s", "scan_s"), ("conv_w", "conv_w"), ("conv_b", "conv_b"), ("conv_s", "conv_s")):
        got[name] = torch.full_like(p[src], float("nan"))
    ppo.ppo_selective_scan_bwd(s["h"], s["dt"], p["A"], B, Cm, dy, dh, ddt, got["A"], dB, dC, p["Dskip"], s["z"], p["dt_bias"], True, p["done"], p["scan_s"], None,
                               got["Dskip"], dz, got["dt_bias"], got["scan_s"], workspace=_ws(ppo.ppo_selective_scan_workspace_bytes(s["h"], B, True)))
    got["w_dt"], got["w_bc"] = s["h"].flatten(0, 1).t() @ ddt.flatten(0, 1), s["h"].flatten(0, 1).t() @ dbc.flatten(0, 1)
    dh = dh + ddt @ p["w_dt"].t() + dbc @ p["w_bc"].t()
    ppo.ppo_causal_conv_bwd(s["u"], p["conv_w"], p["conv_b"], dh, du, got["conv_w"], got["conv_b"], p["done"], p["conv_s"], None, got["conv_s"], "silu",
                            workspace=_ws(ppo.ppo_causal_conv_workspace_bytes(s["u"], W)))
    got["w_in"], got["x"] = p["x"].flatten(0, 1).t() @ drows.flatten(0, 1), drows @ p["w_in"].t()

    leaves = {n: p[n].double().requires_grad_() for n in LEAVES}
    logits, conv_s, scan_s, attn_s = _reference(leaves, p)
    lq = torch.log_softmax(logits, 1)
    lp = lq.gather(1, p["tokens"].long()[:, None])[:, 0]
    r = torch.exp(lp - old.double())
    assert float(torch.minimum((r - 0.8).abs(), (r - 1.2).abs()).min().detach()) > 1e-5
    policy = -torch.minimum(r * p["adv"], r.clamp(0.8, 1.2) * p["adv"]).mean()
    entropy = -(lq.exp() * lq).sum(1).mean()
    want = dict(zip(LEAVES, torch.autograd.grad(policy - ENT * entropy, list(leaves.values()))))
    for n, grad in want.items():
        assert rel_l2(got[n].cpu(), grad.cpu()) <= BOUND, n
    for n, v in (("logits", logits), ("conv_s", conv_s), ("scan_s", scan_s), ("attn_s", attn_s)):
        assert rel_l2(s[n].cpu(), v.detach().cpu()) <= BOUND, n
    assert ppo.ppo_poll_status() == 0


def test_decisions_one_by_one_give_the_logits_of_the_sequence():
    p = _problem()
    s = _forward(p)
    conv, scan, attn, start = p["conv_s"].clone(), p["scan_s"].clone(), p["attn_s"].clone(), None
    for t in range(T):
        u, z = (p["x"][t] @ p["w_in"]).split([C, C], -1)
        h, y = torch.empty(Be, C, device=DEV), torch.empty(Be, C, device=DEV)
        ppo.ppo_causal_conv_step(u, p["conv_w"], p["conv_b"], conv, h, start, "silu")
        B, Cm = _bc(h @ p["w_bc"])
        ppo.ppo_selective_scan_step(h, h @ p["w_dt"], p["A"], B, Cm, scan, y, p["Dskip"], z, p["dt_bias"], True, start)
        q, k, v = _qkv(y @ p["w_qkv"])
        qo, ko, o = torch.empty(Be, HEADS, DK, device=DEV), torch.empty(Be, KV, DK, device=DEV), torch.empty(Be, HEADS, DV, device=DEV)
        ppo.ppo_qk_norm_rotate_fwd(q, k, p["gq"], p["gk"], p["pos"][t], p["freq"], qo, ko)
        ppo.ppo_decay_attention_step(qo, ko, v, p["lam"], attn, o, start, 0.25)
        start = p["done"][t]
        assert rel_l2((o.flatten(1) @ p["w_out"]).cpu(), s["logits"].view(T, Be, V)[t].cpu()) <= BOUND, t
    live = start == 0
    for got, n in ((conv, "conv_s"), (scan, "scan_s"), (attn, "attn_s")):
        assert rel_l2(got[live].cpu(), s[n][live].cpu()) <= BOUND, n
