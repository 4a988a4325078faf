"""A policy in tokens from end to end: projection -> decay attention -> group norm per head with SiLU -> vocabulary -> clipped loss, and
all gradients back to the weights, against automatic differentiation in 64 bits; decisions one by one against the sequence.

In 32 bits every stage is within some 2e-6 (2-norm) of its own formula (their own tests); eight stages in a row, none of which has
a condition above 10 on these inputs (normalisation of heads that vary by about 1, a softmax over 50 tokens), stay below
8 x 10 x 2e-6 = 1.6e-4."""
import pytest
import torch

from paper_2509_16434_b200 import binding as ppo
from helpers import rel_l2

pytestmark = pytest.mark.gpu
DEV = "cuda"
BOUND = 1.6e-4

T, Be, D, HEADS, KV, DK, DV, V = 40, 6, 48, 4, 2, 16, 24, 50
CLIP, KL, ENT = 0.2, 0.1, 0.02


def _problem():
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    width = HEADS * DK + KV * (DK + DV)
    return dict(x=n(T, Be, D), w_in=n(D, width) / D ** 0.5, gamma=1 + 0.2 * n(HEADS * DV), beta=0.2 * n(HEADS * DV), w_out=n(HEADS * DV, V) * 0.2,
                lam=torch.tensor([0.5, 0.8, 0.95, 0.99], device=DEV), done=(torch.rand(T, Be, generator=g, device=DEV) < 0.05).to(torch.uint8),
                s0=n(Be, HEADS, DK, DV), tokens=torch.randint(0, V, (T * Be,), generator=g, device=DEV, dtype=torch.int32), adv=n(T * Be),
                noise=n(2, T * Be), weight=(torch.rand(T * Be, generator=g, device=DEV) > 0.1).float())


def _split(rows):
    q, k, v = rows.split([HEADS * DK, KV * DK, KV * DV], -1)
    return q.unflatten(-1, (HEADS, DK)), k.unflatten(-1, (KV, DK)), v.unflatten(-1, (KV, DV))


def _logits(p):
    rows = p["x"] @ p["w_in"]
    q, k, v = _split(rows)
    o = torch.empty((T, Be, HEADS, DV), device=DEV)
    state = torch.empty_like(p["s0"])
    ppo.ppo_decay_attention_fwd(q, k, v, p["lam"], o, p["done"], p["s0"], state, DK ** -0.5)
    y, mean, rstd = torch.empty((T * Be, 1, HEADS * DV), device=DEV), torch.empty((T * Be, HEADS), device=DEV), torch.empty((T * Be, HEADS), device=DEV)
    ppo.ppo_group_norm_fwd(o.view(T * Be, 1, HEADS * DV), HEADS, p["gamma"], p["beta"], y, mean, rstd, act="silu")
    return rows, o, state, y, mean, rstd, y[:, 0] @ p["w_out"]


def test_a_policy_in_tokens_forward_and_backward():
    p = _problem()
    rows, o, state, y, mean, rstd, logits = _logits(p)
    logp = torch.empty(T * Be, device=DEV)
    ppo.ppo_token_logp(logits, p["tokens"], logp)
    old, ref = logp + 0.2 * p["noise"][0], logp + 0.2 * p["noise"][1]
    dlogits, loss = torch.empty_like(logits), torch.empty(5, device=DEV)
    ws = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV) if n else None  # noqa: E731
    ppo.ppo_token_loss_fwd_bwd(logits, p["tokens"], old, p["adv"], T * Be, dlogits, loss, ref, p["weight"], CLIP, CLIP, KL, ENT,
                               workspace=ws(ppo.ppo_token_loss_workspace_bytes(logits)))
    got = {"w_out": y[:, 0].t() @ dlogits}
    dy = (dlogits @ p["w_out"].t()).view(T * Be, 1, -1)
    do, got["gamma"], got["beta"] = torch.empty_like(y), torch.empty_like(p["gamma"]), torch.empty_like(p["beta"])
    x = o.view(T * Be, 1, -1)
    ppo.ppo_group_norm_bwd(x, HEADS, p["gamma"], p["beta"], mean, rstd, dy, do, got["gamma"], got["beta"], "silu",
                           workspace=ws(ppo.ppo_group_norm_workspace_bytes(x, HEADS, True)))
    drows = torch.empty_like(rows)
    q, k, v = _split(rows)
    got["s0"] = torch.empty_like(p["s0"])
    ppo.ppo_decay_attention_bwd(q, k, v, p["lam"], do.view(T, Be, HEADS, DV), *_split(drows), p["done"], p["s0"], None, got["s0"], DK ** -0.5,
                                ws(ppo.ppo_decay_attention_workspace_bytes(q, k, v, True)))
    got["w_in"] = p["x"].flatten(0, 1).t() @ drows.flatten(0, 1)
    got["x"] = drows @ p["w_in"].t()

    leaves = {n: p[n].double().requires_grad_() for n in ("x", "w_in", "gamma", "beta", "w_out", "s0")}
    q, k, v = _split(leaves["x"] @ leaves["w_in"])
    S, lam, out = leaves["s0"], p["lam"].double()[None, :, None, None], []
    for t in range(T):
        S = lam * S + k[t].repeat_interleave(HEADS // KV, 1)[..., None] * v[t].repeat_interleave(HEADS // KV, 1)[..., None, :]
        out.append((q[t][..., None, :] @ S)[..., 0, :] * DK ** -0.5)
        S = S * (1 - p["done"][t].double())[:, None, None, None]
    z = torch.stack(out).reshape(T * Be, HEADS, DV)
    z = (z - z.mean(2, keepdim=True)) / torch.sqrt(z.var(2, unbiased=False, keepdim=True) + 1e-5)
    z = z.flatten(1) * leaves["gamma"] + leaves["beta"]
    lq = torch.log_softmax((z * torch.sigmoid(z)) @ leaves["w_out"], 1)
    lp = lq.gather(1, p["tokens"].long()[:, None])[:, 0]
    r, d, w = torch.exp(lp - old.double()), ref.double() - lp, p["weight"].double()
    assert float(torch.minimum((r - 1 + CLIP).abs(), (r - 1 - CLIP).abs()).min()) > 1e-5
    s = torch.minimum(r * p["adv"], r.clamp(1 - CLIP, 1 + CLIP) * p["adv"])
    parts = [-s, torch.exp(d) - d - 1, -(lq.exp() * lq).sum(1), old.double() - lp, ((r < 1 - CLIP) | (r > 1 + CLIP)).double()]
    means = torch.stack([(w * t).sum() / (T * Be) for t in parts])
    want = dict(zip(leaves, torch.autograd.grad(means[0] + KL * means[1] - ENT * means[2], list(leaves.values()))))
    for n, grad in want.items():
        assert rel_l2(got[n].cpu(), grad.cpu()) <= BOUND, n
    assert rel_l2(loss.cpu(), means.detach().cpu()) <= BOUND and rel_l2(state.cpu(), S.detach().cpu()) <= BOUND
    assert rel_l2(logp.cpu(), lp.detach().cpu()) <= BOUND


def test_decisions_one_by_one_score_as_the_sequence_does():
    p = _problem()
    *_, state, _, _, _, logits = _logits(p)
    want, H = torch.empty(T * Be, device=DEV), torch.empty(T * Be, device=DEV)
    ppo.ppo_token_logp(logits, p["tokens"], want, H)
    S, start, got = p["s0"].clone(), None, []
    for t in range(T):
        q, k, v = _split(p["x"][t] @ p["w_in"])
        o, y = torch.empty((Be, HEADS, DV), device=DEV), torch.empty((Be, 1, HEADS * DV), device=DEV)
        ppo.ppo_decay_attention_step(q, k, v, p["lam"], S, o, start, DK ** -0.5)
        start = p["done"][t]
        mean, rstd, lp = torch.empty((Be, HEADS), device=DEV), torch.empty((Be, HEADS), device=DEV), torch.empty(Be, device=DEV)
        ppo.ppo_group_norm_fwd(o.view(Be, 1, -1), HEADS, p["gamma"], p["beta"], y, mean, rstd, act="silu")
        ppo.ppo_token_logp(y[:, 0] @ p["w_out"], p["tokens"].view(T, Be)[t].contiguous(), lp)
        got.append(lp)
    assert rel_l2(torch.cat(got).cpu(), want.cpu()) <= BOUND
    live = ~start.bool()
    assert rel_l2(S[live].cpu(), state[live].cpu()) <= BOUND
