"""Plain forms in 64 bits of the operators for policies in tokens, with what their rounding errors are measured by.

Each `*_abs` result is the same sum with every term replaced by its absolute value: a sum of n roundings of unit u is off by at
most n u times it, whatever cancels."""
import torch


def attention(q, k, v, lam, done, s0, scale, do=None, ds=None):
    """The recurrence, step by step, of [T,Be,heads,d] operands.  With do: the gradients instead."""
    T, Be, heads, dk = q.shape
    share = heads // k.shape[2]
    q, k, v, lam = q.double() * scale, k.double().repeat_interleave(share, 2), v.double().repeat_interleave(share, 2), lam.double()[None, :, None, None]
    live = torch.ones(T, Be, dtype=torch.float64, device=q.device) if done is None else (done == 0).double()
    live = live[..., None, None, None]
    zero = torch.zeros(Be, heads, dk, v.shape[3], dtype=torch.float64, device=q.device)
    S, out = zero if s0 is None else s0.double(), []
    for t in range(T):
        S = lam * S + k[t][..., :, None] * v[t][..., None, :]
        out.append(torch.einsum("bhk,bhkv->bhv", q[t], S) if do is None else torch.einsum("bhkv,bhv->bhk", S, do[t].double()) * scale)
        S = S * live[t]
    if do is None:
        return torch.stack(out), S
    dS, dk_, dv_ = zero if ds is None else ds.double(), [], []
    for t in reversed(range(T)):
        dS = live[t] * dS + q[t][..., :, None] * do[t].double()[..., None, :]
        dk_.append(torch.einsum("bhkv,bhv->bhk", dS, v[t]))
        dv_.append(torch.einsum("bhkv,bhk->bhv", dS, k[t]))
        dS = lam * dS
    fold = lambda x: torch.stack(x[::-1]).reshape(T, Be, heads // share, share, -1).sum(3)  # noqa: E731
    return torch.stack(out), fold(dk_), fold(dv_), dS


def attention_abs(q, k, v, lam, done, s0, scale, do=None, ds=None):
    a = lambda x: None if x is None else x.double().abs()  # noqa: E731
    return attention(a(q), a(k), a(v), lam, done, a(s0), abs(scale), a(do), a(ds))


def group_norm(x, groups, gamma, beta, act, eps):
    B, HW, C = x.shape
    g = x.double().reshape(B, HW, groups, C // groups)
    mean, var = g.mean((1, 3)), g.var((1, 3), unbiased=False)
    rstd = 1 / torch.sqrt(var + eps)
    xhat = ((g - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(B, HW, C)
    z = xhat if gamma is None else xhat * gamma.double() + beta.double()
    return {"none": z, "relu": z.clamp(min=0), "silu": z * torch.sigmoid(z)}[act], mean, rstd


def group_norm_grad(x, groups, gamma, beta, mean, rstd, dy, act):
    """dx, dgamma, dbeta by the formulas, from the statistics handed over; then what the errors of each are measured by."""
    B, HW, C = x.shape
    per = C // groups
    wide = lambda s: s.double().repeat_interleave(per, 1)[:, None]  # noqa: E731
    one = torch.ones(C, dtype=torch.float64, device=x.device)
    gamma, beta = (one, 0 * one) if gamma is None else (gamma.double(), beta.double())
    xhat = (x.double() - wide(mean)) * wide(rstd)
    z = xhat * gamma + beta
    sig = torch.sigmoid(z)
    dz = dy.double() * {"none": torch.ones_like(z), "relu": (z > 0).double(), "silu": sig * (1 + z * (1 - sig))}[act]
    g = dz * gamma
    over = lambda t: t.reshape(B, HW, groups, per).mean((1, 3)).repeat_interleave(per, 1)[:, None]  # noqa: E731
    dx = wide(rstd) * (g - over(g) - xhat * over(g * xhat))
    size = wide(rstd) * (g.abs() + over(g.abs()) + xhat.abs() * over((g * xhat).abs()))
    return dx, (dz * xhat).sum((0, 1)), dz.sum((0, 1)), size, (dz * xhat).abs().sum((0, 1)), dz.abs().sum((0, 1))


def token_rows(logits, tokens, scale):
    """logp, entropy, log-probabilities of all tokens; rows without a finite logit: minus infinity and 0."""
    x = logits.double() * scale
    top = x.amax(1, keepdim=True)
    empty = torch.isinf(top[:, 0]) & (top[:, 0] < 0)
    d = torch.where(empty[:, None], torch.zeros_like(x), x - top)
    logq = d - torch.log(torch.exp(d).sum(1, keepdim=True))
    p = torch.exp(logq)
    H = -torch.where(p > 0, p * logq, torch.zeros_like(p)).sum(1)
    inside = (tokens >= 0) & (tokens < logits.shape[1])
    logp = logq.gather(1, torch.where(inside, tokens, torch.zeros_like(tokens)).long()[:, None])[:, 0]
    logp = torch.where(inside, torch.where(empty, torch.full_like(logp, float("-inf")), logp), torch.zeros_like(logp))
    H = torch.where(inside & ~empty, H, torch.zeros_like(H))
    return logp, H, logq, inside & ~empty


def token_loss(logits, tokens, old, adv, B_total, ref=None, weight=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, ent_coef=0.0, scale=1.0):
    """dL/dlogits, logp (0 where left out), the five sums; then, element by element, the absolute size of the gradient's terms."""
    rows, vocab = logits.shape
    w = torch.ones(rows, dtype=torch.float64, device=logits.device) if weight is None else weight.double()
    # rows that are left out may hold anything
    logits = torch.where((w != 0)[:, None] & ((tokens >= 0) & (tokens < vocab))[:, None], logits, torch.zeros_like(logits))
    logp, H, logq, on = token_rows(logits, tokens, scale)
    on = on & (w != 0)
    logp, old, adv = torch.where(on, logp, torch.zeros_like(logp)), old.double(), adv.double()
    r = torch.exp(logp - old)
    free, held = r * adv, r.clamp(1 - clip_low, 1 + clip_high) * adv
    dl = torch.where(free <= held, -free, torch.zeros_like(free))
    size = dl.abs()
    kl = torch.zeros_like(logp)
    if ref is not None:
        d = ref.double() - logp
        kl = torch.exp(d) - d - 1
        dl = dl + kl_coef * (1 - torch.exp(d))
        size = size + abs(kl_coef) * (1 + torch.exp(d))
    share = torch.where(on, w / B_total, torch.zeros_like(w))
    p = torch.exp(logq)
    ent = torch.where(p > 0, p * (logq + H[:, None]), torch.zeros_like(p))
    hot = torch.zeros_like(p).scatter_(1, tokens.clamp(0, vocab - 1).long()[:, None], 1.0)
    grad = share[:, None] * scale * (dl[:, None] * (hot - p) + ent_coef * ent)
    bound = (share * scale)[:, None].abs() * (size[:, None] * (hot + p) + abs(ent_coef) * torch.where(p > 0, p * (logq.abs() + H[:, None]), torch.zeros_like(p)))
    zero = torch.zeros_like(grad)
    grad, bound = torch.where(on[:, None], grad, zero), torch.where(on[:, None], bound, zero)
    out = ((r < 1 - clip_low) | (r > 1 + clip_high)).double()
    terms = [-torch.minimum(free, held), kl, H, old - logp, out]
    sums = torch.stack([torch.where(on, share * t, torch.zeros_like(t)).sum() for t in terms])
    size = torch.stack([torch.where(on, share.abs() * t.abs(), torch.zeros_like(t)).sum() for t in terms])
    return grad, logp, sums, bound, size
