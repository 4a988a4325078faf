"""The 64-bit forms that the kernels are tested against: gradients against differences and automatic differentiation, closed
cases.  And what the library refuses before it launches anything."""
import ctypes as C

import pytest
import torch

import plain_operators as plain
from paper_2509_16434_b200 import binding as ppo


def _normal(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64)


@pytest.mark.parametrize("resets", [False, True])
def test_attention_gradients_against_automatic_differentiation_and_differences(resets):
    g = torch.Generator().manual_seed(1)
    T, Be, heads, kv, dk, dv, scale = 7, 2, 4, 2, 3, 5, 0.6
    q, k, v = _normal(g, T, Be, heads, dk), _normal(g, T, Be, kv, dk), _normal(g, T, Be, kv, dv)
    lam, s0 = torch.tensor([0.0, 0.5, 0.9, 1.0], dtype=torch.float64), _normal(g, Be, heads, dk, dv)
    done = (torch.rand(T, Be, generator=g) < 0.3).to(torch.uint8) if resets else None
    do, ds = _normal(g, T, Be, heads, dv), _normal(g, Be, heads, dk, dv)
    leaves = [x.clone().requires_grad_() for x in (q, k, v, s0)]

    def value(q, k, v, s0):
        o, s = plain.attention(q, k, v, lam, done, s0, scale)
        return (o * do).sum() + (s * ds).sum()

    want = torch.autograd.grad(value(*leaves), leaves)
    got = plain.attention(q, k, v, lam, done, s0, scale, do, ds)
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)
    for i, x in enumerate((q, k, v, s0)):  # along a random direction
        d, h = _normal(g, *x.shape), 1e-6
        at = lambda f: value(*[y + f * d if j == i else y for j, y in enumerate((q, k, v, s0))])  # noqa: E731
        slope = (at(h) - at(-h)) / (2 * h)
        assert abs(slope - (got[i] * d).sum()) <= 1e-6 * (1 + abs(slope))


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_group_norm_gradients_against_automatic_differentiation(act):
    g = torch.Generator().manual_seed(2)
    x, gamma, beta = _normal(g, 3, 5, 12).requires_grad_(), _normal(g, 12).requires_grad_(), _normal(g, 12).requires_grad_()
    y, mean, rstd = plain.group_norm(x, 3, gamma, beta, act, 1e-5)
    dy = _normal(g, 3, 5, 12)
    want = torch.autograd.grad(y, (x, gamma, beta), dy)
    got = plain.group_norm_grad(x.detach(), 3, gamma.detach(), beta.detach(), mean.detach(), rstd.detach(), dy, act)
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-11, atol=1e-11)


def test_token_loss_gradient_against_automatic_differentiation():
    g = torch.Generator().manual_seed(3)
    rows, vocab = 40, 9
    logits = _normal(g, rows, vocab)
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    tokens[3] = -1
    weight = (torch.rand(rows, generator=g) > 0.2).double()
    old, ref, adv = (_normal(g, rows) * f - o for f, o in ((0.5, 2.0), (0.5, 2.0), (1.0, 0.0)))
    x = logits.clone().requires_grad_()
    logq = torch.log_softmax(1.3 * x, 1)
    logp = logq.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0]
    r = torch.exp(logp - old)
    s = torch.minimum(r * adv, r.clamp(0.8, 1.1) * adv)
    d = ref - logp
    H = -(logq.exp() * logq).sum(1)
    terms = -s + 0.3 * (d.exp() - d - 1) - 0.1 * H
    total = (torch.where(tokens >= 0, weight, 0.0) * terms).sum() / 37
    want, = torch.autograd.grad(total, x)
    got, _, sums, _, _ = plain.token_loss(logits, tokens, old, adv, 37, ref, weight, 0.2, 0.1, 0.3, 0.1, 1.3)
    assert torch.allclose(got, want, rtol=1e-11, atol=1e-13)
    assert abs(sums[0] + 0.3 * sums[1] - 0.1 * sums[2] - total.detach()) <= 1e-12


# ---- refusals: found on the host; the addresses are never read ----

P = 1 << 20  # stands for an aligned device address


def _attention(**change):
    d = dict(T=4, Be=2, heads=4, kv_heads=2, dk=16, dv=24, dtype=1, ldq=64, ldk=32, ldv=48, ldo=96, scale=1.0)
    d.update(change)
    return ppo.DecayAttentionDesc(*d.values())


def _fwd(desc, q=P, k=P, v=P, decay=P, done=None, s_in=None, o=P, s_out=None, ws=P, n=1 << 40):
    return ppo.lib().ppo_decay_attention_fwd(C.byref(desc), q, k, v, decay, done, s_in, o, s_out, ws, n, None)


def _bwd(desc, q=P, do=P, dq=P, s=None, ws=P, n=1 << 40):
    return ppo.lib().ppo_decay_attention_bwd(C.byref(desc), q, P, P, P, None, s, do, None, dq, P, P, None, ws, n, None)


def _step(desc, q=P, state=P, o=P):
    return ppo.lib().ppo_decay_attention_step(C.byref(desc), q, P, P, P, None, state, o, None)


@pytest.mark.parametrize("change,status", [
    (dict(T=0), 1), (dict(Be=0), 1), (dict(heads=0), 1), (dict(kv_heads=0), 1), (dict(dk=0), 1), (dict(dv=-1), 1), (dict(dtype=2), 1),
    (dict(dtype=-1), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(kv_heads=3), 2), (dict(ldq=63), 2), (dict(ldk=31), 2),
    (dict(ldv=47), 2), (dict(ldo=95), 2), (dict(dk=129, ldq=1000, ldk=1000), 7), (dict(dv=129, ldv=1000, ldo=1000), 7),
    (dict(T=1 << 30, Be=2), 7)])
def test_attention_descriptors_are_refused(change, status):
    d = _attention(**change)
    assert _fwd(d) == status and _bwd(d) == status and _step(d) == status
    assert ppo.lib().ppo_decay_attention_workspace_bytes(C.byref(d), 1) == 0


def test_attention_arguments_are_refused():
    d = _attention()
    for name in ("q", "k", "v", "decay", "o"):
        assert _fwd(d, **{name: None}) == 1
    assert _fwd(d, q=P + 1) == 3 and _fwd(d, decay=P + 2) == 3 and _fwd(d, s_in=P + 4) == 3 and _fwd(d, s_out=P + 8) == 3
    assert _bwd(d, q=None) == 1 and _bwd(d, do=None) == 1 and _bwd(d, dq=None) == 1 and _bwd(d, dq=P + 1) == 3 and _bwd(d, s=P + 4) == 3
    long = _attention(T=4096, Be=1, kv_heads=1)
    for f, backward in ((_fwd, 0), (_bwd, 1)):
        need = ppo.lib().ppo_decay_attention_workspace_bytes(C.byref(long), backward)
        assert need > 0 and f(long, ws=None, n=need) == 1 and f(long, n=need - 1) == 2 and f(long, ws=P + 4, n=need) == 3
    assert _step(d) == 2  # T == 4
    one = _attention(T=1)
    assert _step(one, q=None) == 1 and _step(one, state=None) == 1 and _step(one, state=P + 4) == 3 and _step(one, o=P + 1) == 3
    assert ppo.lib().ppo_decay_attention_fwd(None, P, P, P, P, None, None, P, None, None, 0, None) == 1


def _norm(**change):
    d = dict(B=2, HW=5, C=12, groups=3, act=1, dtype=1, ldx=12, ldy=16)
    d.update(change)
    return ppo.GroupNormDesc(*d.values())


def _norm_fwd(desc, eps=1e-5, x=P, gamma=P, beta=P, y=2 * P, mean=P, rstd=P, ws=P, n=1 << 40):
    return ppo.lib().ppo_group_norm_fwd(C.byref(desc), eps, x, gamma, beta, y, mean, rstd, ws, n, None)


def _norm_bwd(desc, x=P, gamma=P, beta=P, mean=P, dy=P, dx=2 * P, dgamma=P, dbeta=P, ws=P, n=1 << 40):
    return ppo.lib().ppo_group_norm_bwd(C.byref(desc), x, gamma, beta, mean, P, dy, dx, dgamma, dbeta, 0, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(B=0), 1), (dict(HW=0), 1), (dict(C=0), 1), (dict(groups=0), 1), (dict(act=3), 1), (dict(act=-1), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1),
    (dict(groups=5), 2), (dict(ldx=11), 2), (dict(ldy=11), 2), (dict(B=1 << 30), 7)])
def test_group_norm_descriptors_are_refused(change, status):
    assert _norm_fwd(_norm(**change)) == status and _norm_bwd(_norm(**change)) == status


def test_group_norm_arguments_are_refused():
    d = _norm()
    for name in ("x", "y", "mean", "rstd", "gamma", "beta"):
        assert _norm_fwd(d, **{name: None}) == 1
    assert _norm_fwd(d, eps=-1.0) == 1 and _norm_fwd(d, eps=float("nan")) == 1
    assert _norm_fwd(d, y=P) == 2  # in place, but another stride
    assert _norm_fwd(d, x=P + 1) == 3 and _norm_fwd(d, mean=P + 2) == 3
    for name in ("x", "mean", "dy", "dx", "gamma", "beta", "dgamma", "dbeta"):
        assert _norm_bwd(d, **{name: None}) == 1
    assert _norm_bwd(d, dx=P) == 2 and _norm_bwd(d, dx=2 * P + 1) == 3 and _norm_bwd(d, dgamma=P + 2) == 3
    need = ppo.lib().ppo_group_norm_workspace_bytes(C.byref(d), 1)
    assert need > 0 and _norm_bwd(d, ws=None, n=need) == 1 and _norm_bwd(d, n=need - 1) == 2


def _token(**change):
    d = dict(rows=4, vocab=10, dtype=1, ld=12, scale=1.0)
    d.update(change)
    return ppo.TokenDesc(*d.values())


def _coef(**change):
    c = dict(clip_low=0.2, clip_high=0.2, kl_coef=0.0, ent_coef=0.0, grad_scale=1.0, B_total=4)
    c.update(change)
    return ppo.TokenLossCoef(*c.values())


def _logp(desc, logits=P, tokens=P, logp=P, entropy=None):
    return ppo.lib().ppo_token_logp(C.byref(desc), logits, tokens, logp, entropy, None)


def _token_loss(desc, coef, logits=P, tokens=P, old=P, adv=P, weight=None, grad=2 * P, ld_grad=12, loss=P, ws=P, n=1 << 40):
    return ppo.lib().ppo_token_loss_fwd_bwd(C.byref(desc), C.byref(coef), logits, tokens, old, None, adv, weight, grad, ld_grad, None, loss, 0, ws, n,
                                            None)


@pytest.mark.parametrize("change,status", [(dict(rows=0), 1), (dict(vocab=0), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(scale=0.0), 1),
                                           (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(ld=9), 2)])
def test_token_descriptors_are_refused(change, status):
    assert _logp(_token(**change)) == status and _token_loss(_token(**change), _coef()) == status


def test_token_arguments_are_refused():
    d, c = _token(), _coef()
    assert _logp(d, logits=None) == 1 and _logp(d, tokens=None) == 1 and _logp(d, logp=None) == 1
    assert _logp(d, logits=P + 1) == 3 and _logp(d, tokens=P + 2) == 3 and _logp(d, entropy=P + 1) == 3
    for name in ("logits", "tokens", "old", "adv", "grad", "loss"):
        assert _token_loss(d, c, **{name: None}) == 1
    for change in (dict(B_total=0), dict(clip_low=-0.1), dict(clip_high=float("nan"))):
        assert _token_loss(d, _coef(**change)) == 1
    assert _token_loss(d, c, ld_grad=9) == 2 and _token_loss(d, c, grad=P, ld_grad=11) == 2
    assert _token_loss(d, c, grad=2 * P + 1) == 3 and _token_loss(d, c, weight=P + 2) == 3
    need = ppo.lib().ppo_token_loss_workspace_bytes(C.byref(d))
    assert need > 0 and _token_loss(d, c, ws=None, n=need) == 1 and _token_loss(d, c, n=need - 1) == 2


def test_sizes_and_scales_beyond_the_arithmetic_are_refused():
    assert _logp(_token(scale=2.0e38)) == 1  # times log2(e) it is no 32-bit number
    assert _step(_attention(T=0x7F000001, Be=1)) == 7  # steps are counted in 32 bits, in whole tiles


def test_the_binding_refuses_tensors_that_no_descriptor_says():
    def status(fn, *a, **k):
        with pytest.raises(ppo.PpoError) as e:
            fn(*a, **k)
        return e.value.status

    q, k, v, o, decay = torch.zeros(4, 2, 4, 16), torch.zeros(4, 2, 2, 16), torch.zeros(4, 2, 2, 24), torch.zeros(4, 2, 4, 24), torch.ones(4)
    f = ppo.ppo_decay_attention_fwd
    assert status(f, q, k.bfloat16(), v, decay, o) == 1
    assert status(f, q, k[:, :, :, :8], v, decay, o) == 2
    assert status(f, q.transpose(0, 1).contiguous().transpose(0, 1), k, v, decay, o) == 2  # rows out of order
    assert status(f, q, k, v, decay[:3], o) == 2
    assert status(f, q, k, v, decay.double(), o) == 1
    assert status(f, q, k, v, decay, o, done=torch.zeros(4, 2)) == 1
    assert status(f, q, k, v, decay, o, state_in=torch.zeros(2, 4, 24, 16)) == 2
    assert status(ppo.ppo_decay_attention_bwd, q, k, v, decay, o, q, k, v[:, :, :, :8]) == 2
    x = torch.zeros(2, 5, 12)
    assert status(ppo.ppo_group_norm_fwd, x, 3, None, None, x.half(), torch.zeros(2, 3), torch.zeros(2, 3)) == 1
    assert status(ppo.ppo_group_norm_fwd, x, 3, None, None, x.clone(), torch.zeros(3, 2), torch.zeros(2, 3)) == 2
    assert status(ppo.ppo_group_norm_fwd, x, 3, None, None, x.clone(), torch.zeros(2, 3), torch.zeros(2, 3), act="gelu") == 1
    logits = torch.zeros(4, 10)
    assert status(ppo.ppo_token_logp, logits, torch.zeros(4, dtype=torch.int64), torch.zeros(4)) == 1
    assert status(ppo.ppo_token_logp, logits.t(), torch.zeros(10, dtype=torch.int32), torch.zeros(10)) == 2
    assert status(ppo.ppo_token_logp, logits, torch.zeros(4, dtype=torch.int32), torch.zeros(3)) == 2
    # all of it fits, but it is not on a GPU
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    assert status(f, q, k, v, decay, o) == 1
    assert status(ppo.ppo_decay_attention_bwd, q, k, v, decay, o, q.clone(), k.clone(), v.clone(), workspace=ws) == 1
    assert status(ppo.ppo_decay_attention_step, q[0], k[0], v[0], decay, torch.zeros(2, 4, 16, 24), o[0]) == 1
    assert status(ppo.ppo_group_norm_fwd, x, 3, None, None, x.clone(), torch.zeros(2, 3), torch.zeros(2, 3)) == 1
    assert status(ppo.ppo_group_norm_bwd, x, 3, None, None, torch.zeros(2, 3), torch.zeros(2, 3), x.clone(), x.clone()) == 1
    four = torch.zeros(4)
    assert status(ppo.ppo_token_logp, logits, torch.zeros(4, dtype=torch.int32), four) == 1
    assert status(ppo.ppo_token_loss_fwd_bwd, logits, torch.zeros(4, dtype=torch.int32), four, four, 4, logits.clone(), torch.zeros(5), workspace=ws) == 1
