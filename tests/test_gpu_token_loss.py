"""Token log-probabilities and the clipped token loss on the GPU against 64 bits, row by row and element by element.

Tolerances, u = 2^-24.  e^d of a logit d below the row's largest: 2 u of exp and u |d| of its argument; their sum over a vocabulary
of V at most V / 128 + 16 roundings on any path; its logarithm 2 u (1 + log V).  So a log-probability is off by at most
u (2 |logp| + V / 128 + 32 + 4 log V), where the scale adds u |x|.  A ratio carries that error, and u |old|; a gradient's element
the ratio's, that of p and a few u of its own terms, and half a step of its type."""
import math

import pytest
import torch

import plain_operators as plain
from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _inputs(rows, vocab, dtype, seed=0, masked=True, ld=None, spread=3.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn((rows, vocab), generator=g, device=DEV) * spread
    if masked and vocab >= 8:
        x = x.masked_fill(torch.rand((rows, vocab), generator=g, device=DEV) < 0.05, -math.inf)
        x[:, 0] = 0.5
    x = x.to(dtype)
    if ld:  # what lies behind the rows is not read
        wide = torch.full((rows, ld), float("nan"), dtype=dtype, device=DEV)
        wide[:, :vocab] = x
        x = wide[:, :vocab]
    gumbel = -torch.log(-torch.log(torch.rand((rows, vocab), generator=g, device=DEV).clamp(1e-20, 0.9999999)))
    tokens = (x.float() + gumbel).argmax(1).to(torch.int32)
    n = lambda: torch.randn(rows, generator=g, device=DEV)  # noqa: E731
    logp = plain.token_rows(x, tokens, 1.0)[0].float()
    return x, tokens, logp + 0.3 * n(), logp + 0.3 * n(), n(), (torch.rand(rows, generator=g, device=DEV) > 0.2).float()


def _tol_logp(x, logp, scale):
    V = x.shape[1]
    top = torch.where(torch.isinf(x), torch.zeros_like(x), x).double().abs().amax(1) * scale
    return U * (2 * torch.where(torch.isinf(logp), torch.zeros_like(logp), logp).abs() + V / 128 + 32 + 4 * math.log(V) + (2 * top if scale != 1 else 0))


def _logp(x, tokens, scale=1.0, entropy=True):
    logp = torch.full((x.shape[0],), float("nan"), device=DEV)
    H = torch.full_like(logp, float("nan")) if entropy else None
    ppo.ppo_token_logp(x, tokens, logp, H, scale)
    return logp, H


def _check_logp(x, tokens, scale=1.0):
    logp, H = _logp(x, tokens, scale)
    lw, hw, _, _ = plain.token_rows(x, tokens, scale)
    tol = _tol_logp(x, lw, scale)
    inf = torch.isinf(lw)
    assert torch.equal(torch.isinf(logp), inf) and not torch.isnan(logp).any() and not torch.isnan(H).any()
    assert float(torch.where(inf, 0 * tol, (logp.double() - lw).abs() - tol).max()) <= 0
    # sum of p |log p| is the entropy itself; each term carries the error of log p and of p
    assert float(((H.double() - hw).abs() - 4 * tol * (1 + hw)).max()) <= 0
    assert torch.equal(logp, _logp(x, tokens, scale, entropy=False)[0])


SHAPES = [(1, 1), (5, 2), (40, 3), (1024, 37), (33, 64), (7, 255), (9, 1000), (130, 4096), (3, 12345), (5, 32000), (2, 60001), (3, 131072), (2, 200003), (1, 1100000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_log_probabilities(rows, vocab, dtype):
    x, tokens, *_ = _inputs(rows, vocab, dtype)
    _check_logp(x, tokens)
    _check_logp(x, tokens, 0.7)
    x, tokens, *_ = _inputs(rows, vocab, dtype, 1, ld=vocab + 3)
    _check_logp(x, tokens)
    assert ppo.ppo_poll_status() == 0


def _loss(x, tokens, old, adv, ref=None, weight=None, grad=None, into=None, total=None, grad_scale=1.0, **coef):
    grad = torch.full(x.shape, float("nan"), dtype=x.dtype, device=DEV) if grad is None else grad
    loss = torch.full((5,), float("nan"), device=DEV) if into is None else into
    logp = torch.full((x.shape[0],), float("nan"), device=DEV)
    ws = torch.full((ppo.ppo_token_loss_workspace_bytes(x),), 0xA5, dtype=torch.uint8, device=DEV)
    ppo.ppo_token_loss_fwd_bwd(x, tokens, old, adv, total or x.shape[0], grad, loss, ref, weight, logp_out=logp, accumulate=into is not None,
                               workspace=ws, grad_scale=grad_scale, **coef)
    return grad, logp, loss


def _check_loss(x, tokens, old, adv, ref, weight, got, total=None, grad_scale=1.0, **coef):
    total = total or x.shape[0]
    gw, lw, sw, size, sums = plain.token_loss(x, tokens, old, adv, total, ref, weight, **coef)
    grad, logp, loss = got
    scale = coef.get("scale", 1.0)
    clean = torch.where(torch.isnan(x), torch.zeros_like(x), x)
    tol = _tol_logp(clean, lw, scale)
    assert not torch.isnan(logp).any() and not torch.isnan(grad).any() and not torch.isnan(loss).any()
    assert float(((logp.double() - lw).abs() - tol).max()) <= 0
    # rows whose ratio lies on a border to within its error may take either branch: none here
    r = torch.exp(lw - old.double())
    for border in (1 - coef.get("clip_low", 0.2), 1 + coef.get("clip_high", 0.2)):
        assert float((r - border).abs().min()) > 1e-5
    rel = tol + U * (2 * old.double().abs() + (2 * ref.double().abs() if ref is not None else 0) + 16)
    # p of a logit far below the largest: its argument's rounding
    top = torch.where(torch.isinf(clean), torch.zeros_like(clean), clean).double().abs().amax(1) * scale
    rel = 2 * rel + 4 * U * top
    if ref is not None:  # expm1(d) - its error is that of d, next to values as small as d
        rel = rel * (1 + 2 / 1.0)
        size = size + (weight.double() if weight is not None else 1.0 + 0 * lw)[:, None] / total * scale * coef.get("kl_coef", 0.0)
        size = torch.where((gw != 0).any(1)[:, None], size, 0 * size)
    want = gw * grad_scale
    bound = rel[:, None] * size * grad_scale + torch.finfo(x.dtype).eps / 2 * want.abs() * 1.01
    tiny = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}[x.dtype]
    assert float(((grad.double() - want).abs() - bound - tiny).max()) <= 0
    share = (weight.double() if weight is not None else torch.ones_like(lw)) / total
    slack = (share * rel * (4 + lw.abs() + old.abs().double() + (adv.abs().double() * r))).sum()
    assert float(((loss.double() - sw).abs() - slack - 4 * U * sums).max()) <= 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_loss_and_gradient(rows, vocab, dtype):
    x, tokens, old, ref, adv, weight = _inputs(rows, vocab, dtype)
    gs = 64.0 * rows if dtype == torch.float16 else 1.0
    for kw in (dict(), dict(clip_low=0.1, clip_high=0.3, kl_coef=0.2, ent_coef=0.05)):
        r, w = (ref, weight) if kw else (None, None)
        _check_loss(x, tokens, old, adv, r, w, _loss(x, tokens, old, adv, r, w, grad_scale=gs, **kw), grad_scale=gs, **kw)
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(20, 40), (9, 1001), (4, 32000), (3, 150001)])
def test_strides_scales_shares_and_the_gradient_in_place(rows, vocab, dtype):
    kw = dict(kl_coef=0.1, ent_coef=0.02, scale=1 / 1.5)
    x, tokens, old, ref, adv, weight = _inputs(rows, vocab, dtype, 3, ld=vocab + 5)
    old, ref = old / 1.5 - 1, ref / 1.5 - 1
    gs = 1000.0
    wide = torch.full((rows, vocab + 9), 7.0, dtype=dtype, device=DEV)
    got = _loss(x, tokens, old, adv, ref, weight, grad=wide[:, :vocab], total=1000, grad_scale=gs, **kw)
    _check_loss(x, tokens, old, adv, ref, weight, got, total=1000, grad_scale=gs, **kw)
    assert bool((wide[:, vocab:] == 7).all())
    same = torch.full((rows, vocab + 5), 7.0, dtype=dtype, device=DEV)
    same[:, :vocab] = x
    again = _loss(same[:, :vocab], tokens, old, adv, ref, weight, grad=same[:, :vocab], into=got[2].clone(), total=1000, grad_scale=gs, **kw)
    assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1]) and bool((same[:, vocab:] == 7).all())
    assert torch.allclose(again[2], 2 * got[2], rtol=4 * U, atol=0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [3, 50, 1001, 20000, 150001])
def test_rows_that_are_left_out_and_distributions_at_the_edge(vocab, dtype):
    x, tokens, old, ref, adv, _ = _inputs(12, vocab, dtype, 5, masked=False)
    weight = torch.ones(12, device=DEV)
    weight[0], weight[11] = 0, 0.25
    x[0] = float("nan")           # weight 0: not read
    tokens[1], tokens[2] = -100, vocab
    x[1] = float("inf")           # no token: not read
    x[3] = float("-inf")          # nothing can occur
    x[4] = float("-inf")
    x[4, vocab // 2], tokens[4] = 1.0, vocab // 2  # one token is certain
    x[5] = torch.finfo(dtype).min
    x[5, 1], tokens[5] = 2.0, 1
    x[6] = torch.finfo(dtype).min  # all alike, at the lowest value
    x[7, 0] = torch.finfo(dtype).max if dtype != torch.float32 else 1e30
    tokens[7] = 0
    x[8, tokens[8].long()] = float("-inf")  # a token that cannot occur any more
    logp, H = _logp(x, tokens)
    assert logp[1] == 0 and logp[2] == 0 and H[1] == 0 and logp[3] == -math.inf and H[3] == 0 and logp[4] == 0 and H[4] == 0
    assert logp[5] == 0 and abs(float(logp[6]) + math.log(vocab)) <= 1e-5 * math.log(vocab) and abs(float(H[6]) - math.log(vocab)) <= 1e-5 * math.log(vocab)
    assert logp[7] == 0 and H[7] == 0 and logp[8] == -math.inf and math.isfinite(float(H[8]))
    # the loss: finite rows only keep their place among the others
    keep = [i for i in range(12) if i != 8]
    old = torch.where(torch.isfinite(old), old, torch.zeros_like(old))
    old[4] = old[5] = old[7] = 0.1
    old[6] = -math.log(vocab) + 0.1
    args = x[keep], tokens[keep], old[keep], adv[keep]
    got = _loss(*args, None, weight[keep], ent_coef=0.1, grad_scale=64.0)
    for i in (0, 1, 2, 3):
        assert bool((got[0][i] == 0).all()) and got[1][i] == 0
    # a row of its own for each: the same values
    for i in (4, 5, 6, 7, 8, 9, 10):
        alone = _loss(x[keep][i:i + 1], tokens[keep][i:i + 1], old[keep][i:i + 1], adv[keep][i:i + 1], None, weight[keep][i:i + 1], total=11,
                      ent_coef=0.1, grad_scale=64.0)
        assert torch.equal(alone[0][0], got[0][i]) and torch.equal(alone[1][0], got[1][i])
    assert bool(torch.isfinite(got[0].float()).all()) and bool(torch.isfinite(got[2]).all())
    none = _loss(x[:4], tokens[:4], old[:4], adv[:4], None, weight[:4])
    assert bool((none[0] == 0).all()) and bool((none[2] == 0).all()) and bool((none[1] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 40, 3000, 20000, 150001])
def test_a_nan_in_a_row_that_counts_shows(vocab, dtype):
    x, tokens, old, ref, adv, _ = _inputs(4, vocab, dtype, 6)
    x[1, vocab // 2], x[2] = float("nan"), float("nan")
    logp, H = _logp(x, tokens)
    assert torch.isnan(logp).tolist() == [False, True, True, False] and torch.isnan(H).tolist() == [False, True, True, False]
    grad, lp, loss = _loss(x, tokens, torch.zeros_like(old), adv, ent_coef=0.1)
    assert torch.isnan(grad).any(1).tolist() == [False, True, True, False] and bool(torch.isnan(loss[:4:2]).all())


@pytest.mark.parametrize("rows,vocab,dtype", [(700, 9000, torch.bfloat16), (1500, 4104, torch.float32), (650, 32768, torch.float16), (900, 16384, torch.float32)])
def test_many_rows_are_each_what_a_few_give(rows, vocab, dtype):
    """Rows that go through the GPU in numbers, left-out ones among them, bit for bit as two at a time, and against 64 bits."""
    x, tokens, old, ref, adv, weight = _inputs(rows, vocab, dtype, 11)
    tokens[5], tokens[rows - 1] = -1, vocab
    gs = 64.0 * rows if dtype == torch.float16 else 1.0
    kw = dict(kl_coef=0.1, ent_coef=0.02)
    got = _loss(x, tokens, old, adv, ref, weight, grad_scale=gs, **kw)
    for at in (0, 4, 147, 148, 296, rows - 2):
        few = _loss(x[at:at + 2], tokens[at:at + 2], old[at:at + 2], adv[at:at + 2], ref[at:at + 2], weight[at:at + 2], total=rows, grad_scale=gs, **kw)
        assert torch.equal(few[0], got[0][at:at + 2]) and torch.equal(few[1], got[1][at:at + 2])
    part = slice(0, 60)
    _check_loss(x[part], tokens[part], old[part], adv[part], ref[part], weight[part],
                _loss(x[part], tokens[part], old[part], adv[part], ref[part], weight[part], grad_scale=gs, **kw), grad_scale=gs, **kw)
    logp, H = _logp(x, tokens)
    few_logp, few_H = _logp(x[:300], tokens[:300])
    assert torch.equal(logp[:300], few_logp) and torch.equal(H[:300], few_H)
    counted = (weight != 0) & (tokens >= 0) & (tokens < vocab)
    assert torch.equal(torch.where(counted, logp, torch.zeros_like(logp)), got[1])
    same = x.clone()
    again = _loss(same, tokens, old, adv, ref, weight, grad=same, grad_scale=gs, **kw)
    assert all(torch.equal(a, b) for a, b in zip(again, got))
    assert ppo.ppo_poll_status() == 0


def test_first_epoch_and_micro_batches():
    """Where the policy is still the one that acted every ratio is 1 and no row is clipped; micro-batches add up."""
    x, tokens, _, _, adv, _ = _inputs(300, 777, torch.bfloat16, 8)
    logp, H = _logp(x, tokens)
    grad, lp, loss = _loss(x, tokens, logp, adv, logp, None, kl_coef=0.5)
    assert torch.equal(lp, logp) and float(loss[1]) == 0 and float(loss[3]) == 0 and float(loss[4]) == 0
    assert abs(float(loss[0]) + float(adv.double().mean())) <= 1e-6
    sums = torch.zeros(5, device=DEV)
    for a, b in ((0, 100), (100, 101), (101, 300)):
        g, _, _ = _loss(x[a:b], tokens[a:b], logp[a:b], adv[a:b], logp[a:b], None, into=sums, total=300, kl_coef=0.5)
        assert torch.equal(g, grad[a:b])
    assert torch.allclose(sums, loss, rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("vocab", [37, 5000, 150001])
def test_other_streams_and_captured_calls(vocab):
    x, tokens, old, ref, adv, weight = _inputs(20, vocab, torch.bfloat16, 9)
    kw = dict(kl_coef=0.1, ent_coef=0.02)
    want = _loss(x, tokens, old, adv, ref, weight, **kw)
    grad, logp, loss, H = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty_like(want[2]), torch.empty_like(want[1])
    ws = torch.empty(ppo.ppo_token_loss_workspace_bytes(x), dtype=torch.uint8, device=DEV)

    def call():
        ppo.ppo_token_loss_fwd_bwd(x, tokens, old, adv, 20, grad, loss, ref, weight, logp_out=logp, workspace=ws, **kw)
        ppo.ppo_token_logp(x, tokens, H)

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert torch.equal(grad, want[0]) and torch.equal(logp, want[1]) and torch.equal(loss, want[2])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for t in (grad, logp, loss):
        t.fill_(7)
    ws.fill_(0x5A)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(grad, want[0]) and torch.equal(logp, want[1]) and torch.equal(loss, want[2])
