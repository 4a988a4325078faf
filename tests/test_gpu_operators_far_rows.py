"""Rows so far apart that offsets pass 32 bits: the same bits as of rows side by side."""
import pytest
import torch

from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def _far(like, lead, total=5 << 29):
    """Places for tensors shaped as those of `like`, side by side in rows that are 16-byte aligned and `total` elements in all apart."""
    rows = 1
    for n in like[0].shape[:lead]:
        rows *= n
    width = (total // rows + 63) // 64 * 64
    assert rows * width > 1 << 31
    flat, at, out = torch.empty((rows, width), dtype=like[0].dtype, device=DEV), 0, []
    for t in like:
        n = t.numel() // rows
        out.append(flat[:, at:at + n].view(t.shape))
        at += (n + 63) // 64 * 64
    assert at <= width
    return out


@pytest.mark.parametrize("T,Be,dtype", [(10, 2, BF16), (40, 1, BF16), (130, 2, BF16), (700, 1, BF16), (70, 2, F32)])
def test_decay_attention(T, Be, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    heads, kv, dk, dv = 4, 2, 64, 48
    near = [n(T, Be, h, d).to(dtype) for h, d in ((heads, dk), (kv, dk), (kv, dv), (heads, dv), (heads, dv))]
    lam, s0 = 1 - torch.rand(heads, generator=g, device=DEV) / 20, n(Be, heads, dk, dv)

    def run(q, k, v, do, o, dq, dk_, dv_):
        ws = [torch.empty(ppo.ppo_decay_attention_workspace_bytes(q, k, v, b), dtype=torch.uint8, device=DEV) for b in (False, True)]
        s, ds = torch.empty_like(s0), torch.empty_like(s0)
        ppo.ppo_decay_attention_fwd(q, k, v, lam, o, None, s0, s, 0.125, ws[0])
        ppo.ppo_decay_attention_bwd(q, k, v, lam, do, dq, dk_, dv_, None, s0, s0, ds, 0.125, ws[1])
        return [x.contiguous() for x in (o, s, dq, dk_, dv_, ds)]

    want = run(*near, *(torch.empty_like(x) for x in near[:3]))
    far, out = _far(near, 2), _far(near[:3], 2)
    for a, b in zip(far, near):
        a.copy_(b)
    got = run(*far, *out)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("B,HW,C,groups", [(300, 1, 64, 4), (2, 40, 256, 4), (1, 600, 2048, 8), (3, 50, 30, 5)])
def test_group_norm(B, HW, C, groups):
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    near = [n(B, HW, C).to(BF16) for _ in range(2)]
    if C % 8:  # for rows of any alignment, in rows that no vector fits either
        near = [torch.nn.functional.pad(x, (0, 3))[:, :, :C] for x in near]
    gamma, beta = 1 + n(C) / 4, n(C) / 4

    def run(x, dy, y, dx):
        mean, rstd = (torch.empty((B, groups), device=DEV) for _ in range(2))
        dg, db = torch.empty_like(gamma), torch.empty_like(gamma)
        ws = [torch.empty(max(1, ppo.ppo_group_norm_workspace_bytes(x, groups, b)), dtype=torch.uint8, device=DEV) for b in (False, True)]
        ppo.ppo_group_norm_fwd(x, groups, gamma, beta, y, mean, rstd, "silu", 1e-5, ws[0])
        ppo.ppo_group_norm_bwd(x, groups, gamma, beta, mean, rstd, dy, dx, dg, db, "silu", False, ws[1])
        return [t.contiguous() for t in (y, mean, rstd, dx, dg, db)]

    want = run(*near, *(torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=DEV) for x in near))
    far = _far([*near, near[0], near[0]], 2)
    far[0].copy_(near[0]), far[1].copy_(near[1])
    assert all(torch.equal(a, b) for a, b in zip(run(*far), want))


@pytest.mark.parametrize("rows,vocab", [(600, 1000), (40, 5000), (20, 50001)])
def test_token_loss(rows, vocab):
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    x = (2 * torch.randn((rows, vocab), generator=g, device=DEV)).to(BF16)
    tokens = torch.randint(vocab, (rows,), generator=g, device=DEV, dtype=torch.int32)
    adv = torch.randn(rows, generator=g, device=DEV)

    def run(x, dx):
        logp, loss = torch.empty(rows, device=DEV), torch.empty(5, device=DEV)
        ppo.ppo_token_logp(x, tokens, logp)
        ws = torch.empty(ppo.ppo_token_loss_workspace_bytes(x), dtype=torch.uint8, device=DEV)
        ppo.ppo_token_loss_fwd_bwd(x, tokens, logp, adv, rows, dx, loss, ent_coef=0.01, workspace=ws)
        return logp, dx.contiguous(), loss

    want = run(x, torch.empty_like(x))
    far, out = _far([x, x], 1)
    far.copy_(x)
    assert all(torch.equal(a, b) for a, b in zip(run(far, out), want))
