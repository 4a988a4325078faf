"""Gradients of a selective scan whose channels' states have 2^31 elements and more in all: counts and places pass 32 bits."""
import math

import pytest
import torch

from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("channels", [1 << 25, (1 << 25) + 4])
def test_parameters_of_more_elements_than_32_bits_count(channels):
    """One step of one env: h = exp(d A) s + d x B, y = C h + D x.  With d = 1/2, A = -1, B = C = s = 1 and gradients of 0 to 4 by the channel,
    dL/dA = dy exp(-1/2) / 2 for every element, dL/dD = dy x, dL/ddt_bias = 64 dy (x - exp(-1/2))."""
    N = 64
    torch.cuda.empty_cache()
    x = torch.full((1, 1, channels), 0.25, dtype=torch.bfloat16, device=DEV)
    dt = torch.full_like(x, 0.5)
    dy = (torch.arange(channels, device=DEV) % 5).to(torch.bfloat16).view(1, 1, channels)
    B = torch.ones(1, 1, 1, N, dtype=torch.bfloat16, device=DEV)
    A = torch.full((channels, N), -1.0, device=DEV)
    s0, D, bias = torch.ones(1, channels, N, device=DEV), torch.ones(channels, device=DEV), torch.zeros(channels, device=DEV)
    dx, ddt, dB, dC = (torch.empty_like(t) for t in (x, dt, B, B))
    dA, dD, dbias = torch.full_like(A, float("nan")), torch.full_like(D, float("nan")), torch.full_like(bias, float("nan"))
    ws = torch.empty(ppo.ppo_selective_scan_workspace_bytes(x, B, True), dtype=torch.uint8, device=DEV)
    ppo.ppo_selective_scan_bwd(x, dt, A, B, B, dy, dx, ddt, dA, dB, dC, D, None, bias, False, None, s0, None, dD, None, dbias, None, workspace=ws)
    assert ppo.ppo_poll_status() == 0
    g, f = dy.view(-1).float(), math.exp(-0.5)
    # an exponential (a few units), one product, and sums of 64 such
    for at in range(0, channels, 1 << 22):
        part = slice(at, at + (1 << 22))
        assert float((dA[part] - 0.5 * f * g[part, None]).abs().max()) <= 16 * 2.0 ** -24 * 2
    assert torch.equal(dD, 0.25 * g)
    assert float((dbias - 64 * (0.25 - f) * g).abs().max()) <= 64 * 4 * 80 * 2.0 ** -24
