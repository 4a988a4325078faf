"""States that decay attention hands out are those of 32 bits, whatever the type of the operands: one step adds to an empty state, so
that nothing but its own roundings shows.

S = lambda^n a b^T of one step, element by element.  In units of 2^-24 of the element, the bound is
  4 + 2.1 |n log2 lambda|   the power: exp2f is off by two steps of 2^-23, its argument by |n log2 lambda| times a step of log2f and
                            half a step of the product, ln 2 (2 + 1) = 2.1 units for each
  1                         the power times the scale
  2                         their product with a, in terms of 16 bits that hold at least 2^-23 of it
  8                         up to four sums of such terms, each cut off below 2^-23
  1                         two shares of a state joined
and step by step (32 bits) 5 for the power of each tile of 8 steps, and of the last one, that the state is multiplied by.
A key in two terms instead of the three or four of these kernels is off by up to 1.64 2^-16 (420 units) among as many elements."""
import pytest
import torch

from paper_2509_16434_b200 import binding as ppo
from test_gpu_decay_attention import BF16, DEV, F32, Case

pytestmark = pytest.mark.gpu
LAM = (0.875, 0.98, 0.998, 1.0)


def _bound(n, dtype):
    """[Be, heads, 1, 1] of the distances [Be]."""
    n = torch.tensor(n, dtype=torch.float64)[:, None]
    far = n * torch.tensor(LAM).double().log2().abs()
    tiles = 0 if dtype == BF16 else 5 * (n // 8 + 3)
    return ((16 + 2.1 * far + tiles) * 2.0 ** -24).to(DEV)[..., None, None]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 64), (48, 128), (128, 128), (104, 40)])
@pytest.mark.parametrize("T,Be", [(9, 4), (16, 4), (17, 4), (64, 4), (65, 4), (127, 4), (200, 4), (700, 4), (330, 76)])
def test_one_step(T, Be, dk, dv, dtype):
    c = Case(T, Be, 4, 2, dk, dv, dtype, state=False)
    c.lam = torch.tensor(LAM, device=DEV)
    last = min(T - 1, (T - 1) % 128)  # of its chunk
    n = [min((1, 5, 17, 40)[e % 4], last) for e in range(Be)]
    cut = ppo.ppo_decay_attention_workspace_bytes(c.q, c.k, c.v, False) > 0
    assert cut == (T == 700)
    powers = c.lam.double()[None] ** torch.tensor(n, device=DEV).double()[:, None]  # [Be, heads]
    k, do = c.k.clone(), c.do.clone()
    c.k.zero_(), c.do.zero_()
    want, back = [], []
    for e in range(Be):
        at = T - 1 - n[e]
        c.k[at, e], c.do[n[e] - 1, e] = k[at, e], do[n[e] - 1, e]
        one = k[at, e].double()[:, :, None] * c.v[at, e].double()[:, None, :]
        want.append(one.repeat_interleave(2, 0))
        back.append(c.q[n[e] - 1, e].double()[:, :, None] * do[n[e] - 1, e].double()[:, None, :])
    scale = float(torch.tensor(c.scale, dtype=F32))
    want, back = torch.stack(want) * powers[..., None, None], torch.stack(back) * powers[..., None, None] * scale
    s, ds = c.fwd()[1], c.bwd()[3]
    for got, ref in ((s, want), (ds, back)):
        units = (got.double() - ref).abs() / (ref.abs() * _bound(n, dtype) + 1e-30)
        assert float(units.max()) <= 1, float(units.max())
    assert ppo.ppo_poll_status() == 0
