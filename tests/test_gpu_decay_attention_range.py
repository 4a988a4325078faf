"""Decay attention at the ends of the range of 32 bits: finite operands whose results are finite give finite results, within the bounds
of the other tests of this operator."""
import pytest
import torch

import plain_operators as plain
from paper_2509_16434_b200 import binding as ppo
from test_gpu_decay_attention import DEV, F32, Case, _near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large", ["q", "k", "v", "do"])
@pytest.mark.parametrize("shape", [(1, 2, 4, 2, 16, 24), (20, 2, 4, 2, 40, 64), (203, 1, 4, 4, 128, 33), (700, 1, 4, 2, 64, 64)], ids=lambda s: "-".join(map(str, s)))
def test_operands_near_the_largest_number(shape, large):
    """One operand between a quarter and the whole of the largest 32-bit number, the others small: every product and sum of the formulas
    (up to 700 terms) stays below 1e37."""
    c = Case(*shape, F32, 0.03)
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    c.lam = torch.tensor([0.5, 0.5005, 0.7, 1.0], device=DEV)
    for n in ("q", "k", "v", "do"):
        x = getattr(c, n)
        x.copy_(torch.where(x < 0, -1.0, 1.0) * (1 + 3 * torch.rand(x.shape, generator=g, device=DEV)) * (8.4e37 if n == large else 1e-5))
    c.s0 *= 1e-6
    c.ds *= 1e-6
    assert float(getattr(c, large).abs().max()) > 3e38
    (ow, sw), (oa, sa) = plain.attention(*c.args()), plain.attention_abs(*c.args())
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    assert max(float(x.max()) for x in (oa, sa, *size)) < 1e37
    o, s = c.fwd()
    _near(o, ow, oa, c.T, c.dk, F32)
    _near(s, sw, sa, c.T, c.dk, F32)
    got = c.bwd()
    for i in range(3):
        _near(got[i], want[i], size[i], c.T, max(c.dk, c.dv) * (c.heads // c.kv), F32)
    _near(got[3], want[3], size[3], c.T, c.dk, F32)
    assert ppo.ppo_poll_status() == 0
