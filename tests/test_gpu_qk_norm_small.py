"""Norms of queries and keys where a head's mean square is below the normal numbers of 32 bits."""
import pytest
import torch

import memory_operators as plain
from test_gpu_qk_norm_rotate import _bwd, _fwd, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 50])
def test_heads_of_zeros_with_an_eps_below_the_normal_numbers(d, dtype):
    p = _inputs(6, 4, 2, d, d // 2, dtype)
    p["q"][2, 1] = 0
    p["k"][3] = 0
    qo, ko = _fwd(p, False, eps=1e-40)
    assert not qo[2, 1].any() and not ko[3].any() and bool(torch.isfinite(qo).all()) and bool(torch.isfinite(ko).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 50])
def test_heads_of_values_whose_squares_are_below_the_normal_numbers(d, dtype):
    """Values about 2^-66: a square, about 2^-132, is off by up to 2^-150 and their mean by as much again, relative to it 2^-17 and the
    root by half of that; four times as much where a head's values are smaller than that by chance."""
    p = _inputs(6, 4, 2, d, d // 2, dtype)
    p["q"] = (torch.randn(6, 4, d, device="cuda") * 2.0 ** -66).to(dtype)
    qo, _ = _fwd(p, False, eps=0.0)
    want = plain.qk(p["q"], p["gq"], 0.0, p["pos"], p["freq"], False)
    # a rotation mixes the two elements of a pair: relative to both together
    size = want.v.abs() + want.v.abs().amax(-1, keepdim=True)
    tol = want.e * plain.U + (2.0 ** -16 + torch.finfo(dtype).eps / 2) * size
    assert bool(torch.isfinite(qo).all()) and bool(((qo.double() - want.v).abs() <= tol).all())
    dq = _bwd({**p, "dqo": (p["dqo"].float() * 2.0 ** -66).to(dtype)}, False, eps=0.0)[0]
    assert bool(torch.isfinite(dq).all())
