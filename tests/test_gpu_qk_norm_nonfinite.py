"""Norms of queries and keys with rotation: an infinity or a NaN in gamma or in a gradient shows in the elements that the formulas make of it, and in
no other element, whether or not it is turned with another one."""
import pytest
import torch

import memory_operators as plain
from test_gpu_qk_norm_rotate import EPS, _bwd, _fwd, _inputs

pytestmark = pytest.mark.gpu


def _formulas(p, interleaved):
    out = [plain.qk(p[n], p["g" + n], EPS, p["pos"], p["freq"], interleaved).v for n in "qk"]
    back = [plain.qk(p[n], p["g" + n], EPS, p["pos"], p["freq"], interleaved, p["d" + n + "o"]) for n in "qk"]
    return out + [b[0].v for b in back] + [b[1].v for b in back]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,pairs", [(64, 0), (64, 16), (64, 13), (64, 30), (64, 32), (16, 1), (16, 3), (200, 50), (50, 9)])
@pytest.mark.parametrize("which", ["gq", "gk", "dqo", "dko"])
def test_only_what_the_formulas_make_of_it(which, d, pairs, dtype, interleaved, bad):
    p = _inputs(3, 3, 2, d, pairs, dtype)
    before, exact = _fwd(p, interleaved) + _bwd(p, interleaved), _formulas(p, interleaved)
    for at in {0, 1, pairs - 1, pairs, 2 * pairs - 1, 2 * pairs, 2 * pairs + 1, d - 2, d - 1}:
        if not 0 <= at < d:
            continue
        q = {**p, which: p[which].clone()}
        if which[0] == "g":
            q[which][at] = bad
        else:
            q[which][1, 1, at] = bad
        after, now = _fwd(q, interleaved) + _bwd(q, interleaved), _formulas(q, interleaved)
        for name, a, b, v, w in zip(("q", "k", "dq", "dk", "dgamma_q", "dgamma_k"), before, after, exact, now):
            same = v == w
            assert torch.equal(a[same], b[same]), (name, at)
            assert not torch.isfinite(b[~torch.isfinite(w)]).any(), (name, at)
