"""Gradients of the selective scan where a sequence's last steps do not fill a group of four: what is no number there stays where the formulas put it."""
import pytest
import torch

from test_gpu_selective_scan import GRADS, _bwd, _inputs

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
LENGTHS = [1, 2, 3, 4, 5, 14, 16, 17, 18, 19, 20, 301, 303]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", LENGTHS)
def test_a_last_flag_drops_the_gradient_of_the_state_that_is_left(T, dtype, bad):
    p = _inputs(T, 3, 40, 16, 1, dtype, done=0.0)
    p["done"][T - 1, 1] = 1
    want = _bwd(p)
    q = {**p, "ds": p["ds"].clone()}
    q["ds"][1, 7, 3] = bad
    got = _bwd(q)
    for n in GRADS:
        assert torch.equal(got[n], want[n]), n


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("N", [16, 12, 40])
@pytest.mark.parametrize("T", LENGTHS)
def test_the_last_step_s_input_is_no_part_of_the_gradient_of_a(T, N, bad):
    p = _inputs(T, 2, 40, N, 1, torch.float32, done=0.0)
    want = _bwd(p)
    q = {**p, "x": p["x"].clone()}
    q["x"][T - 1, 1, 7] = bad
    got = _bwd(q)
    for n in ("dA", "dstate"):
        assert torch.equal(got[n], want[n]), n
    assert torch.equal(got["dx"][:T - 1], want["dx"][:T - 1])
    assert not torch.isfinite(got["dC"][T - 1, 1]).any() and torch.equal(got["dC"][:T - 1], want["dC"][:T - 1])


@pytest.mark.parametrize("T", [1, 3, 17, 20, 301])
def test_a_decay_that_is_no_number_leaves_the_last_step_s_own_gradients(T):
    """g of the last step holds no factor: dB and dx there are the formula's whatever A is."""
    p = _inputs(T, 2, 40, 16, 1, torch.float32, done=0.0)
    want = _bwd(p)
    q = {**p, "A": p["A"].clone()}
    q["A"][7, 3] = float("nan")
    got = _bwd(q)
    assert torch.equal(got["dB"][T - 1], want["dB"][T - 1]) and torch.equal(got["dx"][T - 1], want["dx"][T - 1])
