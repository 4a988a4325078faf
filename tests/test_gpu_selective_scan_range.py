"""Selective scan over segments where the factors of a segment, multiplied with one another, leave the range of 32 bits although no state and no gradient
of the recurrence does."""
import pytest
import torch

import memory_operators as plain
from test_gpu_selective_scan import DEV, GRADS, _bwd, _fwd, _inputs, _want

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _steps(T, Be, channels, N, groups, dtype, seed=0):
    """Inputs without softplus, decays between -1.5 and -1.4, and step sizes of 1/8; a segment has 32 steps."""
    p = _inputs(T, Be, channels, N, groups, dtype, seed, done=0.0)
    p["A"] = -1.4 - 0.1 * torch.rand(channels, N, device=DEV)
    p.update(softplus=False, bias=None, dt=torch.full_like(p["dt"], 0.125), s0=None, ds=None)
    return p


def _check(p):
    y, s1 = _fwd(p, s1=torch.full((p["x"].shape[1],) + tuple(p["A"].shape), float("nan"), device=DEV))
    want, left = _want(p, False)
    plain.within(y, want, "y")
    plain.within(s1, left, "state")
    got, want = _bwd(p), _want(p, True)
    for name in GRADS:
        if got[name] is not None:
            plain.within(got[name], want[name], name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Be,channels,N,groups", [(256, 1, 40, 16, 1), (130, 2, 24, 12, 2), (96, 3, 20, 40, 1), (96, 150, 20, 16, 1)])
def test_states_and_gradients_of_zero_that_would_grow(T, Be, channels, N, groups, dtype):
    """Factors of 16 to 20 a step; inputs in the last two steps, gradients in the first two, zeros elsewhere."""
    p = _steps(T, Be, channels, N, groups, dtype)
    p["dt"][:] = -2
    p["x"][:-2] = 0
    p["dy"][2:] = 0
    _check(p)


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N", [16, 12, 40])
@pytest.mark.parametrize("done", [False, True])
def test_what_goes_through_a_segment_far_up_or_down(N, dtype, up, done):
    """Three segments; the factors of the second one come to 2^129 and more, or 2^-129 and less.  Tiny (or huge) values go in and ordinary ones come out."""
    p = _steps(96, 2, 40, N, 1, dtype)
    p["dt"][32:64] = -2 if up else 2
    size = 2.0 ** (-112 if up else 110)
    p["x"][:31] = 0
    p["x"][32:94] = 0
    p["x"][31] = (p["x"][31].float() * size).to(dtype)
    p["dy"][2:64] = 0
    p["dy"][65:] = 0
    p["dy"][64] = (p["dy"][64].float() * size).to(dtype)
    p["z"] = None
    p["D"] = None
    if done:
        p["done"][40, 1] = 1
    _check(p)


@pytest.mark.parametrize("at", [62, 63])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_gradient_from_the_end_of_a_segment_that_grows(dtype, at):
    """Of two segments the second one hands a gradient on that is tiny at its last steps and ordinary at its first."""
    p = _steps(64, 2, 40, 16, 1, dtype)
    p["dt"][32:] = -2
    p["x"][:62] = 0
    p["dy"][:] = 0
    p["dy"][at] = (torch.randn(2, 40, device=DEV) * 2.0 ** -112).to(dtype)
    p["z"] = None
    _check(p)


@pytest.mark.parametrize("channels", [40, 39])
@pytest.mark.parametrize("z", [-80.0, -30.0])
def test_a_gate_that_is_nearly_shut_on_large_values(channels, z):
    """The gradient of the gate: outputs of 2^60 and gradients of 2^70, whose product leaves the range, times a slope of 1e-33 or 1e-12."""
    p = _inputs(20, 2, channels, 16, 1, torch.float32, done=0.0)
    p["x"] = p["x"] * 2.0 ** 60
    p["dy"] = p["dy"] * 2.0 ** 70
    p["z"][:] = z
    p.update(s0=None, ds=None)
    got, want = _bwd(p), _want(p, True)
    for name in ("dz", "ddt", "dx", "dB", "dC"):
        plain.within(got[name], want[name], name)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,N", [(88, 16), (300, 16), (177, 17)])
def test_an_element_that_is_no_number_leaves_its_neighbours_as_they_were(T, N, bad):
    p = _inputs(T, 2, 40, N, 1, torch.float32, done=0.0)
    want = _bwd(p)
    q = {**p, "C": p["C"].clone()}
    q["C"][T - 8, 1, 0, 2] = bad
    got = _bwd(q)
    rest = torch.arange(N, device=DEV) != 2
    assert torch.equal(got["dA"][:, rest], want["dA"][:, rest]) and not torch.isfinite(got["dstate"][1, :, 2]).any()
    assert torch.equal(got["dB"][..., rest], want["dB"][..., rest]) and torch.equal(got["dstate"][..., rest], want["dstate"][..., rest])
