"""Causal convolution on the GPU against 64 bits, element by element, within running error bounds."""
import pytest
import torch

import memory_operators as plain
from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _inputs(T, Be, C, W, dtype, seed=0, done=0.1):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    p = dict(x=n(T, Be, C).to(dtype), w=n(C, W) / W ** 0.5, b=0.3 * n(C), s0=n(Be, W - 1, C).to(dtype), dy=n(T, Be, C).to(dtype),
             ds=n(Be, W - 1, C).to(dtype))
    p["done"] = (torch.rand(T, Be, generator=g, device=DEV) < done).to(torch.uint8)
    return p


def _nan(*s, dtype=torch.float32):
    return torch.full(s, float("nan"), dtype=dtype, device=DEV)


def _fwd(x, w, b, done, s0, act, y=None, s1=None):
    y = torch.full_like(x, float("nan")) if y is None else y
    s1 = _nan(x.shape[1], w.shape[1] - 1, x.shape[2], dtype=x.dtype) if s1 is None else s1
    ppo.ppo_causal_conv_fwd(x, w, b, y, done, s0, s1, act)
    return y, s1


def _bwd(x, w, b, done, s0, act, dy, ds, dx=None, into=None):
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    dw, db = (torch.full_like(w, float("nan")), _nan(w.shape[0])) if into is None else into
    ds0 = _nan(x.shape[1], w.shape[1] - 1, x.shape[2], dtype=x.dtype)
    ws = torch.full((ppo.ppo_causal_conv_workspace_bytes(x, w.shape[1]),), 0xFF, dtype=torch.uint8, device=DEV)
    ppo.ppo_causal_conv_bwd(x, w, b, dy, dx, dw, db, done, s0, ds, ds0, act, into is not None, ws)
    return dx, dw, db, ds0


def _check(p, act, done=True, state=True, bias=True):
    d, s, b = p["done"] if done else None, p["s0"] if state else None, p["b"] if bias else None
    y, s1 = _fwd(p["x"], p["w"], b, d, s, act)
    want, left = plain.conv(p["x"], p["w"], b, d, s, act)
    plain.within(y, want, "y")
    assert torch.equal(s1.double(), left)
    args = (p["x"], p["w"], b, d, s, act, p["dy"], p["ds"] if state else None)
    got = _bwd(*args)
    for a, v, name in zip(got, plain.conv(*args), ("dx", "dw", "db", "ds0")):
        plain.within(a, v, name)
    assert all(torch.equal(a, c) for a, c in zip(got, _bwd(*args)))
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Be,C", [(1, 1, 1), (1, 5, 64), (2, 3, 40), (3, 2, 7), (16, 9, 128), (31, 2, 24), (33, 3, 33), (65, 2, 1000), (257, 1, 48), (700, 2, 9),
                                    (16, 300, 12), (100, 40, 4)])
@pytest.mark.parametrize("W", [2, 4])
def test_values_and_gradients(T, Be, C, W, dtype):
    p = _inputs(T, Be, C, W, dtype)
    for act in ("none", "relu", "silu"):
        _check(p, act)


@pytest.mark.parametrize("W", [3, 5, 6, 7, 8])
@pytest.mark.parametrize("dtype", TYPES)
def test_widths(W, dtype):
    _check(_inputs(45, 3, 56, W, dtype), "silu")
    _check(_inputs(5, 3, 13, W, dtype), "silu")
    _check(_inputs(2, 2, 64, W, dtype, done=0.0), "silu")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("done,state,bias", [(False, False, False), (True, False, True), (False, True, True), (True, True, False)])
def test_without_flags_state_or_bias(done, state, bias, dtype):
    _check(_inputs(70, 3, 72, 4, dtype), "silu", done, state, bias)


def test_every_step_ends_an_episode():
    p = _inputs(40, 2, 16, 4, torch.float32, done=1.1)
    _check(p, "none")
    y, s1 = _fwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "none")
    assert not s1.any()
    plain.within(y[1:], plain.Num(p["w"][:, 3]) * plain.Num(p["x"][1:]) + plain.Num(p["b"]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,ld,at", [(48, 64, 8), (30, 37, 5), (64, 200, 64), (33, 40, 1)])
def test_rows_that_are_parts_of_wider_ones(C, ld, at, dtype):
    p = _inputs(50, 3, C, 4, dtype)
    wide = lambda t: _nan(50, 3, ld, dtype=dtype)[:, :, at:at + C].copy_(t)  # noqa: E731
    x, dy, y, dx = wide(p["x"]), wide(p["dy"]), wide(torch.zeros_like(p["x"])), wide(torch.zeros_like(p["x"]))
    assert not x.is_contiguous()
    want, s1 = _fwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu")
    got, s2 = _fwd(x, p["w"], p["b"], p["done"], p["s0"], "silu", y)
    assert torch.equal(got, want) and torch.equal(s1, s2)
    a = _bwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu", p["dy"], p["ds"])
    b = _bwd(x, p["w"], p["b"], p["done"], p["s0"], "silu", dy, p["ds"], dx)
    assert torch.equal(a[0], b[0]) and torch.equal(a[3], b[3])
    for v, w in zip(b[1:3], plain.conv(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu", p["dy"], p["ds"])[1:3]):
        plain.within(v, w)
    for t in (y, dx):  # what lies between the rows stays as it was
        whole = t.as_strided((50 * 3, ld), (ld, 1), t.storage_offset() - at)
        assert bool(torch.isnan(whole[:, :at]).all()) and bool(torch.isnan(whole[:, at + C:]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 2, 3, 80])
def test_the_state_that_is_left_in_place_of_the_one_that_came(T, dtype):
    p = _inputs(T, 4, 40, 4, dtype)
    want, left = _fwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu")
    state = p["s0"].clone()
    got, _ = _fwd(p["x"], p["w"], p["b"], p["done"], state, "silu", None, state)
    assert torch.equal(got, want) and torch.equal(state, left)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Be,C,W", [(1, 1, 2), (3, 64, 4), (5, 33, 8), (7, 24, 3)])
def test_decisions_one_by_one_give_what_the_sequence_gives(Be, C, W, dtype):
    p = _inputs(30, Be, C, W, dtype, done=0.15)
    want, left = _fwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu")
    state, start = p["s0"].clone(), None
    for t in range(30):
        y = torch.full_like(p["x"][t], float("nan"))
        ppo.ppo_causal_conv_step(p["x"][t], p["w"], p["b"], state, y, start, "silu")
        start = p["done"][t]
        assert torch.equal(y, want[t])
    live = start == 0
    assert torch.equal(state[live], left[live]) and not left[~live].any()


def test_sequences_chain_through_their_states():
    p = _inputs(90, 3, 40, 4, torch.bfloat16)
    want, left = _fwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu")
    state, at = p["s0"], 0
    for n in (1, 2, 40, 47):
        y, state = _fwd(p["x"][at:at + n], p["w"], p["b"], p["done"][at:at + n], state, "silu")
        assert torch.equal(y, want[at:at + n])
        at += n
    assert torch.equal(state, left)


def test_gradients_are_added_to_what_is_there():
    p = _inputs(60, 5, 72, 4, torch.float32)
    args = (p["x"], p["w"], p["b"], p["done"], p["s0"], "silu", p["dy"], p["ds"])
    _, dw, db, _ = _bwd(*args)
    was = torch.randn_like(dw), torch.randn_like(db)
    _, aw, ab, _ = _bwd(*args, into=(was[0].clone(), was[1].clone()))
    assert float((aw - was[0] - dw).abs().max()) <= 2.0 ** -22 * float(aw.abs().max() + dw.abs().max())
    assert float((ab - was[1] - db).abs().max()) <= 2.0 ** -22 * float(ab.abs().max() + db.abs().max())


def test_gradients_of_parameters_may_be_left_out():
    p = _inputs(60, 5, 72, 4, torch.bfloat16)
    want = _bwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu", p["dy"], p["ds"])
    for keep in ((True, False), (False, True), (False, False)):
        dx, dw, db = torch.full_like(p["x"], float("nan")), torch.full_like(p["w"], 7.0), torch.full_like(p["b"], 7.0)
        ws = torch.empty(ppo.ppo_causal_conv_workspace_bytes(p["x"], 4), dtype=torch.uint8, device=DEV)
        ppo.ppo_causal_conv_bwd(p["x"], p["w"], p["b"], p["dy"], dx, dw if keep[0] else None, db if keep[1] else None, p["done"], p["s0"], p["ds"], None,
                                "silu", False, ws)
        assert torch.equal(dx, want[0])
        assert torch.equal(dw, want[1]) if keep[0] else bool((dw == 7).all())
        assert torch.equal(db, want[2]) if keep[1] else bool((db == 7).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("C", [16, 5])
def test_a_value_that_is_no_number_stays_on_its_side_of_a_flag(C, bad):
    """Of env 1's channel 3: its steps 6 .. 9 see step 6's input, but step 7 ends an episode."""
    p = _inputs(40, 3, C, 4, torch.float32, done=0.0)
    p["done"][7, 1] = 1
    y0, _ = _fwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu")
    g0 = _bwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu", p["dy"], p["ds"])
    x = p["x"].clone()
    x[6, 1, 3] = bad
    y1, _ = _fwd(x, p["w"], p["b"], p["done"], p["s0"], "silu")
    same = torch.ones_like(y0, dtype=torch.bool)
    same[6:8, 1, 3] = False
    assert torch.equal(y0[same], y1[same]) and not torch.isfinite(y1[6, 1, 3])
    dy = p["dy"].clone()
    dy[8, 1, 3] = bad  # reaches back to the step behind the flag only
    g1 = _bwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu", dy, p["ds"])
    same = torch.ones_like(y0, dtype=torch.bool)
    same[8, 1, 3] = False
    assert torch.equal(g0[0][same], g1[0][same]) and not torch.isfinite(g1[0][8, 1, 3]) and torch.equal(g0[3], g1[3])
