"""Selective scan on the GPU against 64 bits, element by element, within running error bounds."""
import pytest
import torch

import memory_operators as plain
from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
GRADS = ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias", "dstate")


def _inputs(T, Be, channels, N, groups, dtype, seed=0, done=0.05, gate=True):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    p = dict(x=n(T, Be, channels).to(dtype), dt=n(T, Be, channels).to(dtype), A=-torch.exp(n(channels, N)), B=n(T, Be, groups, N).to(dtype),
             C=n(T, Be, groups, N).to(dtype), D=n(channels), z=n(T, Be, channels).to(dtype) if gate else None, bias=n(channels) - 3,
             s0=n(Be, channels, N), dy=n(T, Be, channels).to(dtype), ds=n(Be, channels, N), softplus=True)
    p["done"] = (torch.rand(T, Be, generator=g, device=DEV) < done).to(torch.uint8)
    return p


def _like(t):
    return None if t is None else torch.full_like(t, float("nan"))


def _space(p, backward):
    need = ppo.ppo_selective_scan_workspace_bytes(p["x"], p["B"], backward)
    return torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) if need else None


def _fwd(p, y=None, s1=None):
    y, s1 = _like(p["x"]) if y is None else y, _like(p["ds"]) if s1 is None else s1
    ppo.ppo_selective_scan_fwd(p["x"], p["dt"], p["A"], p["B"], p["C"], y, p["D"], p["z"], p["bias"], p["softplus"], p["done"], p["s0"], s1, _space(p, False))
    return y, s1


def _bwd(p, into=None, outs=None, accumulate=False):
    o = {"dx": _like(p["x"]), "ddt": _like(p["dt"]), "dA": _like(p["A"]), "dB": _like(p["B"]), "dC": _like(p["C"]), "dD": _like(p["D"]), "dz": _like(p["z"]),
         "ddt_bias": _like(p["bias"]), "dstate": torch.full(p["x"].shape[1:] + p["A"].shape[1:], float("nan"), device=DEV)}
    o.update(into or {})
    ppo.ppo_selective_scan_bwd(p["x"], p["dt"], p["A"], p["B"], p["C"], p["dy"], o["dx"], o["ddt"], o["dA"], o["dB"], o["dC"], p["D"], p["z"], p["bias"],
                               p["softplus"], p["done"], p["s0"], p["ds"], o["dD"], o["dz"], o["ddt_bias"], o["dstate"], accumulate, _space(p, True))
    return o


def _want(p, backward):
    return plain.scan(p["x"], p["dt"], p["A"], p["B"], p["C"], p["D"], p["z"], p["bias"], p["softplus"], p["done"], p["s0"], *((p["dy"], p["ds"]) if backward else ()))


def _check(p):
    y, s1 = _fwd(p)
    want, left = _want(p, False)
    plain.within(y, want, "y")
    plain.within(s1, left, "state")
    got, want = _bwd(p), _want(p, True)
    for name in GRADS:
        if got[name] is not None:
            plain.within(got[name], want[name], name)
    again = _bwd(p)
    assert all(torch.equal(got[n], again[n]) for n in GRADS if got[n] is not None)
    assert ppo.ppo_poll_status() == 0


SHAPES = [(1, 1, 1, 1, 1), (1, 7, 40, 16, 1), (2, 3, 5, 3, 5), (3, 2, 64, 16, 2), (16, 5, 256, 16, 1), (17, 3, 130, 16, 1), (31, 2, 48, 12, 3), (40, 2, 37, 8, 1),
          (33, 3, 66, 32, 2), (64, 1, 129, 64, 1), (50, 2, 24, 17, 4), (129, 2, 200, 16, 2), (600, 1, 70, 16, 1), (16, 130, 20, 10, 1), (5, 40, 300, 64, 3)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_values_and_gradients(shape, dtype):
    _check(_inputs(*shape, dtype))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,Be,channels", [(20, 3, 72), (300, 2, 40)])
def test_without_what_may_be_left_out(T, Be, channels, dtype):
    full = _inputs(T, Be, channels, 16, 1, dtype)
    for gone in (("z",), ("D",), ("bias",), ("done",), ("s0",), ("ds",), ("z", "D", "bias", "done", "s0", "ds")):
        p = {**full, **{n: None for n in gone}}
        if "ds" in gone:  # the state that is left is not wanted either
            y = _like(p["x"])
            ppo.ppo_selective_scan_fwd(p["x"], p["dt"], p["A"], p["B"], p["C"], y, p["D"], p["z"], p["bias"], True, p["done"], p["s0"], None, _space(p, False))
            plain.within(y, _want(p, False)[0], "y")
            got, want = _bwd(p), _want(p, True)
            for name in GRADS:
                if got[name] is not None:
                    plain.within(got[name], want[name], name)
        else:
            _check(p)


@pytest.mark.parametrize("T,Be,channels,N", [(12, 3, 40, 16), (300, 1, 40, 16)])
def test_step_sizes_as_they_are(T, Be, channels, N):
    p = _inputs(T, Be, channels, N, 1, torch.float32)
    p.update(softplus=False, dt=0.2 * p["dt"].abs(), bias=0.01 * p["bias"].abs())
    _check(p)


def test_step_sizes_from_nothing_to_large():
    p = _inputs(60, 2, 64, 16, 1, torch.float32)
    p["dt"] = torch.linspace(-60, 40, 60, device=DEV)[:, None, None].expand(60, 2, 64).contiguous()
    p["bias"] = None
    _check(p)


def test_every_step_ends_an_episode():
    p = _inputs(40, 2, 48, 16, 1, torch.float32, done=1.1)
    _check(p)
    assert not _fwd(p)[1].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,Be", [(16, 6), (300, 1), (2000, 1)])
def test_flags_on_and_next_to_the_borders_of_tiles(T, Be, dtype):
    p = _inputs(T, Be, 40, 16, 1, dtype, done=0.0)
    for t in (0, 3, 4, 14, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, T - 2, T - 1):
        if t < T:
            p["done"][t, t % Be] = 1
    if T < 1000:
        return _check(p)
    y, s1 = _fwd(p)
    want, left = _want(p, False)
    plain.within(y, want, "y")
    plain.within(s1, left, "state")
    got, want = _bwd(p), _want(p, True)
    for name in GRADS:
        plain.within(got[name], want[name], name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [9, 200])
def test_rows_that_are_parts_of_wider_ones(T, dtype):
    """One row of x, dt, z, B and C side by side, as a projection leaves them, aligned and not."""
    channels, N, groups = 48, 16, 2
    p = _inputs(T, 2, channels, N, groups, dtype)
    want, left = _fwd(p)
    grads = _bwd(p)
    for at in (8, 3):
        few = groups * N
        widths = (channels, channels, channels, few, few)
        total = at + sum(widths) + 5 + (3 if at == 8 else 0)
        total += (-total) % 8 if at == 8 else 0

        def wide():
            rows, out, o = torch.full((T, 2, total), float("nan"), dtype=dtype, device=DEV), [], at
            for w in widths:
                out.append(rows[:, :, o:o + w])
                o += w
            out[3], out[4] = (v.unflatten(2, (groups, N)) for v in out[3:])
            return rows, dict(zip(("x", "dt", "z", "B", "C"), out))
        _, part = wide()
        for n in part:
            part[n].copy_(p[n])
        q = {**p, **part}
        got, s1 = _fwd(q)
        assert torch.equal(got.contiguous(), want) and torch.equal(s1, left)
        rows, g = wide()
        out = _bwd(q, {"d" + n: v for n, v in g.items()})
        for n in GRADS:
            if at == 8:
                assert torch.equal(out[n].contiguous(), grads[n]), n
        for name, v in _want(p, True).items():
            plain.within(out[name].contiguous(), v, name)
        assert bool(torch.isnan(rows[:, :, :at]).all()) and bool(torch.isnan(rows[:, :, at + sum(widths):]).all())


@pytest.mark.parametrize("T,Be,channels", [(1, 3, 40), (16, 3, 40), (500, 1, 40)])
def test_states_in_place(T, Be, channels):
    p = _inputs(T, Be, channels, 16, 1, torch.bfloat16)
    want, left = _fwd(p)
    q = {**p, "s0": p["s0"].clone()}
    got, _ = _fwd(q, None, q["s0"])
    assert torch.equal(got, want) and torch.equal(q["s0"], left)
    grads = _bwd(p)
    q = {**p, "ds": p["ds"].clone()}
    out = _bwd(q, {"dstate": q["ds"]})
    assert all(torch.equal(out[n], grads[n]) for n in GRADS)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Be,channels,N,groups", [(1, 1, 1, 1), (3, 64, 16, 1), (2, 30, 12, 2), (5, 48, 64, 4), (2, 50, 7, 1), (70, 130, 16, 1)])
def test_decisions_one_by_one_give_what_the_sequence_gives(Be, channels, N, groups, dtype):
    T = 12
    p = _inputs(T, Be, channels, N, groups, dtype, done=0.15)
    want, left = _want(p, False)
    state, start = p["s0"].clone(), None
    for t in range(T):
        y = _like(p["x"][t])
        ppo.ppo_selective_scan_step(p["x"][t], p["dt"][t], p["A"], p["B"][t], p["C"][t], state, y, p["D"], p["z"][t], p["bias"], True, start)
        start = p["done"][t]
        plain.within(y, want[t], f"y {t}")
    live = start == 0
    plain.within(state[live], left[live], "state")


def test_a_decision_without_what_may_be_left_out():
    p = _inputs(1, 5, 40, 16, 1, torch.bfloat16)
    q = {**p, "D": None, "z": None, "bias": None, "done": None}
    state, y = p["s0"].clone(), _like(p["x"][0])
    ppo.ppo_selective_scan_step(p["x"][0], p["dt"][0], p["A"], p["B"][0], p["C"][0], state, y)
    want, left = _want(q, False)
    plain.within(y, want[0])
    plain.within(state, left)


def test_sequences_chain_through_their_states():
    p = _inputs(700, 1, 48, 16, 1, torch.float32)
    want, left = _want(p, False)
    state, at = p["s0"], 0
    for n in (1, 15, 100, 584):
        q = {k: v[at:at + n] if k in ("x", "dt", "B", "C", "z", "done", "dy") else v for k, v in p.items()}
        y, state = _fwd({**q, "s0": state})
        plain.within(y, want[at:at + n], "y")
        at += n
    plain.within(state, left, "state")


def test_gradients_of_parameters_are_added_or_left_out():
    p = _inputs(40, 5, 72, 16, 1, torch.float32)
    grads = _bwd(p)
    was = {n: torch.randn_like(grads[n]) for n in ("dA", "dD", "ddt_bias")}
    out = _bwd(p, {n: v.clone() for n, v in was.items()}, accumulate=True)
    for n, v in was.items():
        assert float((out[n] - v - grads[n]).abs().max()) <= 2.0 ** -22 * float(out[n].abs().max() + grads[n].abs().max())
    for gone in (("dA",), ("dD", "ddt_bias"), ("dA", "dD", "ddt_bias", "dstate")):
        out = _bwd(p, {n: None for n in gone})
        assert all(torch.equal(out[n], grads[n]) for n in GRADS if n not in gone)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("T,dtype", [(16, torch.float32), (16, torch.bfloat16), (300, torch.float32), (2000, torch.bfloat16)])
def test_a_value_that_is_no_number_stays_between_flags_and_on_its_channel(T, dtype, bad):
    p = _inputs(T, 2, 40, 16, 1, dtype, done=0.0)
    p["done"][3, 1] = p["done"][9, 1] = 1
    y0, s0 = _fwd(p)
    g0 = _bwd(p)
    q = {**p, "x": p["x"].clone()}
    q["x"][6, 1, 5] = bad
    y1, s1 = _fwd(q)
    same = torch.ones_like(y0, dtype=torch.bool)
    same[6:10, 1, 5] = False
    assert torch.equal(y0[same], y1[same]) and torch.equal(s0, s1) and not torch.isfinite(y1[6:10, 1, 5]).any()
    q = {**p, "dy": p["dy"].clone()}
    q["dy"][6, 1, 5] = bad  # reaches back to step 4
    g1 = _bwd(q)
    same[:] = True
    same[4:7, 1, 5] = False
    for n in ("dx", "ddt", "dz"):
        assert torch.equal(g0[n][same], g1[n][same]), n
    assert torch.equal(g0["dstate"], g1["dstate"]) and not torch.isfinite(g1["dx"][4:7, 1, 5]).any()
    rows = torch.ones(T, 2, dtype=torch.bool, device=DEV)
    rows[4:7, 1] = False
    for n in ("dB", "dC"):
        assert torch.equal(g0[n][rows], g1[n][rows]), n


def test_a_state_that_is_no_number_goes_no_further_than_the_first_flag():
    p = _inputs(20, 2, 40, 16, 1, torch.float32, done=0.0)
    p["done"][5, 0] = 1
    y0, s0 = _fwd(p)
    g0 = _bwd(p)
    q = {**p, "s0": p["s0"].clone()}
    q["s0"][0, 7, 3] = float("nan")
    y1, s1 = _fwd(q)
    same = torch.ones_like(y0, dtype=torch.bool)
    same[:6, 0, 7] = False
    assert torch.equal(y0[same], y1[same]) and torch.equal(s0, s1)
    q = {**p, "ds": p["ds"].clone()}
    q["ds"][0, 7, 3] = float("nan")
    g1 = _bwd(q)
    same[:] = True
    same[6:, 0, 7] = False
    assert torch.equal(g0["dx"][same], g1["dx"][same]) and torch.equal(g0["dstate"], g1["dstate"])


@pytest.mark.parametrize("T,Be", [(5, 3), (18, 2), (300, 1)])
def test_decays_of_any_size(T, Be):
    """Elements that forget everything at once (A of minus infinity), next to those that forget nothing (A of 0), as -1e30 and 0 do."""
    p = _inputs(T, Be, 40, 16, 1, torch.float32)
    p["A"][:, 3], p["A"][:, 7] = -1e30, 0.0
    _check(p)
    y, s1 = _fwd(p)
    q = {**p, "A": p["A"].clone()}
    q["A"][:, 3] = float("-inf")
    y2, s2 = _fwd(q)
    assert torch.equal(y, y2) and torch.equal(s1, s2)
    a, b = _bwd(p), _bwd(q)
    for n in ("dx", "dB", "dC", "dz", "dstate"):
        assert torch.equal(a[n], b[n]), n
    state = p["s0"].clone()
    out = _like(p["x"][0])
    ppo.ppo_selective_scan_step(p["x"][0], p["dt"][0], q["A"], p["B"][0], p["C"][0], state, out, p["D"], p["z"][0], p["bias"])
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(state).all())


def test_a_last_flag_leaves_zeros_whatever_was_there():
    for T in (1, 3, 17, 300):
        p = _inputs(T, 2, 40, 16, 1, torch.float32, done=0.0)
        p["done"][T - 1] = 1
        p["A"] = p["A"].clone()
        p["A"][5, 2] = float("nan")
        y, s1 = _fwd(p)
        assert not s1.any() and bool(torch.isnan(y[:, :, 5]).all())
        assert bool(torch.isfinite(y[:, :, torch.arange(40, device=DEV) != 5]).all())
