"""The 64-bit forms of the causal convolution, the selective scan and the norms with rotation against automatic differentiation,
differences and closed cases; and what the library refuses before it launches anything."""
import ctypes as C

import pytest
import torch

import memory_operators as plain
from paper_2509_16434_b200 import binding as ppo


def _normal(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64)


def _slopes(value, leaves, grads, g):
    """Gradients against differences along a random direction."""
    for i, x in enumerate(leaves):
        d, h = _normal(g, *x.shape), 1e-6
        at = lambda f: value(*[y + f * d if j == i else y for j, y in enumerate(leaves)])  # noqa: E731
        slope = (at(h) - at(-h)) / (2 * h)
        assert abs(slope - (grads[i] * d).sum()) <= 2e-6 * (1 + abs(slope)), i


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("T", [1, 2, 7])
@pytest.mark.parametrize("W", [2, 4, 8])
def test_convolution_and_its_gradients(T, W, act):
    g = torch.Generator().manual_seed(1)
    Be, n = 3, 5
    x, w, b, s0 = _normal(g, T, Be, n), _normal(g, n, W), _normal(g, n), _normal(g, Be, W - 1, n)
    done = (torch.rand(T, Be, generator=g) < 0.25).to(torch.uint8)
    dy, ds = _normal(g, T, Be, n), _normal(g, Be, W - 1, n)

    def value(x, w, b, s0):  # a window that a flag empties
        window, total = list(s0.unbind(1)), 0
        for t in range(T):
            window = window + [x[t]]
            s = b + sum(v * w[:, i] for i, v in enumerate(window))
            y = s * torch.sigmoid(s) if act == "silu" else s.clamp(min=0) if act == "relu" else s
            total = total + (y * dy[t]).sum()
            window = [v * (1 - done[t].double())[:, None] for v in window[1:]]
        return total + (torch.stack(window, 1) * ds).sum()

    y, left = plain.conv(x, w, b, done, s0, act)
    leaves = [v.clone().requires_grad_() for v in (x, w, b, s0)]
    total = value(*leaves)
    assert abs(total.detach() - (y.v * dy).sum() - (left * ds).sum()) < 1e-11
    want = torch.autograd.grad(total, leaves)
    got = [v.v for v in plain.conv(x, w, b, done, s0, act, dy, ds)]
    for a, v in zip(got, want):
        assert torch.allclose(a, v, rtol=1e-12, atol=1e-12)
    _slopes(value, (x, w, b, s0), got, g)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("softplus", [False, True])
def test_scan_and_its_gradients(softplus, gate):
    g = torch.Generator().manual_seed(2)
    T, Be, n, groups, N = 6, 2, 6, 2, 3
    v = dict(x=_normal(g, T, Be, n), dt=0.4 * _normal(g, T, Be, n), A=-_normal(g, n, N).abs(), B=_normal(g, T, Be, groups, N),
             C=_normal(g, T, Be, groups, N), D=_normal(g, n), z=_normal(g, T, Be, n) if gate else None, bias=0.3 * _normal(g, n))
    names = [k for k in v if v[k] is not None]
    done = (torch.rand(T, Be, generator=g) < 0.3).to(torch.uint8)
    s0, dy, ds = _normal(g, Be, n, N), _normal(g, T, Be, n), _normal(g, Be, n, N)

    def value(*leaves):
        m, h = dict(zip(names, leaves)), leaves[-1]
        total = 0
        for t in range(T):
            d = m["dt"][t] + m["bias"]
            d = torch.log1p(torch.exp(d)) if softplus else d
            b, c = (m[k][t].repeat_interleave(n // groups, 1) for k in "BC")
            h = torch.exp(d[..., None] * m["A"]) * h + (d * m["x"][t])[..., None] * b
            y = (h * c).sum(2) + m["D"] * m["x"][t]
            if gate:
                y = y * m["z"][t] * torch.sigmoid(m["z"][t])
            total = total + (y * dy[t]).sum()
            h = h * (1 - done[t].double())[:, None, None]
        return total + (h * ds).sum()

    args = (v["x"], v["dt"], v["A"], v["B"], v["C"], v["D"], v["z"], v["bias"], softplus, done, s0)
    y, left = plain.scan(*args)
    leaves = [v[k].clone().requires_grad_() for k in names] + [s0.clone().requires_grad_()]
    total = value(*leaves)
    assert abs(total.detach() - (y.v * dy).sum() - (left.v * ds).sum()) < 1e-11
    want = torch.autograd.grad(total, leaves)
    got = plain.scan(*args, dy, ds)
    got = [got["d" + ("dt_bias" if k == "bias" else k)].v for k in names] + [got["dstate"].v]
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-11, atol=1e-12)
    _slopes(value, [v[k] for k in names] + [s0], got, g)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,pairs", [(8, 4), (10, 3), (6, 0)])
def test_norm_with_rotation_and_its_gradients(d, pairs, interleaved):
    g = torch.Generator().manual_seed(3)
    rows, heads, eps = 5, 2, 1e-3
    x, gamma, dy = _normal(g, rows, heads, d), _normal(g, d), _normal(g, rows, heads, d)
    pos = torch.tensor([0, 1, 7, -3, 100000], dtype=torch.int32)
    freq = 0.5 ** torch.arange(pairs, dtype=torch.float64)

    def value(x, gamma):
        n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gamma
        out = list(n.unbind(-1))
        for j in range(pairs):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
            angle = (pos.double() * freq[j])[:, None]
            out[a], out[b] = n[..., a] * angle.cos() - n[..., b] * angle.sin(), n[..., a] * angle.sin() + n[..., b] * angle.cos()
        return (torch.stack(out, -1) * dy).sum()

    leaves = [x.clone().requires_grad_(), gamma.clone().requires_grad_()]
    total = value(*leaves)
    assert abs(total.detach() - (plain.qk(x, gamma, eps, pos, freq, interleaved).v * dy).sum()) < 1e-11
    want = torch.autograd.grad(total, leaves)
    got = [n.v for n in plain.qk(x, gamma, eps, pos, freq, interleaved, dy)]
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-11, atol=1e-12)
    _slopes(value, (x, gamma), got, g)


def test_rotation_keeps_inner_products_at_equal_distances():
    g = torch.Generator().manual_seed(4)
    q, k = _normal(g, 1, 1, 16).expand(9, 1, 16), _normal(g, 1, 1, 16).expand(9, 1, 16)
    freq = 0.3 ** torch.arange(8, dtype=torch.float64)
    pos = torch.arange(9, dtype=torch.int32) * 1000
    for interleaved in (False, True):
        a = plain.qk(q, None, 0.0, pos + 5, freq, interleaved).v
        b = plain.qk(k, None, 0.0, pos, freq, interleaved).v
        dots = (a * b).sum((1, 2))
        assert float((dots - dots[0]).abs().max()) < 1e-9


# ---- refusals: found on the host; the addresses are never read ----

P = 1 << 20  # stands for an aligned device address
OK, INVALID, SHAPE, ALIGN, UNSUPPORTED = 0, 1, 2, 3, 7


def _conv_call(call, p=None, acc=0, ws=P, ws_bytes=1 << 40, **d):
    f = dict(T=1 if call == "step" else 10, Be=2, C=64, width=4, act=2, dtype=1, ldx=64, ldy=64)
    f.update(d)
    a = dict(x=P, w=P, b=P, done=P, s0=P, y=P, s1=P, dy=P, ds1=P, dx=P, ds0=P, dw=P, db=P)
    a.update(p or {})
    desc = ppo.CausalConvDesc(*[f[n] for n, _ in ppo.CausalConvDesc._fields_])
    L = ppo.lib()
    if call == "fwd":
        return L.ppo_causal_conv_fwd(C.byref(desc), *[a[n] for n in ("x", "w", "b", "done", "s0", "y", "s1")], None)
    if call == "step":
        return L.ppo_causal_conv_step(C.byref(desc), *[a[n] for n in ("x", "w", "b", "done", "s1", "y")], None)
    return L.ppo_causal_conv_bwd(C.byref(desc), *[a[n] for n in ("x", "w", "b", "done", "s0", "dy", "ds1", "dx", "ds0", "dw", "db")], acc, ws, ws_bytes, None)


@pytest.mark.parametrize("call", ["fwd", "bwd", "step"])
def test_convolution_refusals(call):
    for bad in (dict(T=0), dict(Be=0), dict(C=-1), dict(act=3), dict(act=-1), dict(dtype=3)):
        assert _conv_call(call, **bad) == INVALID, bad
    for bad in (dict(ldx=63), dict(ldy=0)):
        assert _conv_call(call, **bad) == SHAPE, bad
    for bad in (dict(width=1), dict(width=9), dict(T=1 << 20, Be=1 << 12)):
        assert _conv_call(call, **bad) == UNSUPPORTED, bad
    for name in {"fwd": ("x", "w", "y"), "bwd": ("x", "w", "dy", "dx"), "step": ("x", "w", "s1", "y")}[call]:
        assert _conv_call(call, {name: None}) == INVALID, name
    for name in {"fwd": ("x", "y", "s0", "s1"), "bwd": ("x", "dy", "dx", "s0", "ds0", "ds1"), "step": ("x", "s1", "y")}[call]:
        assert _conv_call(call, {name: P + 1}) == ALIGN, name
    for name in ("w", "b") + (("dw", "db") if call == "bwd" else ()):
        assert _conv_call(call, {name: P + 2}) == ALIGN, name
    if call == "step":
        assert _conv_call(call, T=2) == SHAPE
    if call == "bwd":
        assert _conv_call(call, ws=None) == INVALID and _conv_call(call, ws=P + 16) == ALIGN and _conv_call(call, ws_bytes=0) == SHAPE


def _scan_call(call, p=None, ws=P, ws_bytes=1 << 50, **d):
    f = dict(T=1 if call == "step" else 10, Be=2, channels=64, N=16, groups=2, dtype=1, softplus=1, ldx=64, lddt=64, ldb=32, ldc=32, ldz=64, ldy=64)
    f.update(d)
    a = {n: P for n in ("x", "dt", "A", "B", "C", "D", "z", "bias", "done", "s0", "y", "s1", "dy", "ds1", "dx", "ddt", "dA", "dB", "dC", "dD", "dz", "dbias", "ds0")}
    a.update(p or {})
    desc = ppo.SelectiveScanDesc(*[f[n] for n, _ in ppo.SelectiveScanDesc._fields_])
    L, ins = ppo.lib(), [a[n] for n in ("x", "dt", "A", "B", "C", "D", "z", "bias", "done")]
    if call == "fwd":
        return L.ppo_selective_scan_fwd(C.byref(desc), *ins, a["s0"], a["y"], a["s1"], ws, ws_bytes, None)
    if call == "step":
        return L.ppo_selective_scan_step(C.byref(desc), *ins, a["s1"], a["y"], None)
    outs = [a[n] for n in ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "dbias", "ds0")]
    return L.ppo_selective_scan_bwd(C.byref(desc), *ins, a["s0"], a["dy"], a["ds1"], *outs, 0, ws, ws_bytes, None)


@pytest.mark.parametrize("call", ["fwd", "bwd", "step"])
def test_scan_refusals(call):
    for bad in (dict(T=0), dict(Be=0), dict(channels=0), dict(N=0), dict(groups=0), dict(dtype=3), dict(dtype=-1)):
        assert _scan_call(call, **bad) == INVALID, bad
    for bad in (dict(groups=3, ldb=48, ldc=48), dict(ldx=63), dict(lddt=63), dict(ldz=63), dict(ldy=63), dict(ldb=31), dict(ldc=31)):
        assert _scan_call(call, **bad) == SHAPE, bad
    for bad in (dict(N=65, ldb=130, ldc=130), dict(T=1 << 20, Be=1 << 12), dict(Be=1 << 24)):
        assert _scan_call(call, **bad) == UNSUPPORTED, bad
    for name in ("x", "dt", "A", "B", "C") + {"fwd": ("y",), "bwd": ("dy", "dx", "ddt", "dB", "dC"), "step": ("y", "s1")}[call]:
        assert _scan_call(call, {name: None}) == INVALID, name
    for name in ("x", "dt", "B", "C", "z") + {"fwd": ("y",), "bwd": ("dy", "dx", "ddt", "dB", "dC", "dz"), "step": ("y",)}[call]:
        assert _scan_call(call, {name: P + 1}) == ALIGN, name
    for name in ("A", "D", "bias") + (("dA", "dD", "dbias") if call == "bwd" else ()):
        assert _scan_call(call, {name: P + 2}) == ALIGN, name
    for name in {"fwd": ("s0", "s1"), "bwd": ("s0", "ds0", "ds1"), "step": ("s1",)}[call]:
        assert _scan_call(call, {name: P + 4}) == ALIGN, name
    if call == "step":
        assert _scan_call(call, T=2) == SHAPE
    if call == "bwd":
        assert _scan_call(call, {"z": None}) == INVALID and _scan_call(call, {"dz": None}) == INVALID
        assert _scan_call(call, ws=None) == INVALID and _scan_call(call, ws=P + 16) == ALIGN and _scan_call(call, ws_bytes=0) == SHAPE
    if call == "fwd":  # one long sequence is cut
        one = dict(T=8192, Be=1)
        assert _scan_call(call, ws=P + 16, **one) == ALIGN


def _qk_call(call, p=None, eps=1e-6, ws=P, ws_bytes=1 << 40, **d):
    f = dict(rows=10, heads=4, kv_heads=2, d=64, pairs=32, interleaved=0, dtype=1, ldq=256, ldk=128, ldqo=256, ldko=128)
    f.update(d)
    a = {n: P + 4096 * i for i, n in enumerate(("q", "k", "gq", "gk", "pos", "freq", "qo", "ko", "dqo", "dko", "dq", "dk", "dgq", "dgk"))}
    a.update(p or {})
    desc = ppo.QkNormDesc(*[f[n] for n, _ in ppo.QkNormDesc._fields_])
    L, ins = ppo.lib(), [a[n] for n in ("q", "k", "gq", "gk", "pos", "freq")]
    if call == "fwd":
        return L.ppo_qk_norm_rotate_fwd(C.byref(desc), eps, *ins, a["qo"], a["ko"], None)
    return L.ppo_qk_norm_rotate_bwd(C.byref(desc), eps, *ins, *[a[n] for n in ("dqo", "dko", "dq", "dk", "dgq", "dgk")], 0, ws, ws_bytes, None)


@pytest.mark.parametrize("call", ["fwd", "bwd"])
def test_norm_with_rotation_refusals(call):
    for bad in (dict(rows=0), dict(heads=0), dict(kv_heads=0), dict(d=0), dict(pairs=-1), dict(dtype=3), dict(eps=-1.0), dict(eps=float("nan"))):
        assert _qk_call(call, **bad) == INVALID, bad
    for bad in (dict(pairs=33), dict(ldq=255), dict(ldk=127), dict(ldqo=255), dict(ldko=127)):
        assert _qk_call(call, **bad) == SHAPE, bad
    assert _qk_call(call, d=257, ldq=4096, ldk=4096, ldqo=4096, ldko=4096) == UNSUPPORTED
    for name in ("q", "k", "pos", "freq") + {"fwd": ("qo", "ko"), "bwd": ("dqo", "dko", "dq", "dk")}[call]:
        assert _qk_call(call, {name: None}) == INVALID, name
    for name in ("q", "k") + {"fwd": ("qo", "ko"), "bwd": ("dqo", "dko", "dq", "dk")}[call]:
        assert _qk_call(call, {name: P + 1}) == ALIGN, name
    for name in ("gq", "gk", "pos", "freq") + (("dgq", "dgk") if call == "bwd" else ()):
        assert _qk_call(call, {name: P + 2}) == ALIGN, name
    assert _qk_call(call, {"freq": P + 4}) == ALIGN
    into = {"fwd": (("qo", "q", "ldqo"), ("ko", "k", "ldko")), "bwd": (("dq", "dqo", "ldqo"), ("dk", "dko", "ldko"))}[call]
    for out, same, ld in into:  # in place, but in rows of another length
        assert _qk_call(call, {out: P, same: P}, **{ld: 512}) == SHAPE
    if call == "bwd":
        assert _qk_call(call, ws=None) == INVALID and _qk_call(call, ws=P + 16) == ALIGN and _qk_call(call, ws_bytes=0) == SHAPE


def test_tensors_that_do_not_fit():
    """The binding's own checks; host tensors go no further than these."""
    f = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    conv = lambda **k: ppo.ppo_causal_conv_fwd(**{**dict(x=f(3, 2, 8), weight=f(8, 4), bias=f(8), y=f(3, 2, 8)), **k})  # noqa: E731
    scan = lambda **k: ppo.ppo_selective_scan_fwd(  # noqa: E731
        **{**dict(x=f(3, 2, 8), dt=f(3, 2, 8), A=f(8, 4), B=f(3, 2, 2, 4), C_=f(3, 2, 2, 4), y=f(3, 2, 8)), **k})
    qk = lambda **k: ppo.ppo_qk_norm_rotate_fwd(  # noqa: E731
        **{**dict(q=f(5, 4, 8), k=f(5, 2, 8), gamma_q=f(8), gamma_k=f(8), pos=f(5, dtype=torch.int32), freq=f(4, dtype=torch.float64), q_out=f(5, 4, 8),
                  k_out=f(5, 2, 8)), **k})
    half = torch.bfloat16
    for call, bad, status in [
        (conv, {}, 1), (conv, dict(y=f(3, 2, 8, dtype=half)), 1), (conv, dict(act="gelu"), 1), (conv, dict(y=f(3, 2, 9)), 2), (conv, dict(weight=f(7, 4)), 2),
        (conv, dict(weight=f(4, 8).t()), 2), (conv, dict(bias=f(9)), 2), (conv, dict(state_in=f(2, 4, 8)), 2), (conv, dict(state_out=f(2, 3, 8, dtype=half)), 1),
        (conv, dict(done=f(3, 2)), 1), (conv, dict(x=f(2, 3, 8).transpose(0, 1)), 2),
        (scan, {}, 1), (scan, dict(dt=f(3, 2, 8, dtype=half)), 1), (scan, dict(A=f(8, 5)), 2), (scan, dict(A=f(4, 8).t()), 2), (scan, dict(C_=f(3, 2, 1, 4)), 2),
        (scan, dict(D=f(7)), 2), (scan, dict(z=f(3, 2, 4)), 2), (scan, dict(state_in=f(2, 8, 5)), 2), (scan, dict(state_in=f(2, 8, 4, dtype=half)), 1),
        (scan, dict(B=f(3, 2, 4, 2).transpose(2, 3)), 2),
        (qk, {}, 1), (qk, dict(k=f(5, 2, 6)), 2), (qk, dict(gamma_q=f(6)), 2), (qk, dict(pos=f(4, dtype=torch.int32)), 2),
        (qk, dict(pos=f(5, dtype=torch.int64)), 1), (qk, dict(freq=f(4)), 1), (qk, dict(k_out=f(5, 2, 8, dtype=half)), 1), (qk, dict(q=f(5, 8, 4).transpose(1, 2)), 2),
    ]:
        with pytest.raises(ppo.PpoError) as err:
            call(**bad)
        assert err.value.status == status, bad


def test_workspaces_are_those_of_the_sizes():
    x, B = torch.zeros(3, 2, 8), torch.zeros(3, 2, 2, 4)
    assert ppo.ppo_selective_scan_workspace_bytes(x, B, True) > 0 and ppo.ppo_causal_conv_workspace_bytes(x, 4) > 0
    assert ppo.ppo_qk_norm_rotate_workspace_bytes(torch.zeros(5, 4, 8), torch.zeros(5, 2, 8)) > 0
    assert ppo.ppo_causal_conv_workspace_bytes(x, 9) == 0
