"""The causal convolution, the selective scan and the norms with rotation as programs use them: first calls of a process inside a capture and on two
streams at once, graphs that are replayed on new inputs, rows so far apart that offsets pass 32 bits."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32

CHILD = """
import sys, torch
from paper_2509_16434_b200 import binding as ppo
def problem(seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    h = lambda *s: n(*s).bfloat16()
    p = dict(w=n(72, 4), b=n(72), A=-torch.exp(n(72, 16)), D=n(72), x=h(900, 1, 72), dt=h(900, 1, 72), B=h(900, 1, 1, 16), C=h(900, 1, 1, 16), z=h(900, 1, 72),
             dy=h(900, 1, 72), s=n(1, 72, 16), q=h(400, 4, 64), k=h(400, 2, 64), gq=n(64), gk=n(64), pos=torch.arange(400, device="cuda", dtype=torch.int32),
             freq=torch.rand(16, generator=g, device="cuda", dtype=torch.float64), dq=h(400, 4, 64), dk=h(400, 2, 64))
    e = lambda t: torch.zeros_like(t)
    p["out"] = [e(p["x"]), e(p["x"]), e(p["w"]), e(p["b"]), e(p["x"]), e(p["s"]), e(p["x"]), e(p["x"]), e(p["A"]), e(p["B"]), e(p["C"]), e(p["D"]), e(p["x"]), e(p["b"]),
                e(p["s"]), e(p["q"]), e(p["k"]), e(p["q"]), e(p["k"]), e(p["gq"]), e(p["gk"]), p["s"].clone(), e(p["x"][0])]
    b = lambda m: torch.zeros(max(m, 32), dtype=torch.uint8, device="cuda")
    p["ws"] = [b(ppo.ppo_causal_conv_workspace_bytes(p["x"], 4))] + [b(ppo.ppo_selective_scan_workspace_bytes(p["x"], p["B"], w)) for w in (False, True)] + [
        b(ppo.ppo_qk_norm_rotate_workspace_bytes(p["q"], p["k"]))]
    return p
def calls(p):
    o, ws = p["out"], p["ws"]
    ppo.ppo_causal_conv_fwd(p["x"], p["w"], p["b"], o[0], act="silu")
    ppo.ppo_causal_conv_bwd(p["x"], p["w"], p["b"], p["dy"], o[1], o[2], o[3], act="silu", workspace=ws[0])
    ppo.ppo_selective_scan_fwd(p["x"], p["dt"], p["A"], p["B"], p["C"], o[4], p["D"], p["z"], p["b"], state_in=p["s"], state_out=o[5], workspace=ws[1])
    ppo.ppo_selective_scan_bwd(p["x"], p["dt"], p["A"], p["B"], p["C"], p["dy"], o[6], o[7], o[8], o[9], o[10], p["D"], p["z"], p["b"], state_in=p["s"], dD=o[11],
                               dz=o[12], ddt_bias=o[13], dstate_in=o[14], workspace=ws[2])
    ppo.ppo_qk_norm_rotate_fwd(p["q"], p["k"], p["gq"], p["gk"], p["pos"], p["freq"], o[15], o[16])
    ppo.ppo_qk_norm_rotate_bwd(p["q"], p["k"], p["gq"], p["gk"], p["pos"], p["freq"], p["dq"], p["dk"], o[17], o[18], o[19], o[20], workspace=ws[3])
    o[21].copy_(p["s"])
    ppo.ppo_selective_scan_step(p["x"][0], p["dt"][0], p["A"], p["B"][0], p["C"][0], o[21], o[22], p["D"], p["z"][0], p["b"])
a, b = problem(1), problem(2)
torch.cuda.synchronize()
if sys.argv[1] == "capture":
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls(a)
    g.replay()
    calls(b)
    c = problem(3)  # the graph on other inputs
    calls(c)
    old = {k: v.clone() for k, v in a.items() if torch.is_tensor(v)}
    for k in old:
        a[k].copy_(c[k])
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c["out"], a["out"]))
    for k in old:
        a[k].copy_(old[k])
    g.replay()
else:
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for p, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                calls(p)
torch.cuda.synchronize()
for seed, p in ((1, a), (2, b)):
    w = problem(seed)
    calls(w)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(w["out"], p["out"])) and all(bool(torch.isfinite(x).all()) and bool(x.any()) for x in p["out"])
assert ppo.ppo_poll_status() == 0
print("ok")
"""


@pytest.mark.parametrize("how", ["capture", "streams"])
def test_first_calls_of_a_process(how):
    run = subprocess.run([sys.executable, "-c", CHILD, how], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout + run.stderr[-2000:]


def _far(like, lead, total=5 << 29):
    """Places for tensors shaped as those of `like`, side by side in rows that are 16-byte aligned and `total` elements in all apart."""
    rows = 1
    for n in like[0].shape[:lead]:
        rows *= n
    width = (total // rows + 63) // 64 * 64
    assert rows * width > 1 << 31
    flat, at, out = torch.empty((rows, width), dtype=like[0].dtype, device=DEV), 0, []
    for t in like:
        n = t.numel() // rows
        out.append(flat[:, at:at + n].view(t.shape))
        at += (n + 63) // 64 * 64
    assert at <= width
    return out


def _same(run, near, lead, outs):
    """run(*inputs, *outputs) gives the same bits with its rows far apart."""
    want = run(*near, *(torch.empty_like(t) for t in outs))
    far, to = _far(near, lead), _far(outs, lead)
    for a, b in zip(far, near):
        a.copy_(b)
    assert all(torch.equal(a, b) for a, b in zip(run(*far, *to), want))
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("T,Be,dtype", [(3, 2, BF16), (40, 2, BF16), (100, 1, F32)])
def test_convolution_of_far_rows(T, Be, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    w, b, s0 = n(64, 4), n(64), n(Be, 3, 64).to(dtype)

    def run(x, dy, y, dx):
        s1, dw, db = torch.empty_like(s0), torch.empty_like(w), torch.empty_like(b)
        ppo.ppo_causal_conv_fwd(x, w, b, y, None, s0, s1, "silu")
        ppo.ppo_causal_conv_bwd(x, w, b, dy, dx, dw, db, None, s0, s0, None, "silu", workspace=torch.empty(ppo.ppo_causal_conv_workspace_bytes(x, 4), dtype=torch.uint8, device=DEV))
        return [t.contiguous() for t in (y, s1, dx, dw, db)]
    near = [n(T, Be, 64).to(dtype) for _ in range(2)]
    _same(run, near, 2, near)


@pytest.mark.parametrize("T,Be,dtype", [(10, 2, BF16), (40, 3, BF16), (300, 1, BF16), (70, 2, F32)])
def test_scan_of_far_rows(T, Be, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    C, N = 64, 16
    A, D, s0 = -torch.exp(n(C, N)), n(C), n(Be, C, N)

    def run(x, dt, z, dy, B, Cm, y, dx, ddt, dz, dB, dC):
        ws = [torch.empty(ppo.ppo_selective_scan_workspace_bytes(x, B, b), dtype=torch.uint8, device=DEV) for b in (False, True)]
        s1, ds, dA = torch.empty_like(s0), torch.empty_like(s0), torch.empty_like(A)
        ppo.ppo_selective_scan_fwd(x, dt, A, B, Cm, y, D, z, None, True, None, s0, s1, ws[0] if ws[0].numel() else None)
        ppo.ppo_selective_scan_bwd(x, dt, A, B, Cm, dy, dx, ddt, dA, dB, dC, D, z, None, True, None, s0, s0, None, dz, None, ds, workspace=ws[1])
        return [t.contiguous() for t in (y, s1, dx, ddt, dA, dB, dC, dz, ds)]
    wide, few = [n(T, Be, C).to(dtype) for _ in range(4)], [n(T, Be, 1, N).to(dtype) for _ in range(2)]
    _same(run, wide + few, 2, [wide[0]] * 4 + few)


@pytest.mark.parametrize("rows,d,dtype", [(4, 64, BF16), (300, 128, BF16), (70, 50, F32)])
def test_norms_of_far_rows(rows, d, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(0)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    gq, gk, pos = n(d), n(d), torch.arange(rows, device=DEV, dtype=torch.int32)
    freq = torch.rand(d // 4, generator=g, device=DEV, dtype=torch.float64)

    def run(q, k, dqo, dko, qo, ko, dq, dk):
        a, b = torch.empty_like(gq), torch.empty_like(gk)
        ppo.ppo_qk_norm_rotate_fwd(q, k, gq, gk, pos, freq, qo, ko)
        ppo.ppo_qk_norm_rotate_bwd(q, k, gq, gk, pos, freq, dqo, dko, dq, dk, a, b,
                                   workspace=torch.empty(ppo.ppo_qk_norm_rotate_workspace_bytes(q, k), dtype=torch.uint8, device=DEV))
        return [t.contiguous() for t in (qo, ko, dq, dk, a, b)]
    near = [n(rows, h, d).to(dtype) for h in (4, 2, 4, 2)]
    _same(run, near, 1, near)
