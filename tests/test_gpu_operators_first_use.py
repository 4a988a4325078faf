"""First calls of a process: inside a stream capture, and by two streams at once."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys, torch
from paper_2509_16434_b200 import binding as ppo
def problem(seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    p = dict(q=n(900, 1, 4, 64).bfloat16(), k=n(900, 1, 2, 64).bfloat16(), v=n(900, 1, 2, 64).bfloat16(), lam=torch.tensor([.5, .9, .99, .999], device="cuda"),
             do=n(900, 1, 4, 64).bfloat16(), x=n(3, 700, 64).bfloat16(), dy=n(3, 700, 64).bfloat16(), big=n(1, 30000, 64).bfloat16(), gamma=n(64), beta=n(64),
             logits=n(30, 90000).bfloat16(), tokens=torch.arange(30, device="cuda", dtype=torch.int32), f32=n(50, 2, 3, 40), lam3=torch.tensor([.5, .9, .99], device="cuda"))
    e = lambda t: torch.zeros_like(t)
    p["out"] = [e(p["do"]), e(p["q"]), e(p["k"]), e(p["v"]), e(p["x"]), e(p["x"]), e(p["gamma"]), e(p["beta"]), e(p["logits"]), torch.zeros(5, device="cuda"),
                torch.zeros(30, device="cuda"), e(p["big"]), e(p["f32"]), torch.zeros(3, 8, device="cuda"), torch.zeros(3, 8, device="cuda"),
                torch.zeros(1, 8, device="cuda"), torch.zeros(1, 8, device="cuda")]
    b = lambda m: torch.zeros(max(m, 32), dtype=torch.uint8, device="cuda")
    p["ws"] = [b(ppo.ppo_decay_attention_workspace_bytes(p["q"], p["k"], p["v"], w)) for w in (False, True)] + [
        b(ppo.ppo_group_norm_workspace_bytes(p["x"], 8, True)), b(ppo.ppo_group_norm_workspace_bytes(p["big"], 8, False)), b(ppo.ppo_token_loss_workspace_bytes(p["logits"]))]
    return p
def calls(p):
    o, ws, z = p["out"], p["ws"], p["gamma"]
    ppo.ppo_decay_attention_fwd(p["q"], p["k"], p["v"], p["lam"], o[0], scale=.1, workspace=ws[0])
    ppo.ppo_decay_attention_bwd(p["q"], p["k"], p["v"], p["lam"], p["do"], o[1], o[2], o[3], scale=.1, workspace=ws[1])
    ppo.ppo_decay_attention_fwd(p["f32"], p["f32"], p["f32"], p["lam3"], o[12])
    ppo.ppo_group_norm_fwd(p["x"], 8, p["gamma"], p["beta"], o[4], o[13], o[14], act="relu")
    ppo.ppo_group_norm_bwd(p["x"], 8, p["gamma"], p["beta"], o[13], o[14], p["dy"], o[5], o[6], o[7], act="relu", workspace=ws[2])
    ppo.ppo_group_norm_fwd(p["big"], 8, p["gamma"], p["beta"], o[11], o[15], o[16], act="silu", workspace=ws[3])
    ppo.ppo_token_logp(p["logits"], p["tokens"], o[10])
    ppo.ppo_token_loss_fwd_bwd(p["logits"], p["tokens"], o[10], o[10], 30, o[8], o[9], ent_coef=.1, workspace=ws[4])
a, b = problem(1), problem(2)
torch.cuda.synchronize()
if sys.argv[1] == "capture":
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls(a)
    g.replay()
    calls(b)
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
