"""Sizes at which the memory layers run the loops and variants that real sizes run: two channels a thread, several envs or pieces a thread or block.
Each test counts from its sizes that they come to that."""
import pytest
import torch

import memory_operators as plain
import test_gpu_causal_conv as conv
import test_gpu_qk_norm_rotate as qk
import test_gpu_selective_scan as scan
from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SMS = 148


def _cdiv(a, b):
    return -(-a // b)


def _scan_plan(T, Be, channels, N, groups, dtype):
    """Segments forwards and backwards, blocks of a pass with two channels a thread, items and slices of the gradients."""
    lanes, per = 1 if N <= 16 else 2 if N <= 32 else 4, channels // groups
    tiles = groups * _cdiv(per, 64 // lanes)
    slices = max(1, (3 if dtype == torch.float32 else 4) * SMS // tiles)
    wide = Be * groups * _cdiv(per, 256 // lanes)

    def segments(n):
        n = max(1, min(n, _cdiv(T, 32), 64))
        return _cdiv(T, _cdiv(_cdiv(T, n), 16) * 16)
    back = segments(max(1, 2 * slices // Be))
    return segments(max(1, 4 * SMS // wide)), back, wide, Be * back, slices


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Be,channels,N,groups", [(16, 300, 20, 16, 1), (20, 300, 20, 12, 1), (31, 150, 20, 16, 2), (7, 300, 12, 32, 1), (18, 300, 6, 64, 1)])
def test_scans_with_two_channels_a_thread(T, Be, channels, N, groups, dtype):
    fwd, back, wide, _, _ = _scan_plan(T, Be, channels, N, groups, dtype)
    assert fwd == 1 and back == 1 and wide >= 2 * SMS and channels // groups % 2 == 0
    scan._check(scan._inputs(T, Be, channels, N, groups, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Be,channels,N,groups", [(96, 150, 20, 16, 1), (113, 75, 20, 16, 2), (90, 160, 6, 32, 1)])
def test_scans_over_segments_with_two_channels_a_thread(T, Be, channels, N, groups, dtype):
    fwd, _, wide, _, _ = _scan_plan(T, Be, channels, N, groups, dtype)
    assert fwd > 1 and wide * (fwd - 1) >= 2 * SMS and channels // groups % 2 == 0
    p = scan._inputs(T, Be, channels, N, groups, dtype)
    y, s1 = scan._fwd(p)
    want, left = scan._want(p, False)
    plain.within(y, want, "y")
    plain.within(s1, left, "state")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Be,channels,N,groups", [(16, 700, 20, 16, 1), (20, 700, 20, 16, 1), (6, 200, 200, 10, 2), (33, 1300, 3, 16, 1), (5, 700, 12, 32, 1),
                                                    (21, 650, 4, 64, 2)])
def test_gradients_of_scans_with_several_envs_a_block(T, Be, channels, N, groups, dtype):
    _, back, _, items, slices = _scan_plan(T, Be, channels, N, groups, dtype)
    assert back == 1 and items > slices
    p = scan._inputs(T, Be, channels, N, groups, dtype)
    got, want = scan._bwd(p), scan._want(p, True)
    for name in scan.GRADS:
        plain.within(got[name], want[name], name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Be,channels,N,groups", [(96, 250, 20, 16, 1), (75, 210, 13, 16, 1), (70, 70, 200, 16, 2), (65, 250, 6, 40, 1)])
def test_gradients_of_scans_with_several_segments_a_block(T, Be, channels, N, groups, dtype):
    _, back, _, items, slices = _scan_plan(T, Be, channels, N, groups, dtype)
    assert back > 1 and items > slices
    p = scan._inputs(T, Be, channels, N, groups, dtype)
    got, want = scan._bwd(p), scan._want(p, True)
    for name in scan.GRADS:
        plain.within(got[name], want[name], name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Be,channels,N,groups", [(1000, 12, 16, 1), (1777, 5, 16, 1), (900, 300, 64, 1), (950, 44, 8, 2), (1001, 12, 3, 1), (460, 40, 32, 2), (890, 7, 4, 1),
                                                  (1400, 520, 16, 2)])
def test_decisions_of_scans_with_several_envs_a_block(Be, channels, N, groups, dtype):
    lanes = 1 if N <= 4 else 2 if N <= 8 else 4 if N <= 16 else 8 if N <= 32 else 16
    cols = groups * _cdiv(channels // groups, 4 * (256 // lanes))
    assert _cdiv(Be, max(1, 3 * SMS // cols)) > 1
    T = 2
    p = scan._inputs(T, Be, channels, N, groups, dtype, done=0.3)
    want, left = scan._want(p, False)
    state, start = p["s0"].clone(), None
    for t in range(T):
        y = scan._like(p["x"][t])
        ppo.ppo_selective_scan_step(p["x"][t], p["dt"][t], p["A"], p["B"][t], p["C"][t], state, y, p["D"], p["z"][t], p["bias"], True, start)
        start = p["done"][t]
        plain.within(y, want[t], f"y {t}")
    plain.within(state[start == 0], left[start == 0], "state")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Be,C,W", [(1215, 1000, 4), (701, 333, 3), (2001, 512, 2), (1301, 520, 8)])
def test_decisions_of_the_convolution_with_several_envs_a_thread(Be, C, W, dtype):
    V = 128 // torch.finfo(dtype).bits
    cols = C // V if C % V == 0 else C
    assert cols * Be // (SMS * 256) >= 2
    p = conv._inputs(3, Be, C, W, dtype, done=0.3)
    want, left = conv._fwd(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu")
    state, start = p["s0"].clone(), None
    exact, _ = plain.conv(p["x"], p["w"], p["b"], p["done"], p["s0"], "silu")
    for t in range(3):
        y = torch.full_like(p["x"][t], float("nan"))
        ppo.ppo_causal_conv_step(p["x"][t], p["w"], p["b"], state, y, start, "silu")
        start = p["done"][t]
        assert torch.equal(y, want[t])
        plain.within(y, exact[t], f"y {t}")
    live = start == 0
    assert torch.equal(state[live], left[live])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,Be,C,W", [(3, 5000, 64, 4), (5, 320, 2048, 4), (70, 110, 2048, 2), (4, 1300, 37, 8), (40, 700, 37, 3), (2, 4800, 64, 8)])
def test_gradients_of_the_convolution_with_several_pieces_a_thread(T, Be, C, W, dtype):
    V = 64 // torch.finfo(dtype).bits
    V = V if C % V == 0 else 1
    lanes = 1
    while lanes < 32 and lanes * V < C:
        lanes *= 2
    blocks = max(1, 4 * SMS // _cdiv(C, lanes * V))
    assert Be * _cdiv(T, 32) > blocks * (128 // lanes)
    p = conv._inputs(T, Be, C, W, dtype)
    args = (p["x"], p["w"], p["b"], p["done"], p["s0"], "silu", p["dy"], p["ds"])
    for a, v, name in zip(conv._bwd(*args), plain.conv(*args), ("dx", "dw", "db", "ds0")):
        plain.within(a, v, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,kv,d,pairs", [(2000, 3, 1, 50, 9), (1300, 2, 2, 100, 50), (9000, 2, 1, 64, 16)])
def test_norms_with_several_heads_or_rows_a_warp(rows, heads, kv, d, pairs, interleaved, dtype):
    assert rows * (heads + kv) > 8 * 4 * SMS
    qk._check(qk._inputs(rows, heads, kv, d, pairs, dtype), interleaved)
