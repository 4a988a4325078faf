"""Group norm with activation on the GPU against 64 bits, element by element.

Tolerances, u = 2^-24.  Statistics of n values: at most 2 + log2 n + n / 256 roundings of partial sums on any path, of values of
size |x| (mean), |x - mean|^2 (variance).  xhat then carries the mean's error times rstd and half the variance's relative
error; an activation's derivative is at most 1.1, and its own arithmetic a few u.  Outputs of 16 bits: half a step of the type."""
import pytest
import torch

import plain_operators as plain
from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _inputs(B, HW, C, dtype, seed=0, level=0.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x = (n(B, HW, C) * (0.5 + torch.rand(C, generator=g, device=DEV)) + n(C) + level).to(dtype)
    return x, 1 + 0.3 * n(C), 0.3 * n(C), n(B, HW, C).to(dtype)


def _roundings(n):
    return 4 + n.bit_length() + n / 256


def _below(got, want, tol):
    assert got.shape == want.shape and not torch.isnan(got).any()
    off = (got.double() - want).abs() - tol
    assert float(off.max()) <= 0, float(off.max())


def _fwd(x, groups, gamma, beta, act, eps=1e-5, y=None):
    y = torch.full_like(x, float("nan")) if y is None else y
    mean, rstd = (torch.full((x.shape[0], groups), float("nan"), device=DEV) for _ in range(2))
    need = ppo.ppo_group_norm_workspace_bytes(x, groups, False)
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV) if need else None
    ppo.ppo_group_norm_fwd(x, groups, gamma, beta, y, mean, rstd, act, eps, ws)
    return y, mean, rstd


def _check_fwd(x, groups, gamma, beta, act, got, eps=1e-5):
    (y, mean, rstd), (yw, mw, rw) = got, plain.group_norm(x, groups, gamma, beta, act, eps)
    B, HW, C = x.shape
    per = C // groups
    k = _roundings(HW * per)
    size = x.double().abs().reshape(B, HW, groups, per).mean((1, 3))
    tol_mean = (k * size + mw.abs()) * U
    _below(mean, mw, tol_mean)
    # the variance about a mean that is off by d is d^2 too large; its root is relative
    tol_rstd = rw * ((k + 8) * U + 0.5 * (tol_mean * rw) ** 2)
    _below(rstd, rw, tol_rstd)
    wide = lambda s: s.repeat_interleave(per, 1)[:, None]  # noqa: E731
    a = (torch.ones(C, device=DEV) if gamma is None else gamma).double().abs()
    b = torch.zeros(C, device=DEV).double() if beta is None else beta.double().abs()
    xhat = (x.double() - wide(mw)).abs() * wide(rw)
    tol = a * (wide(tol_mean) * wide(rw) + xhat * wide(tol_rstd / rw) + 4 * U * (xhat + wide(mw.abs() * rw))) + 8 * U * (a * xhat + b)
    _below(y, yw, 1.1 * tol + 8 * U * yw.abs() + (torch.finfo(x.dtype).eps / 2) * (yw.abs() + tol) + (2.0 ** -25 if x.dtype == torch.float16 else 0))


def _bwd(x, groups, gamma, beta, mean, rstd, dy, act, dx=None, into=None):
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    C = x.shape[2]
    dg, db = into if into is not None else (torch.full((C,), float("nan"), device=DEV) for _ in range(2))
    ws = torch.full((ppo.ppo_group_norm_workspace_bytes(x, groups, True),), 0xA5, dtype=torch.uint8, device=DEV)
    ppo.ppo_group_norm_bwd(x, groups, gamma, beta, mean, rstd, dy, dx, dg, db, act, into is not None, ws)
    return dx, dg, db


def _check_bwd(x, groups, gamma, beta, mean, rstd, dy, act, got):
    dx, dg, db, size, sg, sb = plain.group_norm_grad(x, groups, gamma, beta, mean, rstd, dy, act)
    B, HW, C = x.shape
    per = C // groups
    wide = lambda s: s.double().repeat_interleave(per, 1)[:, None]  # noqa: E731
    k = _roundings(HW * per)
    # xhat: one subtraction of values of size |x| and |mean|; SiLU's derivative moves by at most half of what z moves
    a = (torch.ones(C, device=DEV) if gamma is None else gamma).double().abs()
    b = torch.zeros(C, device=DEV).double() if beta is None else beta.double().abs()
    dxhat = 2 * U * wide(rstd) * (x.double().abs() + wide(mean).abs())
    dz = dy.double().abs() * ((0.5 * (a * dxhat + 4 * U * b) + 12 * U) if act == "silu" else 4 * U)
    over = lambda t: t.reshape(B, HW, groups, per).mean((1, 3)).repeat_interleave(per, 1)[:, None]  # noqa: E731
    h = (x.double() - wide(mean)).abs() * wide(rstd)
    g = a * dy.double().abs() * 1.1
    tol = wide(rstd) * (a * dz + over(a * dz) + h * over(a * dz * h + g * dxhat) + dxhat * over(g * h)) + (k + 10) * U * size
    _below(got[0], dx, tol + torch.finfo(x.dtype).eps / 2 * (dx.abs() + tol) + (2.0 ** -25 if x.dtype == torch.float16 else 0))
    n = _roundings(HW) + 4
    _below(got[1], dg, (dz * h + 1.1 * dy.double().abs() * dxhat).sum((0, 1)) + n * U * sg + U * dg.abs())
    _below(got[2], db, dz.sum((0, 1)) + n * U * sb + U * db.abs())


SHAPES = [(1, 1, 1, 1), (1, 1, 8, 2), (3, 1, 64, 4), (5, 1, 1024, 16), (2, 1, 96, 1), (2, 7, 6, 3), (3, 33, 24, 8), (2, 100, 64, 8), (3, 713, 96, 3),
          (2, 1200, 64, 8), (1, 4800, 32, 4), (2, 5000, 10, 5), (1, 19200, 16, 2), (2, 3000, 256, 32), (1, 1001, 513, 27), (300, 4, 32, 32), (4097, 1, 16, 2),
          (700, 56, 24, 1), (50, 20, 240, 2), (3, 9, 512, 2), (2, 18309, 96, 4), (1, 40000, 128, 32), (40, 3000, 64, 16)]


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_values_and_gradients(shape, dtype, act):
    B, HW, C, groups = shape
    x, gamma, beta, dy = _inputs(B, HW, C, dtype)
    y, mean, rstd = _fwd(x, groups, gamma, beta, act)
    _check_fwd(x, groups, gamma, beta, act, (y, mean, rstd))
    got = _bwd(x, groups, gamma, beta, mean, rstd, dy, act)
    _check_bwd(x, groups, gamma, beta, mean, rstd, dy, act, got)
    assert all(torch.equal(a, b) for a, b in zip(got, _bwd(x, groups, gamma, beta, mean, rstd, dy, act)))
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape,ld,at", [((3, 50, 48, 6), 64, 8), ((2, 40, 30, 3), 37, 5), ((6, 1, 64, 4), 200, 64), ((1, 2000, 64, 8), 96, 16)])
def test_pixels_that_are_parts_of_wider_rows(shape, ld, at, dtype):
    B, HW, C, groups = shape
    x, gamma, beta, dy = _inputs(B, HW, C, dtype)
    wide = torch.full((B, HW, ld), float("nan"), dtype=dtype, device=DEV)
    part = wide[:, :, at:at + C]
    part.copy_(x)
    into = torch.full((B, HW, ld + 3), 7.0, dtype=dtype, device=DEV)
    y, mean, rstd = _fwd(part, groups, gamma, beta, "silu", y=into[:, :, 1:1 + C])
    _check_fwd(x, groups, gamma, beta, "silu", (y, mean, rstd))
    assert bool((into[:, :, 0] == 7).all()) and bool((into[:, :, 1 + C:] == 7).all())
    dwide = torch.full((B, HW, ld), 7.0, dtype=dtype, device=DEV)
    got = _bwd(part, groups, gamma, beta, mean, rstd, dy, "silu", dx=dwide[:, :, at:at + C])
    _check_bwd(x, groups, gamma, beta, mean, rstd, dy, "silu", got)
    assert bool((dwide[:, :, :at] == 7).all()) and bool((dwide[:, :, at + C:] == 7).all())


@pytest.mark.parametrize("shape", [(3, 1, 64, 4), (2, 300, 32, 4), (2, 6000, 64, 8)])
def test_without_scale_and_shift_in_place_and_added_to(shape):
    B, HW, C, groups = shape
    x, gamma, beta, dy = _inputs(B, HW, C, torch.bfloat16)
    y, mean, rstd = _fwd(x, groups, None, None, "relu")
    _check_fwd(x, groups, None, None, "relu", (y, mean, rstd))
    _check_bwd(x, groups, None, None, mean, rstd, dy, "relu", _bwd(x, groups, None, None, mean, rstd, dy, "relu"))
    same = x.clone()
    _fwd(same, groups, None, None, "relu", y=same)
    assert torch.equal(same, y)
    want = _bwd(x, groups, gamma, beta, mean, rstd, dy, "silu")
    into = (torch.full((C,), 2.0, device=DEV), torch.full((C,), -3.0, device=DEV))
    got = _bwd(x, groups, gamma, beta, mean, rstd, dy, "silu", into=into)
    for a, b, start in zip(got[1:], want[1:], (2.0, -3.0)):
        assert torch.allclose(a, b + start, rtol=4 * U, atol=4 * U * (b.abs().max().item() + 3))
    over = dy.clone()
    ppo.ppo_group_norm_bwd(x, groups, gamma, beta, mean, rstd, over, over, act="silu", workspace=torch.empty(
        ppo.ppo_group_norm_workspace_bytes(x, groups, True), dtype=torch.uint8, device=DEV))
    assert torch.equal(over, want[0])


def test_values_far_from_zero_and_constant_groups():
    """A mean a thousand deviations away loses three digits of x itself, none of the deviations; a group of one value gives beta."""
    for shape in ((2, 1, 256, 4), (3, 500, 32, 4), (1, 9000, 64, 8)):
        B, HW, C, groups = shape
        x, gamma, beta, _ = _inputs(B, HW, C, torch.float32, level=1000.0)
        _check_fwd(x, groups, gamma, beta, "none", _fwd(x, groups, gamma, beta, "none"))
        y, mean, rstd = _fwd(torch.full_like(x, 3.0), groups, gamma, beta, "none")
        assert torch.equal(y, beta.expand_as(y)) and bool((mean == 3).all()) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=4 * U)


def test_nan_stays_in_its_group():
    for shape in ((4, 1, 64, 4), (3, 500, 32, 4), (2, 9000, 64, 8)):
        B, HW, C, groups = shape
        x, gamma, beta, dy = _inputs(B, HW, C, torch.bfloat16)
        y, mean, rstd = _fwd(x, groups, gamma, beta, "silu")
        bad = x.clone()
        bad[1, HW // 2, 0] = float("nan")
        yb, mb, rb = _fwd(bad, groups, gamma, beta, "silu")
        hit = torch.zeros(B, 1, C, dtype=torch.bool, device=DEV)
        hit[1, :, :C // groups] = True
        assert bool(torch.isnan(yb[hit.expand_as(yb)]).all()) and torch.equal(yb[~hit.expand_as(yb)], y[~hit.expand_as(y)])


@pytest.mark.parametrize("shape", [(4, 1200, 64, 8), (2, 20000, 64, 8), (9, 1, 64, 4), (3, 50, 30, 5)])
def test_other_streams_and_captured_calls(shape):
    B, HW, C, groups = shape
    x, gamma, beta, dy = _inputs(B, HW, C, torch.bfloat16)
    y, mean, rstd = _fwd(x, groups, gamma, beta, "relu")
    want = _bwd(x, groups, gamma, beta, mean, rstd, dy, "relu")
    out = [torch.empty_like(t) for t in (y, mean, rstd, *want)]
    n = [ppo.ppo_group_norm_workspace_bytes(x, groups, b) for b in (False, True)]
    ws = torch.empty(max(n), dtype=torch.uint8, device=DEV)
    call = lambda: (ppo.ppo_group_norm_fwd(x, groups, gamma, beta, *out[:3], act="relu", workspace=ws),  # noqa: E731
                    ppo.ppo_group_norm_bwd(x, groups, gamma, beta, mean, rstd, dy, *out[3:], act="relu", workspace=ws))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, (y, mean, rstd, *want)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for t in out:
        t.fill_(7)
    ws.fill_(0x5A)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, (y, mean, rstd, *want)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(70, 1, 768, 32), (9, 2, 48, 2), (33, 5, 72, 3), (5, 3, 320, 8), (700, 1, 60, 5), (12, 7, 168, 7)])
def test_groups_whose_vectors_are_no_power_of_two(shape, dtype):
    B, HW, C, groups = shape
    x, gamma, beta, dy = _inputs(B, HW, C, dtype, seed=9)
    y, mean, rstd = _fwd(x, groups, gamma, beta, "silu")
    _check_fwd(x, groups, gamma, beta, "silu", (y, mean, rstd))
    _check_bwd(x, groups, gamma, beta, mean, rstd, dy, "silu", _bwd(x, groups, gamma, beta, mean, rstd, dy, "silu"))


def test_more_groups_than_a_grid_has_rows():
    # 17 pixels of one vector: a warp each, eight a block, more than 65535 blocks
    B, HW, C, groups = 1, 17, 8 * 524289, 524289
    x, gamma, beta, dy = _inputs(B, HW, C, torch.bfloat16, seed=8)
    y, mean, rstd = _fwd(x, groups, gamma, beta, "relu")
    _check_fwd(x, groups, gamma, beta, "relu", (y, mean, rstd))
    _check_bwd(x, groups, gamma, beta, mean, rstd, dy, "relu", _bwd(x, groups, gamma, beta, mean, rstd, dy, "relu"))
