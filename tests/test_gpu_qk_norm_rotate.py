"""Norms of queries and keys with rotation on the GPU against 64 bits, element by element, within running error bounds."""
import pytest
import torch

import memory_operators as plain
from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
EPS = 1e-6


def _inputs(rows, heads, kv, d, pairs, dtype, seed=0, far=100000):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    return dict(q=(n(rows, heads, d) * (0.2 + 3 * torch.rand(heads, 1, generator=g, device=DEV))).to(dtype), k=n(rows, kv, d).to(dtype), gq=1 + 0.3 * n(d),
                gk=1 + 0.3 * n(d), pos=torch.randint(0, far, (rows,), generator=g, device=DEV, dtype=torch.int32),
                freq=10000.0 ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / max(pairs, 1)), dqo=n(rows, heads, d).to(dtype), dko=n(rows, kv, d).to(dtype))


def _fwd(p, interleaved, qo=None, ko=None, eps=EPS):
    qo, ko = torch.full_like(p["q"], float("nan")) if qo is None else qo, torch.full_like(p["k"], float("nan")) if ko is None else ko
    ppo.ppo_qk_norm_rotate_fwd(p["q"], p["k"], p["gq"], p["gk"], p["pos"], p["freq"], qo, ko, eps, interleaved)
    return qo, ko


def _bwd(p, interleaved, dq=None, dk=None, into=None, eps=EPS):
    dq, dk = torch.full_like(p["q"], float("nan")) if dq is None else dq, torch.full_like(p["k"], float("nan")) if dk is None else dk
    gq, gk = into or (torch.full((p["q"].shape[2],), float("nan"), device=DEV) for _ in range(2))
    ws = torch.full((ppo.ppo_qk_norm_rotate_workspace_bytes(p["q"], p["k"]),), 0xFF, dtype=torch.uint8, device=DEV)
    ppo.ppo_qk_norm_rotate_bwd(p["q"], p["k"], p["gq"], p["gk"], p["pos"], p["freq"], p["dqo"], p["dko"], dq, dk, gq, gk, eps, interleaved, into is not None, ws)
    return dq, dk, gq, gk


def _check(p, interleaved, eps=EPS):
    qo, ko = _fwd(p, interleaved, eps=eps)
    plain.within(qo, plain.qk(p["q"], p["gq"], eps, p["pos"], p["freq"], interleaved), "q")
    plain.within(ko, plain.qk(p["k"], p["gk"], eps, p["pos"], p["freq"], interleaved), "k")
    got = _bwd(p, interleaved, eps=eps)
    for n, i in (("q", 0), ("k", 1)):
        dx, dgamma = plain.qk(p[n], p["g" + n], eps, p["pos"], p["freq"], interleaved, p["d" + n + "o"])
        plain.within(got[i], dx, "d" + n)
        plain.within(got[2 + i], dgamma, "dgamma " + n)
    assert all(torch.equal(a, b) for a, b in zip(got, _bwd(p, interleaved, eps=eps)))
    assert ppo.ppo_poll_status() == 0


SHAPES = [(1, 1, 1, 1, 0), (1, 16, 4, 128, 64), (3, 2, 1, 2, 1), (5, 4, 2, 64, 32), (7, 3, 3, 80, 40), (9, 5, 1, 96, 24), (2, 40, 8, 128, 32), (33, 1, 1, 256, 128),
          (4, 2, 2, 255, 127), (6, 4, 4, 50, 9), (11, 2, 2, 64, 0), (700, 4, 1, 32, 16), (3000, 8, 2, 64, 16), (40, 6, 2, 112, 56), (5, 7, 3, 16, 8), (64, 2, 2, 200, 8)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_values_and_gradients(shape, dtype, interleaved):
    _check(_inputs(*shape, dtype), interleaved)


@pytest.mark.parametrize("dtype", TYPES)
def test_positions_from_the_lowest_to_the_highest(dtype):
    p = _inputs(8, 4, 2, 64, 32, dtype)
    p["pos"] = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, 123456789, -77], dtype=torch.int32, device=DEV)
    _check(p, False)
    _check(p, True)


def test_without_gamma_or_rotation():
    p = _inputs(20, 4, 2, 64, 32, torch.bfloat16)
    _check({**p, "gq": None}, False)
    _check({**p, "gk": None}, False)
    q = {**p, "gq": None, "gk": None, "pos": None, "freq": None}
    for a, n in zip(_fwd(q, False), "qk"):
        plain.within(a, plain.qk(p[n], None, EPS, None, None, False))
    for a, n in zip(_bwd(q, False), "qk"):
        plain.within(a, plain.qk(p[n], None, EPS, None, None, False, p["d" + n + "o"])[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_heads_of_zeros_and_of_tiny_values(dtype):
    p = _inputs(6, 4, 2, 64, 32, dtype)
    p["q"][2, 1] = 0
    p["k"][3] = 0
    p["q"][4, 2] *= 1e-3
    _check(p, False, eps=1e-3)
    assert not _fwd(p, False)[0][2, 1].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,at,gap", [(64, 0, 0), (64, 8, 8), (64, 3, 2), (50, 0, 0), (96, 16, 0)])
def test_one_row_of_queries_keys_and_values_side_by_side(d, at, gap, dtype):
    """As a projection leaves them; outputs in place, gradients in place."""
    rows, heads, kv = 40, 4, 2
    p = _inputs(rows, heads, kv, d, d // 4, dtype)
    want, grads = _fwd(p, False), _bwd(p, False)
    width = at + (heads + 2 * kv) * d + gap

    def wide(q, k):
        row = torch.full((rows, width), float("nan"), dtype=dtype, device=DEV)
        parts = row[:, at:at + heads * d].unflatten(1, (heads, d)), \
            row[:, at + heads * d:at + (heads + kv) * d].unflatten(1, (kv, d))
        parts[0].copy_(q), parts[1].copy_(k)
        return row, parts
    row, (q, k) = wide(p["q"], p["k"])
    _fwd({**p, "q": q, "k": k}, False, q, k)
    aligned = at % 8 == 0 and width % 8 == 0
    if aligned and d % 16 == 0:
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    else:  # element by element: the sum of squares in another order, which the bound counts whatever the order
        for a, n in ((q, "q"), (k, "k")):
            plain.within(a.contiguous(), plain.qk(p[n], p["g" + n], EPS, p["pos"], p["freq"], False))
    assert bool(torch.isnan(row[:, :at]).all()) and bool(torch.isnan(row[:, at + (heads + kv) * d:]).all())
    drow, (dq, dk) = wide(p["dqo"], p["dko"])
    _, (q, k) = wide(p["q"], p["k"])
    got = _bwd({**p, "q": q, "k": k, "dqo": dq, "dko": dk}, False, dq, dk)
    for n, i in (("q", 0), ("k", 1)):
        dx, dgamma = plain.qk(p[n], p["g" + n], EPS, p["pos"], p["freq"], False, p["d" + n + "o"])
        plain.within(got[i].contiguous(), dx)
        plain.within(got[2 + i], dgamma)
        assert not (aligned and d % 16 == 0) or torch.equal(got[i], grads[i])
    assert bool(torch.isnan(drow[:, :at]).all()) and bool(torch.isnan(drow[:, at + (heads + kv) * d:]).all())


def test_gradients_of_gamma_are_added_or_left_out():
    p = _inputs(100, 4, 2, 64, 32, torch.float32)
    dq, dk, gq, gk = _bwd(p, False)
    was = torch.randn_like(gq), torch.randn_like(gk)
    _, _, aq, ak = _bwd(p, False, into=(was[0].clone(), was[1].clone()))
    for a, w, v in ((aq, was[0], gq), (ak, was[1], gk)):
        assert float((a - w - v).abs().max()) <= 2.0 ** -22 * float(a.abs().max() + v.abs().max())
    for keep_q, keep_k in ((True, False), (False, True), (False, False)):
        a, b, x, y = torch.full_like(p["q"], 9.0), torch.full_like(p["k"], 9.0), torch.zeros_like(gq), torch.zeros_like(gk)
        ws = torch.empty(ppo.ppo_qk_norm_rotate_workspace_bytes(p["q"], p["k"]), dtype=torch.uint8, device=DEV) if keep_q or keep_k else None
        ppo.ppo_qk_norm_rotate_bwd(p["q"], p["k"], p["gq"], p["gk"], p["pos"], p["freq"], p["dqo"], p["dko"], a, b, x if keep_q else None,
                                   y if keep_k else None, EPS, False, False, ws)
        assert torch.equal(a, dq) and torch.equal(b, dk)
        assert torch.equal(x, gq if keep_q else 0 * gq) and torch.equal(y, gk if keep_k else 0 * gk)


@pytest.mark.parametrize("d", [64, 50])
def test_a_value_that_is_no_number_stays_in_its_head(d):
    p = _inputs(10, 4, 2, d, d // 2, torch.bfloat16)
    q0, k0 = _fwd(p, False)
    g0 = _bwd(p, False)
    p["q"] = p["q"].clone()
    p["q"][3, 1, 5] = float("nan")
    q1, k1 = _fwd(p, False)
    same = torch.ones_like(q0, dtype=torch.bool)
    same[3, 1] = False
    assert torch.equal(q0[same], q1[same]) and torch.equal(k0, k1) and bool(torch.isnan(q1[3, 1]).all())
    g1 = _bwd(p, False)
    assert torch.equal(g0[0][same], g1[0][same]) and torch.equal(g0[1], g1[1]) and torch.equal(g0[3], g1[3])


def test_a_row_gives_the_same_bits_alone_and_among_others():
    for dtype, d in ((torch.bfloat16, 128), (torch.float32, 72)):
        p = _inputs(500, 12, 4, d, d // 2, dtype)
        qo, ko = _fwd(p, False)
        for r in (0, 77, 499):
            one = {n: v[r:r + 1] if n in ("q", "k", "pos") else v for n, v in p.items()}
            a, b = _fwd(one, False)
            assert torch.equal(a[0], qo[r]) and torch.equal(b[0], ko[r])
