"""Decay attention on the GPU against the recurrence in 64 bits, element by element.

Tolerances.  An output is a sum of terms; `size` is the sum of their absolute values.  In 32 bits a term passes at most two
roundings per step of the recurrence, one per addition of the inner product, a few scales, and where products of chunks are
taken their accumulation, which we allow two units for each of the same additions: off by at most
(4 T + 2 d + 16) 2^-24 size.  Powers of the decay (one exp2 of a product n log2 lambda, at most 128 or a segment's length) add
2^-23 (4 + |n log2 lambda|) of terms that are themselves lambda^n: below 8 2^-23 of them.  bf16 adds half a step, 2^-8 relative,
for the output and for each operand that is rounded: the weights of pairs of steps and the states (their terms are
different ones, so once over all), and 2^-17 for weighted keys in two terms: (2 * 2^-8 + 2^-16) size.  A state that is handed out
is built from three terms: below 2^-24."""
import pytest
import torch

import plain_operators as plain
from paper_2509_16434_b200 import binding as ppo

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def _near(got, want, size, steps, d, dtype):
    u = (4 * min(steps, 4096) + 2 * d + 16 + 16) * 2.0 ** -24 + (0 if dtype == F32 else 2 * 2.0 ** -8 + 2.0 ** -16)
    assert got.shape == want.shape
    off = (got.double() - want).abs() - u * size
    assert not torch.isnan(got).any()
    assert float(off.max()) <= 1e-30, (float(off.max()), float((got.double() - want).norm() / want.norm()))


class Case:
    def __init__(self, T, Be, heads, kv, dk, dv, dtype, done=0.0, state=True, seed=0, pack=False, offset=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        n = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.T, self.Be, self.heads, self.kv, self.dk, self.dv, self.dtype = T, Be, heads, kv, dk, dv, dtype
        if pack:  # parts of one projection's rows, at odd places where offset says so
            width = heads * dk + kv * (dk + dv) + offset
            rows = n(T, Be, width).to(dtype)
            at, parts = offset, []
            for h, d in ((heads, dk), (kv, dk), (kv, dv)):
                parts.append(rows[:, :, at:at + h * d].unflatten(2, (h, d)))
                at += h * d
            self.q, self.k, self.v = parts
        else:
            self.q, self.k, self.v = (n(T, Be, h, d).to(dtype) for h, d in ((heads, dk), (kv, dk), (kv, dv)))
        self.do = n(T, Be, heads, dv).to(dtype)
        self.lam = 1 - torch.exp2(-torch.linspace(0, 9, heads, device=DEV))  # the first is 0
        if heads > 1:
            self.lam[-1] = 1.0
        self.done = (torch.rand(T, Be, generator=g, device=DEV) < done).to(torch.uint8) if done else None
        self.s0 = n(Be, heads, dk, dv) if state else None
        self.ds = n(Be, heads, dk, dv) if state else None
        self.scale = dk ** -0.5

    def args(self):
        return self.q, self.k, self.v, self.lam, self.done, self.s0, self.scale

    def workspace(self, backward):
        need = ppo.ppo_decay_attention_workspace_bytes(self.q, self.k, self.v, backward)
        return torch.full((need,), 0xA5, dtype=torch.uint8, device=DEV) if need else None  # junk

    def fwd(self, o=None, s=None, workspace=None):
        o = torch.full((self.T, self.Be, self.heads, self.dv), float("nan"), dtype=self.dtype, device=DEV) if o is None else o
        s = torch.full((self.Be, self.heads, self.dk, self.dv), float("nan"), device=DEV) if s is None else s
        ppo.ppo_decay_attention_fwd(self.q, self.k, self.v, self.lam, o, self.done, self.s0, s, self.scale,
                                    self.workspace(False) if workspace is None else workspace)
        return o, s

    def grads(self):
        def like(x):  # strided as x, in a storage of its own
            return torch.full((x.untyped_storage().nbytes() // x.element_size(),), float("nan"), dtype=x.dtype, device=DEV).as_strided(
                x.shape, x.stride(), x.storage_offset())
        return [like(x) for x in (self.q, self.k, self.v)] + [torch.full((self.Be, self.heads, self.dk, self.dv), float("nan"), device=DEV)]

    def bwd(self, out=None, workspace=None):
        out = self.grads() if out is None else out
        ppo.ppo_decay_attention_bwd(self.q, self.k, self.v, self.lam, self.do, *out[:3], self.done, self.s0, self.ds, out[3], self.scale,
                                    self.workspace(True) if workspace is None else workspace)
        return out


SHAPES = [
    # T, Be, heads, kv, dk, dv, done
    (1, 1, 1, 1, 1, 1, 0.0), (1, 3, 4, 2, 64, 64, 0.5), (2, 2, 2, 1, 5, 7, 0.3), (15, 3, 4, 4, 16, 24, 0.1), (16, 5, 16, 16, 64, 64, 0.05),
    (17, 2, 6, 3, 48, 80, 0.2), (33, 1, 2, 2, 128, 128, 0.0), (63, 2, 4, 1, 33, 100, 0.05), (64, 2, 2, 2, 64, 64, 0.03), (65, 2, 2, 1, 128, 64, 0.03),
    (130, 3, 4, 2, 64, 128, 0.02), (200, 1, 3, 3, 72, 56, 1.0), (513, 1, 2, 1, 64, 64, 0.0), (700, 1, 4, 2, 40, 128, 0.004), (1100, 2, 2, 2, 128, 128, 0.002),
]


@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_outputs_and_states(shape, dtype, state):
    c = Case(*shape[:6], dtype, shape[6], state)
    (o, s), (ow, sw), (oa, sa) = c.fwd(), plain.attention(*c.args()), plain.attention_abs(*c.args())
    _near(o, ow, oa, c.T, c.dk, dtype)
    _near(s, sw, sa, c.T, c.dk, F32)
    o2 = torch.empty_like(o)  # without a state handed out
    ppo.ppo_decay_attention_fwd(c.q, c.k, c.v, c.lam, o2, c.done, c.s0, None, c.scale, c.workspace(False))
    _near(o2, ow, oa, c.T, c.dk, dtype)
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_gradients(shape, dtype, state):
    c = Case(*shape[:6], dtype, shape[6], state)
    got = c.bwd()
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    for i in range(3):
        _near(got[i], want[i], size[i], c.T, max(c.dk, c.dv) * (c.heads // c.kv), dtype)
    _near(got[3], want[3], size[3], c.T, c.dk, F32)
    assert all(torch.equal(a, b) for a, b in zip(got, c.bwd()))  # the same bits again
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1500, 5, 16, 4, 64, 64, 0.002), (900, 9, 8, 8, 128, 128, 0.002), (700, 6, 16, 4, 64, 128, 0.0), (650, 7, 8, 8, 104, 48, 0.01)],
                         ids=lambda s: "-".join(map(str, s)))
def test_many_blocks_of_many_chunks(shape, dtype):
    """Blocks that share an SM and run at different speeds, several chunks each."""
    c = Case(*shape[:6], dtype, shape[6])
    (o, s), (ow, sw), (oa, sa) = c.fwd(), plain.attention(*c.args()), plain.attention_abs(*c.args())
    _near(o, ow, oa, c.T, c.dk, dtype)
    _near(s, sw, sa, c.T, c.dk, F32)
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    first = c.bwd()
    for i in range(3):
        _near(first[i], want[i], size[i], c.T, max(c.dk, c.dv) * (c.heads // c.kv), dtype)
    _near(first[3], want[3], size[3], c.T, c.dk, F32)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, c.bwd()))
        assert all(torch.equal(a, b) for a, b in zip((o, s), c.fwd()))
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("shape", [(500, 40, 8, 8, 64, 64, 0.004), (400, 38, 8, 4, 48, 128, 0.004), (330, 20, 16, 16, 128, 64, 0.0)], ids=lambda s: "-".join(map(str, s)))
def test_states_of_many_heads_over_several_chunks(shape):
    """Heads enough that no sequence is cut: the state that is left is built in the pass that writes the outputs."""
    c = Case(*shape[:6], BF16, shape[6])
    assert ppo.ppo_decay_attention_workspace_bytes(c.q, c.k, c.v, False) == 0
    (o, s), (ow, sw), (oa, sa) = c.fwd(), plain.attention(*c.args()), plain.attention_abs(*c.args())
    _near(o, ow, oa, c.T, c.dk, BF16)
    _near(s, sw, sa, c.T, c.dk, F32)
    got, again = c.bwd(), c.bwd()
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    for i in range(3):
        _near(got[i], want[i], size[i], c.T, max(c.dk, c.dv) * (c.heads // c.kv), BF16)
    _near(got[3], want[3], size[3], c.T, c.dk, F32)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert ppo.ppo_poll_status() == 0


@pytest.mark.parametrize("offset", [0, 8, 3])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_that_are_parts_of_wider_ones(dtype, offset):
    c = Case(90, 2, 4, 2, 32, 64, dtype, 0.05, pack=True, offset=offset)
    wide = torch.full((c.T, c.Be, c.heads * c.dv + 5), 7.0, dtype=dtype, device=DEV)
    o, s = c.fwd(wide[:, :, 5:].unflatten(2, (c.heads, c.dv)))
    (ow, sw), (oa, sa) = plain.attention(*c.args()), plain.attention_abs(*c.args())
    _near(o, ow, oa, c.T, c.dk, dtype)
    _near(s, sw, sa, c.T, c.dk, F32)
    assert bool((wide[:, :, :5] == 7).all())
    got = c.bwd()
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    for i in range(3):
        _near(got[i], want[i], size[i], c.T, max(c.dk, c.dv) * 2, dtype)
    # what lies between the rows' parts stays as it was
    whole = torch.as_strided(got[0], (c.T * c.Be, c.q.stride(1)), (c.q.stride(1), 1), 0)
    first = c.q.storage_offset()
    rest = torch.cat([whole[:, :first], whole[:, first + c.heads * c.dk:]], 1)
    assert bool(torch.isnan(rest).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [3, 100, 600])
def test_state_in_place_and_sequences_cut_in_two(T, dtype):
    c = Case(T, 2, 4, 2, 64, 32, dtype, 0.02)
    o, s = c.fwd()
    cut, state, parts = T // 3, c.s0.clone(), []
    for a, b in ((0, cut), (cut, T)):
        part = torch.empty_like(o[a:b])
        done = c.done[a:b].contiguous()
        need = ppo.ppo_decay_attention_workspace_bytes(c.q[a:b], c.k[a:b], c.v[a:b], False)
        ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
        ppo.ppo_decay_attention_fwd(c.q[a:b], c.k[a:b], c.v[a:b], c.lam, part, done, state, state, c.scale, ws)
        parts.append(part)
    (ow, sw), (oa, sa) = plain.attention(*c.args()), plain.attention_abs(*c.args())
    _near(torch.cat(parts), ow, oa, T, c.dk, dtype)
    _near(state, sw, sa, T, c.dk, F32)
    g = c.grads()
    g[3].copy_(c.ds)
    ppo.ppo_decay_attention_bwd(c.q, c.k, c.v, c.lam, c.do, *g[:3], c.done, c.s0, g[3], g[3], c.scale, c.workspace(True))
    assert all(torch.equal(a, b) for a, b in zip(g, c.bwd()))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("Be,heads,kv,dk,dv", [(1, 1, 1, 1, 1), (3, 4, 2, 64, 64), (5, 8, 2, 128, 128), (2, 3, 1, 33, 50), (7, 2, 2, 100, 7), (4, 4, 4, 16, 128)])
def test_single_steps_are_the_sequence(Be, heads, kv, dk, dv, dtype):
    T = 9
    c = Case(T, Be, heads, kv, dk, dv, dtype, 0.3)
    state, start, o = c.s0.clone(), None, torch.empty((T, Be, heads, dv), dtype=dtype, device=DEV)
    for t in range(T):
        ppo.ppo_decay_attention_step(c.q[t], c.k[t], c.v[t], c.lam, state, o[t], start, c.scale)
        start = c.done[t].contiguous()
        state[start.bool()] = float("nan")  # whatever a started env's rows hold
    (ow, sw), (oa, sa) = plain.attention(*c.args()), plain.attention_abs(*c.args())
    _near(o, ow, oa, T, dk, dtype)
    live = ~start.bool()
    _near(state[live], sw[live], sa[live], T, dk, F32)


def test_what_no_step_reaches_changes_nothing():
    """Rows of other envs hold NaN."""
    for dtype in (F32, BF16):
        c = Case(70, 3, 2, 2, 64, 64, dtype, 0.0)
        c.done = torch.zeros(70, 3, dtype=torch.uint8, device=DEV)
        c.done[40] = 1
        want, s_want = c.fwd()
        got_b = c.bwd()
        d = Case(70, 3, 2, 2, 64, 64, dtype, 0.0)
        d.done = c.done
        for x in (d.q, d.k, d.v, d.do):
            x[:, 1] = float("nan")
        o, s = d.fwd()
        assert torch.equal(o[:, [0, 2]], want[:, [0, 2]]) and torch.equal(s[[0, 2]], s_want[[0, 2]])
        for a, b in zip(d.bwd()[:3], got_b[:3]):
            assert torch.equal(a[:, [0, 2]], b[:, [0, 2]])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 40), (24, 104), (5, 7)])
def test_later_steps_and_those_before_a_reset_reach_nothing(dk, dv, dtype, bad):
    """Infinities and NaN at some steps: outputs in front of them and behind the next reset are those of finite numbers there."""
    T = 200
    c = Case(T, 2, 4, 2, dk, dv, dtype, 0.0)
    c.done = torch.zeros(T, 2, dtype=torch.uint8, device=DEV)
    c.done[[20, 70, 71, 150]] = 1
    for x in (c.q, c.k, c.v, c.do):
        x[60:66] = 1.0
        x[110:112] = -1.0
    (ow, sw), (oa, sa) = plain.attention(*c.args()), plain.attention_abs(*c.args())
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    for x in (c.q, c.k, c.v, c.do):
        x[60:66], x[110:112] = bad, bad
    o, s = c.fwd()
    back = c.bwd()
    # what sees the bad steps: outputs and dq from them on to the next reset, dk and dv from them back to the last one
    after = [t for t in range(T) if not (60 <= t <= 70 or 110 <= t <= 150)]
    front = [t for t in range(T) if not (21 <= t < 66 or 72 <= t < 112)]
    _near(o[after], ow[after], oa[after], T, dk, dtype)
    _near(s, sw, sa, T, dk, F32)
    _near(back[0][after], want[0][after], size[0][after], T, dv, dtype)
    for i in (1, 2):
        _near(back[i][front], want[i][front], size[i][front], T, 2 * max(dk, dv), dtype)
    _near(back[3], want[3], size[3], T, dk, F32)
    assert not bool(torch.isfinite(o[62].float()).any()) and not bool(torch.isfinite(back[1][62].float()).any())


def test_many_heads_of_many_envs():
    """More states than a grid has rows, and offsets of the states that pass 32 bits."""
    Be, heads, dk, dv = 5000, 16, 16, 16
    c = Case(2, Be, heads, heads, dk, dv, BF16, 0.2)
    o, s = c.fwd()
    at = torch.tensor([0, 1, 4095, 4096, 4999], device=DEV)
    sub = lambda x, dim: None if x is None else x.index_select(dim, at)  # noqa: E731
    args = sub(c.q, 1), sub(c.k, 1), sub(c.v, 1), c.lam, sub(c.done, 1), sub(c.s0, 0), c.scale
    (ow, sw), (oa, sa) = plain.attention(*args), plain.attention_abs(*args)
    _near(sub(o, 1), ow, oa, 2, dk, BF16)
    _near(sub(s, 0), sw, sa, 2, dk, F32)
    Be, heads = 16500, 8  # 132 000 states of 64 KB: 8.6 GB
    state = torch.ones((Be, heads, 128, 128), device=DEV)
    one = torch.ones((Be, heads, 128), dtype=BF16, device=DEV)
    o = torch.empty_like(one)
    lam = torch.full((heads,), 0.5, device=DEV)
    ppo.ppo_decay_attention_step(one, one, one, lam, state, o)
    assert bool((state == 1.5).all()) and bool((o == 192.0).all())


def test_other_streams_and_captured_calls():
    c, side = Case(600, 1, 4, 2, 64, 64, BF16, 0.01), torch.cuda.Stream()
    want, want_b = c.fwd(), c.bwd()
    ws, wsb = c.workspace(False), c.workspace(True)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got, got_b = c.fwd(workspace=ws), c.bwd(workspace=wsb)
    side.synchronize()
    o, s = torch.empty_like(want[0]), torch.empty_like(want[1])
    out = [torch.empty_like(x) for x in want_b]
    state, q = c.s0.clone(), c.q[0].clone()
    one = torch.empty_like(o[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.fwd(o, s, ws)
        c.bwd(out, wsb)
        ppo.ppo_decay_attention_step(q, c.k[0], c.v[0], c.lam, state, one, None, c.scale)
    ws.fill_(0x5A), wsb.fill_(0x5A)
    state.copy_(c.s0)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    for a, b in zip([*got, *got_b, o, s, *out], [*want, *want_b, *want, *want_b]):
        assert torch.equal(a, b)
    again = c.s0.clone()
    for _ in range(2):
        ppo.ppo_decay_attention_step(q, c.k[0], c.v[0], c.lam, again, one, None, c.scale)
    assert torch.equal(state, again)
    assert ppo.ppo_poll_status() == 0
