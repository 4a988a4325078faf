"""Infinities and NaN among the operands of decay attention: they reach what the recurrence lets them reach, and nothing else, at
every length, whichever operand holds them, also where the step's own done flag is set, next to it and at the borders of chunks and
of the segments that long sequences are cut into.

A bad step b of k or v reaches the outputs and dq of the steps t >= b with no flag in b .. t - 1, and the state that is left if there
is none in b .. T - 1; one of q or dO reaches dk and dv of the steps t <= b with no flag in t .. b - 1, and the gradient of the state
that came in if there is none in 0 .. b - 1.  The operand that a result is multiplied by (q for outputs, dO for dq, v for dk, k for dv)
reaches that step alone.  Everything else has to be what finite numbers give, within the bounds of the other tests of this operator.
Where a whole row is bad and the decay is 1, what it reaches is not finite."""
import pytest
import torch

import plain_operators as plain
from paper_2509_16434_b200 import binding as ppo
from test_gpu_decay_attention import BF16, DEV, F32, Case, _near

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _reached(done, bad):
    """[T, Be]: forwards and backwards, whether a bad step reaches it through the state; [Be]: both ends."""
    T, Be = done.shape
    fwd, back = torch.zeros(T, Be, dtype=torch.bool), torch.zeros(T, Be, dtype=torch.bool)
    live = torch.zeros(Be, dtype=torch.bool)
    for t in range(T):
        live = live | bad[t]
        fwd[t] = live
        live = live & ~done[t]
    left, live = live, torch.zeros(Be, dtype=torch.bool)
    for t in reversed(range(T)):
        live = (live & ~done[t]) | bad[t]
        back[t] = live
    return fwd, back, left, live


def _check(shape, dtype, done, bad, values, cut=None):
    """done, bad: bool [T, Be] on the host."""
    T, Be, heads, kv, dk, dv = shape
    c = Case(*shape, dtype)
    if cut is not None:
        assert (ppo.ppo_decay_attention_workspace_bytes(c.q, c.k, c.v, False) > 0) == cut
    c.done = done.to(torch.uint8).to(DEV)
    (ow, sw), (oa, sa) = plain.attention(*c.args()), plain.attention_abs(*c.args())
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    fwd, back, left, first = (x.to(DEV) for x in _reached(done, bad))
    own = bad.to(DEV)
    none = torch.zeros_like(own)
    share = heads // kv

    def near(got, want, size, reached, steps, d, dtype, dims):
        keep = ~reached
        if bool(keep.any()):
            _near(got[keep], want[keep], size[keep], steps, d, dtype)
        if bool(reached.any()):  # of the last head, whose decay is 1
            assert not bool(torch.isfinite(got[reached][:, -1].float()).any()), dims

    for value in values:
        for which in ("v", "k", "q", "do", "kv q do"):
            held = {n: getattr(c, n).clone() for n in ("q", "k", "v", "do")}
            through, into = "v" in which or "k" in which, "q" in which or "do" in which
            for n in held:
                if n in which:
                    getattr(c, n)[own] = value
            o, s = c.fwd()
            g = c.bwd()
            here = lambda n: own if n in which else none  # noqa: E731
            near(o, ow, oa, (fwd if through else none) | here("q"), T, dk, dtype, (which, value, "o"))
            near(g[0], want[0], size[0], (fwd if through else none) | here("do"), T, dv, dtype, (which, value, "dq"))
            near(g[1], want[1], size[1], (back if into else none) | here("v"), T, max(dk, dv) * share, dtype, (which, value, "dk"))
            near(g[2], want[2], size[2], (back if into else none) | here("k"), T, max(dk, dv) * share, dtype, (which, value, "dv"))
            near(s, sw, sa, left if through else torch.zeros_like(left), T, dk, F32, (which, value, "state"))
            near(g[3], want[3], size[3], first if into else torch.zeros_like(first), T, dk, F32, (which, value, "dstate"))
            for n, x in held.items():
                setattr(c, n, x)
    assert ppo.ppo_poll_status() == 0


def _steps(T, Be, *places):
    m = torch.zeros(T, Be, dtype=torch.bool)
    for e, at in enumerate(places[:Be]):
        m[[t for t in at if t < T], e] = True
    return m


@pytest.mark.parametrize("shape", [(2000, 8, 8, 4, 64, 64), (1500, 9, 8, 8, 128, 128), (1300, 4, 16, 8, 48, 104), (700, 4, 4, 2, 104, 64)],
                         ids=lambda s: "-".join(map(str, s)))
def test_sequences_that_are_cut(shape):
    """Bad steps in several chunks of one segment (chunks are 128 steps, segments a multiple of them), with flags at them, behind
    them and at the ends of chunks; an env that is bad throughout a chunk, and one that is not bad at all."""
    T, Be = shape[:2]
    bad = _steps(T, Be, (5, 127, 128, 300, 301, 511, 640), (130, 260, 390), (), range(256, 384))
    done = _steps(T, Be, (5, 127, 130, 300, 305, 511, 650), (131, 259, 260, 400), (17, 127, 255, 600), (383,))
    for e in range(4, Be):
        bad[e::97, e] = True
        done[3 * e::89, e] = True
    _check(shape, BF16, done, bad, (NAN, INF), cut=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 4, 4, 2, 64, 64), (2, 4, 2, 2, 16, 128), (9, 5, 4, 2, 64, 64), (16, 5, 4, 4, 128, 48), (17, 5, 4, 2, 64, 128), (50, 6, 4, 2, 104, 64),
                                   (64, 6, 2, 1, 64, 64), (65, 6, 4, 2, 64, 64), (200, 6, 4, 2, 128, 128), (50, 6, 4, 2, 7, 33)], ids=lambda s: "-".join(map(str, s)))
def test_sequences_of_one_piece(shape, dtype):
    """Envs whose bad steps carry a flag, lie in front of one or behind one, the first and the last step among them."""
    T, Be = shape[:2]
    last = T - 1
    bad = _steps(T, Be, (0, 7, 40), (1, 6, 15, 63), (), (last,), (8, 16, 33, 64, 127), (0, 3, last))
    done = _steps(T, Be, (0, 7, 40), (2, 6, 16, 63), (3, 11, 48), (last, 5), (9, 15, 16, 34, 64, 128), (2, last))
    _check(shape, dtype, done, bad, (NAN, INF, -INF), cut=False)


@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shape", [(1, 4, 4, 2, 64, 64), (9, 4, 4, 2, 64, 64), (50, 4, 4, 2, 104, 64), (200, 4, 4, 2, 128, 128), (700, 4, 4, 2, 64, 128), (50, 4, 4, 2, 7, 33)],
                         ids=lambda s: "-".join(map(str, s)))
def test_states_that_come_in(shape, dtype, value):
    """A bad state that comes in reaches the steps up to the first flag, the gradient of the one that is left those behind the last."""
    T, Be = shape[:2]
    c = Case(*shape, dtype)
    done = _steps(T, Be, (T // 2,), (0, T - 1), (T // 3, T // 2 + 1))  # none for the last env
    c.done = done.to(torch.uint8).to(DEV)
    (ow, sw), (oa, sa) = plain.attention(*c.args()), plain.attention_abs(*c.args())
    want, size = (f(*c.args(), c.do, c.ds) for f in (plain.attention, plain.attention_abs))
    fwd = (done.cumsum(0) - done.long() == 0).to(DEV)
    back = (done.flip(0).cumsum(0).flip(0) == 0).to(DEV)
    free = ~done.any(0).to(DEV)
    c.s0.fill_(value), c.ds.fill_(value)
    o, s = c.fwd()
    g = c.bwd()
    d = max(c.dk, c.dv) * 2
    for got, ref, span, reached, type_ in ((o, ow, oa, fwd, dtype), (g[0], want[0], size[0], fwd, dtype), (g[1], want[1], size[1], back, dtype),
                                           (g[2], want[2], size[2], back, dtype), (s, sw, sa, free, F32), (g[3], want[3], size[3], free, F32)):
        if bool((~reached).any()):
            _near(got[~reached], ref[~reached], span[~reached], T, d, type_)
        assert not bool(torch.isfinite(got[reached][:, -1].float()).any())  # of the last head, whose decay is 1
    assert ppo.ppo_poll_status() == 0
