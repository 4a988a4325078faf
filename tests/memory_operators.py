"""Plain forms in 64 bits of the causal convolution, the selective scan, and the norms of queries and keys with rotation, each with a bound
of what 32-bit arithmetic may be off by.

A `Num` carries a value and a running bound of its error, first order, in units of 2^-24: an operation passes the errors of its operands on and
adds the roundings of its own (one half unit each, counted as whole ones), and a sum of n terms adds up to n of them on any path, each at most
the sum of the absolute values."""
import torch

U = 2.0 ** -24


class Num:
    def __init__(self, v, e=None):
        self.v = v.double()
        self.e = torch.zeros_like(self.v) if e is None else e

    def __add__(self, o):
        return Num(self.v + o.v, self.e + o.e + self.v.abs() + o.v.abs())

    def __mul__(self, o):
        v = self.v * o.v
        return Num(v, self.v.abs() * o.e + o.v.abs() * self.e + v.abs())

    def sum(self, dims, roundings):
        return Num(self.v.sum(dims), (self.e + roundings * self.v.abs()).sum(dims))

    def map(self, value, slope, roundings):
        """A function of it: its value, a bound of its slope, and its own roundings relative to the value."""
        return Num(value, slope * self.e + roundings * value.abs())

    def __getitem__(self, i):
        return Num(self.v[i], self.e[i])

    def where(self, keep):
        return Num(torch.where(keep, self.v, torch.zeros_like(self.v)), torch.where(keep, self.e, torch.zeros_like(self.e)))

    def apply(self, f):
        """A rearrangement."""
        return Num(f(self.v), f(self.e))


def stack(nums, dim=0):
    return Num(torch.stack([n.v for n in nums], dim), torch.stack([n.e for n in nums], dim))


def within(got, want: Num, name=""):
    """Each element is within the bound and one rounding to its type."""
    assert got.shape == want.v.shape, (name, got.shape, want.v.shape)
    if got.numel() == 0:
        return
    tol = want.e * U
    tol = tol + torch.finfo(got.dtype).eps / 2 * (want.v.abs() + tol) + (2.0 ** -25 if got.dtype == torch.float16 else 0) + 1e-37
    assert not torch.isnan(got).any(), name
    off = (got.double() - want.v).abs() - tol
    assert float(off.max()) <= 0, (name, float(off.max()), float(((got.double() - want.v).abs() / tol).max()))


def sigmoid(x: Num):
    p = torch.sigmoid(x.v)
    # exp(-z) with its argument rounded: |z| units, and a few for the exponential, the sum and the quotient
    return Num(p, p * (1 - p) * (x.e + 2 * x.v.abs()) + 8 * p)


def activate(x: Num, act):
    if act == "silu":
        return x * sigmoid(x)
    return Num(x.v.clamp(min=0), x.e) if act == "relu" else x


def grad_act(x: Num, act):
    if act == "silu":
        p = sigmoid(x)
        one = Num(torch.ones_like(x.v))
        return p * (one + x * (one + Num(-p.v, p.e)))
    return Num((x.v > 0).double()) if act == "relu" else Num(torch.ones_like(x.v))


# -------------------------------------------------------------------------------------------------------- causal convolution --


def _reach(done, T, Be, W, device):
    """[W, T + W - 1, Be]: whether row r (of W - 1 rows of state and then the sequence) is seen by the step that its tap i belongs to,
    r - i + ... ; as a list over taps of [T, Be]: step t sees row t + i."""
    flags = torch.zeros(T + W, Be, dtype=torch.int64, device=device)
    if done is not None:
        flags[W:] = (done != 0).long()
    count = flags.cumsum(0)  # count[r]: flags in front of row r, with row t + W - 1 being step t
    return [count[i:i + T] == count[W - 1:W - 1 + T] for i in range(W)], count[T:T + W - 1] == count[T + W - 1]


def conv(x, weight, bias, done, state, act, dy=None, dstate=None):
    """y and the state that is left; with dy the gradients of x, weight, bias, state instead.  [T,Be,C], [Be,W-1,C]."""
    T, Be, C = x.shape
    W = weight.shape[1]
    old = torch.zeros(W - 1, Be, C, dtype=torch.float64, device=x.device) if state is None else state.double().transpose(0, 1)
    rows = torch.cat([old, x.double()])
    seen, left = _reach(done, T, Be, W, x.device)
    taps = [Num(torch.where(seen[i][..., None], rows[i:i + T], torch.zeros_like(rows[:1]))) for i in range(W)]
    w = [Num(weight[:, i]) for i in range(W)]
    s = stack([t * a for t, a in zip(taps, w)] + [Num((torch.zeros(C, device=x.device) if bias is None else bias).double().expand(T, Be, C))]).sum(0, W + 1)
    if dy is None:
        return activate(s, act), torch.where(left[..., None], rows[T:], torch.zeros_like(rows[:1])).transpose(0, 1)
    g = Num(dy) * grad_act(s, act)
    parts = [[] for _ in range(T + W - 1)]
    shares = Num(torch.zeros(W, T + W - 1, Be, C, dtype=torch.float64, device=x.device))
    for i in range(W):
        p = (g * w[i]).where(seen[i][..., None])
        shares.v[i, i:i + T], shares.e[i, i:i + T] = p.v, p.e
    del parts
    dx = shares.sum(0, W + 1)
    if dstate is not None:
        more = Num(torch.where(left[..., None], dstate.double().transpose(0, 1), torch.zeros_like(rows[:1])))
        tail = dx[T:] + more
        dx.v[T:], dx.e[T:] = tail.v, tail.e
    n = T * Be
    dw = stack([(g * t).sum((0, 1), n) for t in taps], 1)
    return dx[W - 1:], dw, g.sum((0, 1), n), dx[:W - 1].apply(lambda t: t.transpose(0, 1))


# -------------------------------------------------------------------------------------------------------------- selective scan --


def _steps(dt, bias, softplus):
    """Step sizes and the derivative by dt."""
    v = Num(dt) if bias is None else Num(dt) + Num(bias)
    if not softplus:
        return v, Num(torch.ones_like(v.v))
    d = torch.nn.functional.softplus(v.v, threshold=1e9)
    # the slope is at most 1, and sigmoid / softplus below 1.45; the function's own roundings: exponential (argument |v|), logarithm, sum
    return Num(d, torch.sigmoid(v.v) * (v.e + 2 * v.v.abs()) + 8 * d), sigmoid(v)


def scan(x, dt, A, B, C, D, z, bias, softplus, done, state, dy=None, dstate=None):
    """y and the state that is left; with dy a dict of gradients instead.  [T,Be,channels], [T,Be,groups,N]."""
    T, Be, channels = x.shape
    groups, N = B.shape[2:]
    share = channels // groups
    wide = lambda m: m.double().repeat_interleave(share, -2)  # noqa: E731
    d, slope = _steps(dt, bias, softplus)
    xs, An = Num(x), Num(A)
    live = torch.ones(T, Be, dtype=torch.bool, device=x.device) if done is None else done == 0
    u = d * xs
    h = Num(torch.zeros(Be, channels, N, dtype=torch.float64, device=x.device) if state is None else state)
    factors, before, after, ys = [], [], [], []
    for t in range(T):
        p = d[t].apply(lambda v: v[..., None]) * An
        a = torch.exp(p.v)
        # the argument times log2(e), rounded: |p| more units each; the exponential itself a few
        a = Num(a, a * (p.e + 3 * p.v.abs() + 4))
        before.append(h)
        factors.append(a)
        h = a * h + u[t].apply(lambda v: v[..., None]) * Num(wide(B[t]))
        after.append(h)
        ys.append((h * Num(wide(C[t]))).sum(-1, N + 1))
        h = h.where(live[t][:, None, None])
    y = stack(ys)
    if D is not None:
        y = y + Num(D) * xs
    gate = None if z is None else activate(Num(z), "silu")
    if dy is None:
        return (y if z is None else y * gate), h
    dout = Num(dy)
    dv = dout if z is None else dout * gate
    out = {"dx": [], "ddt": [], "dB": [], "dC": []}
    dA = Num(torch.zeros(channels, N, dtype=torch.float64, device=x.device))
    dbias = Num(torch.zeros(channels, dtype=torch.float64, device=x.device))
    g = Num(torch.zeros_like(h.v) if dstate is None else dstate)
    fold = lambda m: m.apply(lambda v: v.unflatten(1, (groups, share)).transpose(2, 3)).sum(-1, share)  # noqa: E731
    n = T * Be
    for t in reversed(range(T)):
        bt, ct, dvt = Num(wide(B[t])), Num(wide(C[t])), dv[t].apply(lambda v: v[..., None])
        g = ct * dvt + g.where(live[t][:, None, None])
        s1 = (g * bt).sum(-1, N + 1)
        out["dB"].append(fold(g * u[t].apply(lambda v: v[..., None])))
        out["dC"].append(fold(after[t] * dvt))
        g = g * factors[t]
        q = g * before[t]
        s2 = (q * An).sum(-1, N + 1)
        dA = dA + (q * d[t].apply(lambda v: v[..., None])).sum(0, n)
        out["dx"].append(s1 * d[t] if D is None else s1 * d[t] + Num(D) * dv[t])
        dd = (xs[t] * s1 + s2) * slope[t]
        out["ddt"].append(dd)
        dbias = dbias + dd.sum(0, n)
    out = {k: stack(v[::-1]) for k, v in out.items()}
    out.update(dA=dA, ddt_bias=dbias, dD=(dv * xs).sum((0, 1), n), dstate=g)
    if z is not None:
        out["dz"] = dout * y * grad_act(Num(z), "silu")
    return out


# --------------------------------------------------------------------------------------------- queries and keys, norm and rotation --


def _pairs(d, pairs, interleaved, device):
    i = torch.arange(pairs, device=device)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)


def _turn(pos, freq):
    """cos and sin of each row's angles, [rows, 1, pairs]: a few roundings, and those of the angle in 64 bits."""
    angle = (pos.double()[:, None] * freq.double())[:, None]
    e = 8 + angle.abs() * 2.0 ** -51 / U
    return Num(torch.cos(angle), e), Num(torch.sin(angle), e)


def _minus(n):
    return Num(-n.v, n.e)


def _norm(x, gamma, eps):
    d = x.shape[-1]
    xs = Num(x)
    m = (xs * xs).sum(-1, d).apply(lambda v: v[..., None] / d)
    r = 1 / torch.sqrt(m.v + eps)
    r = Num(r, r * (0.5 * m.e / (m.v + eps) + 6))
    return xs * r, r, Num(torch.ones(d, device=x.device) if gamma is None else gamma)


def rotate(n: Num, pos, freq, interleaved, back=False):
    if freq is None or freq.numel() == 0:
        return n
    a, b = _pairs(n.v.shape[-1], freq.numel(), interleaved, n.v.device)
    c, s = _turn(pos, freq)
    if back:
        s = _minus(s)
    first, second = n[..., a], n[..., b]
    x, y = first * c + _minus(second) * s, first * s + second * c
    out = Num(n.v.clone(), n.e.clone())
    out.v[..., a], out.e[..., a], out.v[..., b], out.e[..., b] = x.v, x.e, y.v, y.e
    return out


def qk(x, gamma, eps, pos, freq, interleaved, dy=None):
    """The heads of [rows,heads,d]; with dy the gradients of x and gamma instead."""
    xhat, r, gam = _norm(x, gamma, eps)
    if dy is None:
        return rotate(xhat * gam, pos, freq, interleaved)
    dn = rotate(Num(dy), pos, freq, interleaved, back=True)
    d = x.shape[-1]
    g = dn * gam
    dot = (g * xhat).sum(-1, d).apply(lambda v: v[..., None] / d)
    dot = Num(dot.v, dot.e + dot.v.abs())
    return r * (g + _minus(xhat * dot)), (dn * xhat).sum((0, 1), x.shape[0] * x.shape[1])
