"""References of the layer operators in 64 bits, on the CPU, with bounds on what 32-bit arithmetic may add.

`Num` carries a value and a bound of its error through the formulas: every operation passes on the errors of its operands and adds its own rounding,
u = 2^-24 of the result (hardware exp2, rcp, rsq and sqrt: 2u); a sum of terms adds `depth` roundings of the sum of their sizes, depth being how many additions a
term can go through.  A rounding to bf16 at the end is 2^-8 / 2 = HALF of the value.
"""
import math

import torch

from _decode import HALF, IO, U, check_within, cuda, gen, randn, rows_of, strided  # noqa: F401

TINY = 1e-36              # of what underflows
LN2 = math.log(2.0)
EPS = 1e-5
ROW = 64                  # additions that a term of a row's sum goes through: 16 in a thread, 6 in a wave, 16 waves, and room


class Num:
    def __init__(self, v, e=None):
        self.v = v.double()
        self.e = torch.zeros_like(self.v) if e is None else e

    def _of(self, o):
        return o if isinstance(o, Num) else Num(torch.as_tensor(o, dtype=torch.float64))

    def __add__(self, o):
        o = self._of(o)
        v = self.v + o.v
        return Num(v, self.e + o.e + U * v.abs())

    def __sub__(self, o):
        o = self._of(o)
        v = self.v - o.v
        return Num(v, self.e + o.e + U * v.abs())

    def __mul__(self, o):
        o = self._of(o)
        v = self.v * o.v
        return Num(v, self.v.abs() * o.e + o.v.abs() * self.e + self.e * o.e + U * v.abs() + TINY)

    def sum(self, dim, depth, keepdim=False):
        return Num(self.v.sum(dim, keepdim=keepdim), self.e.sum(dim, keepdim=keepdim) + depth * U * self.v.abs().sum(dim, keepdim=keepdim))

    def rsqrt(self):
        v = self.v.rsqrt()
        return Num(v, v * (0.51 * self.e / self.v + 3 * U))

    def where(self, mask, other=0.0):
        o = torch.tensor(other, dtype=torch.float64)
        return Num(torch.where(mask, self.v, o), torch.where(mask, self.e, torch.zeros((), dtype=torch.float64)))

    def bound(self, io):
        """Of the value as stored in `io` ("f32": nothing is added)."""
        return self.e + (HALF[io] * (self.v.abs() + self.e) if io == "bf16" else 0.0) + TINY


def num(t):
    return None if t is None else Num(t)


def sigmoid(n):
    """1 / (1 + 2^(-v log2 e)): two roundings of the exponent move e^-v by 3u |v|, then an addition and two hardware functions."""
    s = torch.sigmoid(n.v)
    return Num(s, s * (1 - s) * n.e + s * (3 * n.v.abs().clamp(max=120) + 8) * U + TINY)


def opposite(n):
    """1 - sigmoid, as accurate."""
    return sigmoid(Num(-n.v, n.e))


def silu(n):
    return n * sigmoid(n)


def silu_slope(n):
    s = sigmoid(n)
    return s * (n * (Num(1 + 0 * n.v) - s) + 1.0)


# ---- between two blocks ---------------------------------------------------------------------------------------------------


def norm_forward(x, z, res, post, scale, pre, alpha):
    """(a, sigma, p, r, rho, n) as Num; None where there is none.  eps and alpha as fp32 has them."""
    eps, alpha = float(torch.tensor(EPS)), float(torch.tensor(alpha))
    a = sigma = p = None
    r = num(res)
    if x is not None:
        a = num(x) if z is None else num(x) * silu(num(z))
        p = a
        if post is not None:
            C = a.v.shape[-1]
            sigma = ((a * a).sum(-1, ROW, True) * (1.0 / C) + eps).rsqrt()
            p = a * sigma * num(post)
        t = p * alpha
        if scale is not None:
            t = t * num(scale)
        r = t if r is None else r + t
    rho = ((r * r).sum(-1, ROW, True) * (1.0 / r.v.shape[-1]) + eps).rsqrt()
    n = r * rho
    return a, sigma, p, r, rho, n if pre is None else n * num(pre)


def norm_backward(x, z, res, post, scale, pre, alpha, dr, dn):
    """Gradients as a dict of Num."""
    a, sigma, p, r, rho, _ = norm_forward(x, z, res, post, scale, pre, alpha)
    alpha, out, rows = float(torch.tensor(alpha)), {}, r.v.shape[0]
    depth = 64 + rows // 128                                       # of a vector's sum: a thread's rows, then 512 parts in 16 strands
    d = num(dr) if dr is not None else Num(torch.zeros_like(r.v))
    if dn is not None:
        dn = num(dn)
        g = dn if pre is None else dn * num(pre)
        mean = (g * r).sum(-1, ROW, True) * (1.0 / r.v.shape[-1])
        d = d + rho * (g - r * (rho * rho * mean))
        if pre is not None:
            out["dpre"] = (dn * rho * r).sum(0, depth)
    elif pre is not None:
        out["dpre"] = Num(torch.zeros_like(pre))
    if res is not None:
        out["dres"] = d
    if x is None:
        return out
    d = d * alpha
    if scale is not None:
        out["dscale"] = (d * p).sum(0, depth)
        d = d * num(scale)
    if post is not None:
        out["dpost"] = (d * sigma * a).sum(0, depth)
        g = d * num(post)
        mean = (g * a).sum(-1, ROW, True) * (1.0 / a.v.shape[-1])
        d = sigma * (g - a * (sigma * sigma * mean))
    if z is not None:
        out["dz"] = d * num(x) * silu_slope(num(z))
        d = d * silu(num(z))
    out["dx"] = d
    return out


# ---- the gated recurrence -------------------------------------------------------------------------------------------------


def coefficients(x, f, i, A, f_bias, i_bias):
    """Num of everything a token brings: decay a, m, s = -ln a, r, 1 - r, sigmoid of i, 1 - that, u = i x, v = m u."""
    f = num(f) if f_bias is None else num(f) + num(f_bias)
    r, nr = sigmoid(f), opposite(f)
    x = num(x)
    si = ni = None
    u = x
    if i is not None:
        i = num(i) if i_bias is None else num(i) + num(i_bias)
        si, ni = sigmoid(i), opposite(i)
        u = x * si
    if A is None:
        a, m, s, m2 = r, nr, None, None
    else:
        s = r * Num(-A)                                             # natural units; the kernel's factors log2 e and ln 2 are two roundings more
        s = Num(s.v, s.e + 3 * U * s.v)
        av = torch.exp(-s.v)
        a = Num(av, av * (s.e + 2 * U))
        m2v = -torch.expm1(-2 * s.v)
        near = 2 * s.v < 0.35
        m2 = Num(m2v, torch.where(near, 2 * s.e + m2v * (10 * U + 2e-8), 2 * av * a.e + 2 * U))
        mv = m2v.sqrt()
        m = Num(mv, torch.where(mv > 0, 0.51 * m2.e / mv.clamp(min=1e-300), torch.zeros(())) + 2 * U * mv)
    return dict(a=a, m=m, s=s, m2=m2, r=r, nr=nr, si=si, ni=ni, u=u, v=m * u)


def _chain(a, add, start):
    """All values of c <- a c + add along dim 1, with the error of any order of combination: a product of n decays is off by n u besides its
    factors' errors, and a term goes through at most 24 additions that the token-by-token order does not have."""
    out_v, out_e = [], []
    v, e, mag = start.v, start.e, start.v.abs()
    for t in range(a.v.shape[1]):
        at, ea, w, ew = a.v[:, t], a.e[:, t], add.v[:, t], add.e[:, t]
        e = at * e + ea * mag + 3 * U * at * mag + ew
        v = at * v + w
        mag = at * mag + w.abs()
        e = e + U * mag
        out_v.append(v)
        out_e.append(e + 24 * U * mag)
    return Num(torch.stack(out_v, 1), torch.stack(out_e, 1))


def _live(lens, b, n):
    lens = torch.full((b,), n) if lens is None else lens.clamp(0, n).long()
    return lens, (torch.arange(n)[None, :] < lens[:, None])[..., None]


def gated_forward(x, f, i=None, z=None, A=None, f_bias=None, i_bias=None, h_in=None, src=None, lens=None):
    """(y, h ahead of every token [b][n], h after a sequence's tokens [b], coefficients)."""
    b, n, C = x.shape
    lens, live = _live(lens, b, n)
    k = coefficients(x, f, i, A, f_bias, i_bias)
    start = rows_of(h_in, src, b)
    start = Num(torch.zeros(b, C) if start is None else start)
    h = _chain(k["a"].where(live, 1.0), k["v"].where(live), start)
    before = Num(torch.cat([start.v[:, None], h.v[:, :-1]], 1), torch.cat([start.e[:, None], h.e[:, :-1]], 1))
    y = h if z is None else h * silu(num(z))
    return y.where(live), before, Num(h.v[:, -1], h.e[:, -1]), k


def gated_backward(x, f, dy, i=None, z=None, A=None, f_bias=None, i_bias=None, h_in=None, lens=None, dh_out=None, states=None):
    """Gradients as a dict of Num; states (the kernel's own) replaces the bound of h ahead of every 64th token by nothing where given."""
    b, n, C = x.shape
    lens, live = _live(lens, b, n)
    _, before, _, k = gated_forward(x, f, i, z, A, f_bias, i_bias, h_in, None, lens)
    h = k["a"] * before + k["v"]
    dy, out = num(dy).where(live), {}
    g = dy
    if z is not None:
        out["dz"] = (dy * h * silu_slope(num(z))).where(live)
        g = dy * silu(num(z))
    a = k["a"].where(live, 1.0)
    flip = lambda q: Num(q.v.flip(1), q.e.flip(1))
    start = Num(torch.zeros(b, C) if dh_out is None else dh_out)
    # what flows out of token t's front: c <- a (g + c)
    c = _chain(flip(a), flip((a * g).where(live)), start)
    out["dh_in"] = Num(c.v[:, -1], c.e[:, -1])
    into = flip(Num(torch.cat([start.v[:, None], c.v[:, :-1]], 1), torch.cat([start.e[:, None], c.e[:, :-1]], 1)))
    G = g + into
    sums = (0, 1)
    depth = 64 + n // 8 + b * 16
    if A is None:
        df = G * (k["r"] * k["nr"]) * (before - k["u"])
    else:
        inv = Num(1 / k["m2"].v.clamp(min=1e-37), k["m2"].e / k["m2"].v.clamp(min=1e-37) ** 2 + 2 * U / k["m2"].v.clamp(min=1e-37))
        E = (k["s"] * k["a"]) * G * (k["v"] * k["a"] * inv - before)
        df = E * k["nr"]
        total = E.where(live).sum(sums, depth)
        zero = A == 0
        Av = torch.where(zero, torch.ones_like(A), A).double()
        out["dA"] = Num(torch.where(zero, 0.0, total.v / Av), torch.where(zero, 0.0, total.e / Av.abs() + 2 * U * (total.v / Av).abs()))
    out["df"] = df.where(live)
    if f_bias is not None:
        out["df_bias"] = out["df"].sum(sums, depth)
    out["dx"] = (G * k["m"] if i is None else G * k["m"] * k["si"]).where(live)
    if i is not None:
        out["di"] = (G * k["v"] * k["ni"]).where(live)
        if i_bias is not None:
            out["di_bias"] = out["di"].sum(sums, depth)
    return out


# ---- rules on logits ------------------------------------------------------------------------------------------------------


def rules_reference(logits, hist=None, hist_len=None, src=None, token=None, prompt=None, rep=None, freq=None, pres=None, bias_token=None, bias=None, mask=None, mask_row=None):
    """(values, bounds, histories as lists): row by row."""
    rows, V = logits.shape
    out, err, said_all = logits.double().clone(), torch.zeros(rows, V, dtype=torch.float64), []
    for b in range(rows):
        l, e, said = out[b], err[b], []
        if hist is not None:
            j = b if src is None else int(src[b])
            if 0 <= j < hist.shape[0]:
                said = hist[j, :min(max(int(hist_len[j]), 0), hist.shape[1])].tolist()
            if token is not None:
                said = said + [int(token[b])]
            start = 0 if prompt is None else int(prompt[b])
            for v in set(t for t in said if 0 <= t < V):
                if rep is not None:
                    r = float(rep[b])
                    l[v] = l[v] / r if l[v] > 0 else l[v] * r
                    e[v] += U * abs(float(l[v])) if math.isfinite(float(l[v])) else 0.0
                n = sum(t == v for t in said[max(start, 0):])
                if n:
                    a, p = (0.0 if freq is None else float(freq[b])), (0.0 if pres is None else float(pres[b]))
                    if math.isfinite(float(l[v])):
                        e[v] += U * (abs(a * n) + abs(float(l[v]) - a * n) + abs(float(l[v]) - a * n - p))
                    l[v] = l[v] - a * n - p
        said_all.append(said)
        if bias_token is not None:
            for v, w in zip(bias_token[b].tolist(), bias[b].tolist()):
                if 0 <= v < V:
                    l[v] += w
                    if math.isfinite(w) and math.isfinite(float(l[v])):
                        e[v] += U * (abs(w) * bias_token.shape[1] + abs(float(l[v])))
        if mask is not None:
            m = b if mask_row is None else int(mask_row[b])
            if 0 <= m < mask.shape[0]:
                at = torch.arange(V)
                off = (mask[m].long()[at // 32] >> (at % 32)) & 1 == 0
                l[off], e[off] = -math.inf, 0.0
    return out, err, said_all


def check_rules(got, want, err, io, what):
    """Infinities and NaN where they belong, the rest within the bound."""
    got = got.detach().cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(torch.where(torch.isinf(want), want, torch.zeros(())).nan_to_num(nan=0), torch.where(torch.isinf(got), got, torch.zeros(())).nan_to_num(nan=0)), what
    fin = torch.isfinite(want)
    bound = err + (HALF[io] * want.abs().nan_to_num(posinf=0, neginf=0) * (1 + 1e-6) if io == "bf16" else 0.0) + TINY
    zero = torch.zeros((), dtype=torch.float64)
    check_within(torch.where(fin, got, zero), torch.where(fin, want, zero), bound, what)


def check(got, want, io, what):
    check_within(got, want.v, want.bound(io), what)
