"""References of the state-to-state operators in 64 bits, on the CPU, with bounds on what 32-bit arithmetic may add.

Bounds follow the kernels' order of operations: a rounding to fp32 is off by at most u = 2^-24 relative, the hardware's exp2 and
reciprocal by 2u, one to bf16 by 2^-8; errors are propagated through the recurrence beside the values.
"""
import math

import torch

import paper_2408_15237_amd as ssmv

U = 2.0 ** -24
IO = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {io: torch.finfo(t).eps / 2 for io, t in IO.items()}
NAN = float("nan")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, io=None):
    t = torch.randn(*shape, generator=g)
    return t if io is None else t.to(IO[io])


def strided(t, before, after, fill=NAN):
    """The same values inside a wider last dimension whose other columns hold `fill`: a view."""
    parent = torch.full(t.shape[:-1] + (before + t.shape[-1] + after,), fill, dtype=t.dtype, device=t.device)
    parent[..., before:before + t.shape[-1]] = t
    return parent[..., before:before + t.shape[-1]]


def silu(v):
    return v / (1 + torch.exp(-v))


def silu_err(v, ev):
    """Error of v * rcp(1 + exp2(-v log2 e)) for a v that is off by ev: slope at most 1.1; the exponent's rounding 3u |v| of e^-v, then four ulps."""
    return 1.1 * ev + silu(v).abs() * (3 * v.abs().clamp(max=120) + 8) * U


def rows_of(state, src, batch):
    """The rows that a call starts from: zeros where the index is outside."""
    if state is None:
        return None
    if src is None:
        return state[:batch]
    out = torch.zeros((batch,) + tuple(state.shape[1:]), dtype=state.dtype)
    for b, r in enumerate(src.tolist()):
        if 0 <= r < state.shape[0]:
            out[b] = state[r]
    return out


def conv_reference(x, w, bias, conv_in, act, io, src=None, lens=None):
    """(out, bound, conv_out): all tensors on the CPU."""
    b, n, C = x.shape
    hist = rows_of(conv_in, src, b)
    hist = torch.zeros(b, 3, C, dtype=x.dtype) if hist is None else hist
    out, bound = torch.zeros(b, n, C, dtype=torch.float64), torch.zeros(b, n, C, dtype=torch.float64)
    conv = torch.empty(b, 3, C, dtype=x.dtype)
    w64, bias64 = w.double(), (torch.zeros(C) if bias is None else bias).double()
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        raw = torch.cat([hist[i], x[i, :m]])
        conv[i] = raw[m:m + 3]
        terms = torch.stack([raw[k:k + m].double() * w64[:, k] for k in range(4)] + [bias64.expand(m, C)])
        v, e = terms.sum(0), 4 * U * terms.abs().sum(0)
        if act == "silu":
            v, e = silu(v), silu_err(v, e)
        out[i, :m], bound[i, :m] = v, e + HALF[io] * (v.abs() + e) + 1e-37
    return out, bound, conv


def softplus(v):
    return torch.logaddexp(v, torch.zeros((), dtype=torch.float64))


def scan_reference(x, dt, A, B, C, D, io, dt_bias=None, soft=False, z=None, h_in=None, src=None, lens=None):
    """Token by token: (y, bound of y, h, bound of h).  x [b][n][H][P], dt [b][n][H], A [H][N] or [H], B, C [b][n][G][N], z like x."""
    b, n, H, P = x.shape
    N, G = B.shape[-1], B.shape[2]
    start = rows_of(h_in, src, b)
    h = torch.zeros(b, H, P, N, dtype=torch.float64) if start is None else start.double().reshape(b, H, P, N)
    mag, err = h.abs(), torch.zeros_like(h)                     # magnitudes summed, and the error so far
    y, ey = torch.zeros(b, n, H, P, dtype=torch.float64), torch.zeros(b, n, H, P, dtype=torch.float64)
    A64 = A.double().reshape(1, H, 1, -1)
    group = torch.arange(H) // (H // G)
    lens = torch.full((b,), n) if lens is None else lens.clamp(0, n)
    for t in range(n):
        live = (t < lens).reshape(b, 1, 1, 1)
        d, rel = dt[:, t].double(), torch.zeros(b, H, dtype=torch.float64)
        if soft:
            v = d + (0.0 if dt_bias is None else dt_bias.double())
            d = softplus(v)
            # the sum's rounding moves log(1 + e^v) by at most u |v|; the exponent's rounding e^-|v| by 3u |v|; sixteen roundings behind
            rel = (4 * v.abs() + 16) * U + U * v.abs() / d.clamp(min=1e-30) * torch.sigmoid(v)
        xt, Bt, Ct = x[:, t].double(), B[:, t].double()[:, group], C[:, t].double()[:, group]
        arg = (d[:, :, None, None] * A64)
        decay = torch.exp(arg)
        relx = rel[:, :, None, None]
        u = (d[:, :, None] * xt)[..., None] * Bt[:, :, None, :]
        new = decay * h + u
        newmag = decay * mag + u.abs()
        e_decay = arg.abs().clamp(max=200) * (3 * U + relx) + 2 * U                       # A log2 e, times dt', exp2
        newerr = decay * err + decay * mag * e_decay + u.abs() * (relx + 3 * U) + U * newmag
        h, mag, err = torch.where(live, new, h), torch.where(live, newmag, mag), torch.where(live, newerr, err)
        Cn = Ct[:, :, None, :]
        o = (h * Cn).sum(-1) + D.double()[:, None] * xt
        terms = (mag * Cn.abs()).sum(-1) + (D.double()[:, None] * xt).abs()
        e = (err * Cn.abs()).sum(-1) + (N + 4) * U * terms
        if z is not None:
            zt = z[:, t].double()
            e = e * silu(zt).abs() + o.abs() * silu_err(zt, torch.zeros_like(zt)) + 2 * U * (o * silu(zt)).abs()
            o = o * silu(zt)
        lv = live[..., 0]
        y[:, t] = torch.where(lv, o, torch.zeros_like(o))
        ey[:, t] = torch.where(lv, e + HALF[io] * (o.abs() + e) + 1e-37, torch.zeros_like(o))
    return y, ey, h, err + 1e-37


def beam_reference(logits, scores, beams_out, batch, done=None, eos=-1):
    """Per sequence the candidates in order as (score, row, token): scores in 64 bits, ties by row, then by logit and token."""
    W = logits.shape[0] // batch
    top = torch.finfo(torch.float32).max
    out = []
    for s in range(batch):
        cand = []
        for r in range(s * W, (s + 1) * W):
            l = torch.nan_to_num(logits[r].float(), nan=-math.inf, posinf=top, neginf=-math.inf).double()
            given = float(torch.nan_to_num(scores[r], nan=-math.inf, posinf=top, neginf=-math.inf))
            keep = min(beams_out, l.numel())
            if done is not None and int(done[r]):
                cand += [(given if i == 0 else -math.inf, r, i, eos) for i in range(keep)]
                continue
            lp = l - l.max().clamp(min=-top) - torch.log(torch.exp(l - l.max().clamp(min=-top)).sum()) if float(l.max()) > -math.inf else l
            order = torch.sort(l, descending=True, stable=True).indices[:keep].tolist()
            cand += [(given + float(lp[v]) if float(l[v]) > -math.inf else -math.inf, r, i, v) for i, v in enumerate(order)]
        cand.sort(key=lambda c: (-c[0], c[1], c[2]))
        out.append([(c[0], c[1], c[3]) for c in cand])
    return out


def check_within(got, ref, bound, what):
    got = got.detach().cpu().double()
    off = (got - ref).abs()
    bad = ~(off <= bound)                                        # NaN is bad too
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d outside, first at %s: got %r, want %r +- %r" % (what, int(bad.sum()), bad.numel(), i, float(got[i]), float(ref[i]), float(bound[i])))


def cuda(t):
    """The same values and strides on the GPU (a view of a wider tensor stays one)."""
    if t is None:
        return None
    if t.is_contiguous():
        return t.cuda()
    base = t._base
    return base.cuda().as_strided(t.shape, t.stride(), t.storage_offset())


def lib():
    return ssmv
