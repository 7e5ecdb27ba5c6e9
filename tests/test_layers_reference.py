"""The 64-bit references of the layer operators against automatic differentiation of the definitions and against differences, on the CPU."""
import pytest
import torch

import _layers as ref
from _decode import gen


def _close(a, b, what):
    assert torch.allclose(a, b, rtol=1e-9, atol=1e-11), (what, float((a - b).abs().max()))


@pytest.mark.parametrize("flags", [(1, 1, 1, 1, 1), (0, 1, 0, 1, 1), (1, 0, 1, 0, 1), (0, 0, 0, 1, 1), (1, 1, 1, 1, 0)])
def test_norm_gradients(flags):
    gate, post, scale, pre, residual = flags
    g = gen(3)
    t = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_()
    x, z, res, w2, c, w1 = t(4, 7), t(4, 7) if gate else None, t(4, 7) if residual else None, t(7) if post else None, t(7) if scale else None, t(7) if pre else None
    dr, dn, alpha = torch.randn(4, 7, generator=g, dtype=torch.float64), torch.randn(4, 7, generator=g, dtype=torch.float64), 0.5

    def loss(*_):
        eps = float(torch.tensor(ref.EPS))
        p = x if z is None else x * torch.nn.functional.silu(z)
        if w2 is not None:
            p = p / (p.square().mean(-1, keepdim=True) + eps).sqrt() * w2
        r = alpha * p * (1 if c is None else c) + (0 if res is None else res)
        n = r / (r.square().mean(-1, keepdim=True) + eps).sqrt() * (1 if w1 is None else w1)
        return (r * dr).sum() + (n * dn).sum()

    leaves = dict(dx=x, dz=z, dres=res, dpost=w2, dscale=c, dpre=w1)
    leaves = {k: v for k, v in leaves.items() if v is not None}
    want = torch.autograd.grad(loss(), list(leaves.values()))
    d = lambda v: None if v is None else v.detach()
    got = ref.norm_backward(d(x), d(z), d(res), d(w2), d(c), d(w1), alpha, dr, dn)
    assert set(got) == set(leaves)
    for (k, leaf), w in zip(leaves.items(), want):
        _close(got[k].v, w, k)
        # and a difference along a random direction
        way = torch.randn(leaf.shape, generator=g, dtype=torch.float64)
        with torch.no_grad():
            leaf += 1e-5 * way
            up = loss()
            leaf -= 2e-5 * way
            down = loss()
            leaf += 1e-5 * way
        assert abs(float((up - down) / 2e-5 - (w * way).sum())) < 1e-6


@pytest.mark.parametrize("form", ["lru", "mix"])
@pytest.mark.parametrize("inp,gate", [(1, 1), (0, 0), (1, 0)])
def test_recurrence_gradients(form, inp, gate):
    g = gen(5)
    b, n, C = 3, 9, 4
    t = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_()
    x, f, i, z, fb, ib, h0 = t(b, n, C), t(b, n, C), t(b, n, C) if inp else None, t(b, n, C) if gate else None, t(C), t(C) if inp else None, t(b, C)
    A = (-torch.rand(C, generator=g, dtype=torch.float64) * 3).requires_grad_() if form == "lru" else None
    lens = torch.tensor([9, 4, 0])
    dy, dh = torch.randn(b, n, C, generator=g, dtype=torch.float64), torch.randn(b, C, generator=g, dtype=torch.float64)

    def run():
        r = torch.sigmoid(f + fb)
        a = torch.exp(A * r) if form == "lru" else r
        v = (1 - a * a).sqrt() * x if form == "lru" else (1 - a) * x
        if inp:
            v = v * torch.sigmoid(i + ib)
        total, hs = 0, []
        for s in range(b):
            h = h0[s]
            for k in range(int(lens[s])):
                h = a[s, k] * h + v[s, k]
                total = total + ((h * torch.nn.functional.silu(z[s, k]) if gate else h) * dy[s, k]).sum()
            hs.append(h)
        return total + (torch.stack(hs) * dh).sum(), torch.stack(hs)

    leaves = dict(dx=x, df=f, di=i, dz=z, dA=A, df_bias=fb, di_bias=ib, dh_in=h0)
    leaves = {k: v for k, v in leaves.items() if v is not None}
    total, h = run()
    want = torch.autograd.grad(total, list(leaves.values()))
    d = lambda v: None if v is None else v.detach()
    got = ref.gated_backward(d(x), d(f), dy, d(i), d(z), d(A), d(fb), d(ib), d(h0), lens, dh)
    assert set(got) == set(leaves)
    for (k, leaf), w in zip(leaves.items(), want):
        _close(got[k].v, w, k)
        way = torch.randn(leaf.shape, generator=g, dtype=torch.float64)
        with torch.no_grad():
            leaf += 1e-5 * way
            up = run()[0]
            leaf -= 2e-5 * way
            down = run()[0]
            leaf += 1e-5 * way
        assert abs(float((up - down) / 2e-5 - (w * way).sum())) < 1e-5
    _close(ref.gated_forward(d(x), d(f), d(i), d(z), d(A), d(fb), d(ib), d(h0), None, lens)[2].v, h.detach(), "h")


def test_bounds_hold_for_fp32_arithmetic():
    """The bounds are for 32-bit arithmetic in any order: torch's own must be inside them, and near the values they must be small."""
    g = gen(8)
    x, z, res, w = (torch.randn(5, 300, generator=g) for _ in range(4))
    w = w[0]
    a, sigma, p, r, rho, n = ref.norm_forward(x, z, res, w, None, w, 0.5)
    a32 = x * z * torch.sigmoid(z)
    r32 = res + 0.5 * (a32 * torch.rsqrt((a32 * a32).mean(-1, keepdim=True) + ref.EPS) * w)
    n32 = r32 * torch.rsqrt((r32 * r32).mean(-1, keepdim=True) + ref.EPS) * w
    ref.check(n32, n, "f32", "n")
    assert float((n.e / n.v.abs().clamp(min=1e-2)).max()) < 1e-3
    f = torch.randn(2, 200, 30, generator=g)
    A = -torch.rand(30, generator=g)
    y, _, h, k = ref.gated_forward(f.flip(0), f, A=A)
    s = A * torch.sigmoid(f)
    aa, vv = torch.exp(s), torch.sqrt(-torch.expm1(2 * s)) * f.flip(0)
    cur, ys = torch.zeros(2, 30), []
    for t in range(200):
        cur = aa[:, t] * cur + vv[:, t]
        ys.append(cur)
    ref.check(torch.stack(ys, 1), y, "f32", "y")
    assert float(y.e.max()) < 1e-3                                  # 200 tokens, some of which are never forgotten
