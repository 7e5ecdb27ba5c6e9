"""ssm_gated_recurrence and its gradients in every kind of plan: narrow and wide workgroups, sequences whole and cut into segments of one tile and of several.  Every case's launches are looked at, so that one
that another plan lays out in another way fails here."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _harness import launches
from _layers import IO, check, cuda, gated_backward, gated_forward, gen
from test_gpu_gated_recurrence import _call, _check_backward, _check_forward, _inputs, _space

pytestmark = pytest.mark.gpu

# (type, workgroup, segments of the longest sequence, batch, tokens, channels); a wide workgroup has 64 channels in bf16 and 32 in fp32, a narrow one half of them
FORWARD = [("bf16", "narrow", 1, 1, 129, 33), ("bf16", "narrow", 1, 37, 602, 65), ("bf16", "narrow", 4, 21, 912, 71), ("bf16", "narrow", 3, 28, 1499, 65), ("bf16", "wide", 1, 1, 68, 67),
           ("bf16", "wide", 1, 40, 300, 451), ("bf16", "wide", 8, 1, 450, 65), ("bf16", "wide", 5, 1, 513, 65), ("f32", "narrow", 1, 1, 129, 19), ("f32", "narrow", 1, 37, 602, 35),
           ("f32", "narrow", 4, 22, 920, 39), ("f32", "narrow", 3, 36, 1373, 35), ("f32", "wide", 1, 1, 68, 43), ("f32", "wide", 1, 62, 300, 83), ("f32", "wide", 8, 1, 450, 35),
           ("f32", "wide", 5, 1, 514, 35)]
BACKWARD = [("bf16", "narrow", 1, 1, 68, 35), ("bf16", "narrow", 1, 1, 350, 35), ("bf16", "narrow", 4, 1, 385, 33), ("bf16", "narrow", 3, 28, 658, 67), ("bf16", "wide", 1, 24, 70, 451),
            ("bf16", "wide", 1, 40, 300, 451), ("bf16", "wide", 8, 1, 450, 71), ("bf16", "wide", 5, 1, 514, 65), ("f32", "narrow", 1, 1, 68, 17), ("f32", "narrow", 1, 1, 350, 17),
            ("f32", "narrow", 4, 1, 385, 17), ("f32", "narrow", 3, 31, 642, 33), ("f32", "wide", 1, 62, 72, 83), ("f32", "wide", 1, 62, 300, 83), ("f32", "wide", 8, 1, 449, 33),
            ("f32", "wide", 5, 1, 513, 45)]
IDS = lambda cases: ["%s-%s-%dseg-%dx%dx%d" % c for c in cases]


def _launches(case, backward):
    io, width, segments, b, n, C = case
    E = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")
    x, f, s = E(b, n, C, t=IO[io]), E(b, n, C, t=IO[io]), E(b, (n + 63) // 64, C)
    if not backward:
        y, w = torch.empty_like(x), _space(ssmv.ssm_gated_recurrence_workspace(b, C, n))
        return launches(lambda: ssmv.ssm_gated_recurrence(x=x, f=f, y_out=y, states=s, batch=b, channels=C, L=n, io=io, form="mix", workspace=w))
    dx, fb, dfb, w = torch.empty_like(x), E(C), E(C), _space(ssmv.ssm_gated_recurrence_backward_workspace(b, C, n))
    return launches(lambda: ssmv.ssm_gated_recurrence_backward(x=x, f=f, f_bias=fb, states=s, dy=f, dx=dx, df_bias=dfb, batch=b, channels=C, L=n, io=io, form="mix", workspace=w))


def _expected(case, backward):
    io, width, segments, b, n, C = case
    channels = (2 if io == "bf16" else 1) * (32 if width == "wide" else 16)
    groups, threads = b * -(-C // channels), 1024 if width == "narrow" and not backward else 512
    return ([(groups * (segments - 1), threads)] if segments > 1 else []) + [(groups * segments, threads)] + ([(3 * -(-C // 32), 1024)] if backward else [])


def _lens(b, n):
    """Of ends inside and at the ends of tiles and segments, none at all, and more than there are."""
    return [n] if b == 1 else [[n, 0, n - 1, 1, 63, 64, 65, n // 2, 256, 257, -3, n + 9][i % 12] for i in range(b)]


@pytest.mark.parametrize("form", ["lru", "mix"])
@pytest.mark.parametrize("case", FORWARD, ids=IDS(FORWARD))
def test_forward(case, form):
    io, _, _, b, n, C = case
    assert _launches(case, False) == _expected(case, False)
    _check_forward(b, n, C, io, form, seed=1, slow=True)
    _check_forward(b, n, C, io, form, seed=2, lens=_lens(b, n), in_place=True)
    _check_forward(b, n, C, io, form, seed=3, lens=[n - 70] * b, src=[(3 * i + 1) % (b + 1) - 1 for i in range(b)], inp=0, gate=0, wide=(1, 2))


@pytest.mark.parametrize("form", ["lru", "mix"])
@pytest.mark.parametrize("case", BACKWARD, ids=IDS(BACKWARD))
def test_backward(case, form):
    io, _, _, b, n, C = case
    assert _launches(case, True) == _expected(case, True)
    _check_backward(b, n, C, io, form, seed=1, slow=True)
    _check_backward(b, n, C, io, form, seed=2, lens=_lens(b, n), dh=False)
    _check_backward(b, n, C, io, form, seed=3, lens=[max(n - 70, 1)] * b, inp=0, gate=0, wide=(1, 2))


@pytest.mark.parametrize("b,n,C", [(1, 450, 71), (21, 912, 71), (2, 70, 33), (3, 1, 40)])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_workspaces_are_not_left(io, b, n, C):
    """What lies behind the bytes that a call asks for is left as it was."""
    t, up = _inputs(b, n, C, io, "lru", 4)
    d, u = {k: cuda(v) for k, v in t.items()}, {k: cuda(v) for k, v in up.items()}
    y, s, h = torch.empty_like(d["x"]), torch.empty(b, (n + 63) // 64, C, device="cuda"), torch.empty(b, C, device="cuda")
    vec = dict(dA=torch.empty(C, device="cuda"), df_bias=torch.empty(C, device="cuda"), di_bias=torch.empty(C, device="cuda"))
    sizes = [ssmv.ssm_gated_recurrence_workspace(b, C, n), ssmv.ssm_gated_recurrence_backward_workspace(b, C, n)]
    work = [torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda") for size in sizes]
    ssmv.ssm_gated_recurrence(**d, h_out=h, states=s, y_out=y, batch=b, channels=C, L=n, io=io, form="lru", workspace=work[0])
    ssmv.ssm_gated_recurrence_backward(**{k: v for k, v in d.items() if k != "h_in"}, **u, states=s, dx=torch.empty_like(y), **vec, batch=b, channels=C, L=n, io=io, form="lru", workspace=work[1])
    torch.cuda.synchronize()
    assert all(bool((w[size:] == 0x5A).all()) for w, size in zip(work, sizes))


@pytest.mark.parametrize("form", ["lru", "mix"])
def test_gradients_along_themselves_against_differences(form):
    """The loss sum(y dy) + sum(h dh) of fp32 forward calls, moved both ways along each input's own gradient in 64 bits (a random direction is nearly orthogonal to it).  What may lie between the difference
    and the kernel's gradient: the same difference in 64 bits less the slope there, for the step's length; the bounds of both forward calls' outputs times dy and dh over the step; the gradient's own bound.
    All of it has to be under a quarter of the slope, so that no gradient of zeros or of another sign passes."""
    b, n, C, step = 2, 70, 30, 2.0 ** -4
    t, up = _inputs(b, n, C, "f32", form, 6)
    if form == "lru":
        t["A"] = -0.4 - 0.4 * torch.rand(C, generator=gen(13))
    want = gated_backward(**t, **up)
    _, _, s, d = _call(t, b, n, C, "f32", form)
    got = {k: torch.empty(w.v.shape, device="cuda") for k, w in want.items()}
    ssmv.ssm_gated_recurrence_backward(**{k: v for k, v in d.items() if k != "h_in"}, states=s, dy=cuda(up["dy"]), dh_out=cuda(up["dh_out"]), **got, batch=b, channels=C, L=n, io="f32", form=form,
                                       workspace=_space(ssmv.ssm_gated_recurrence_backward_workspace(b, C, n)))
    names = dict(dx="x", df="f", di="i", dz="z", dA="A", df_bias="f_bias", di_bias="i_bias", dh_in="h_in")

    def losses(moved):
        """By the kernel, in 64 bits, and how far apart they may be."""
        y, h, _, _ = _call(moved, b, n, C, "f32", form, states=False)
        wy, _, wh, _ = gated_forward(**moved)
        total = lambda y, h: float((y.double() * up["dy"]).sum() + (h.double() * up["dh_out"]).sum())
        return total(y.cpu(), h.cpu()), total(wy.v, wh.v), total(wy.e * up["dy"].sign(), wh.e * up["dh_out"].sign())

    for k, w in want.items():
        name = names[k]
        way = (w.v / w.v.norm() * (1.0 if k == "dA" else 4.0)).float()
        a, b64, ea = losses({**t, name: t[name] + step * way})
        c, d64, ec = losses({**t, name: t[name] - step * way})
        slope = float((w.v * way).sum())
        room = abs((b64 - d64) / (2 * step) - slope) + (ea + ec) / (2 * step) + float((w.e * way.abs()).sum())
        assert room < slope / 4, (k, room, slope)
        assert abs((a - c) / (2 * step) - float((got[k].cpu().double() * way).sum())) <= room, (k, room, slope)
