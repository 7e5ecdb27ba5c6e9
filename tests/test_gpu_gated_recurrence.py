"""ssm_gated_recurrence and its gradients on the GPU against the formulas in 64 bits."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _layers import IO, check, cuda, gated_backward, gated_forward, gen, randn, strided

pytestmark = pytest.mark.gpu
TILE = ssmv.SSMV_GATED_TILE


def _inputs(b, n, C, io, form, seed, inp=1, gate=1, bias=1, hist=1, rows_in=None, slow=False):
    g = gen(seed)
    A = None
    if form == "lru":
        A = -8 * torch.rand(C, generator=g) * (0.01 if slow else 0.1)
    t = dict(x=randn(g, b, n, C, io=io), f=randn(g, b, n, C, io=io), i=randn(g, b, n, C, io=io) if inp else None, z=randn(g, b, n, C, io=io) if gate else None, A=A,
             f_bias=randn(g, C) + (2.0 if form == "mix" else 0.0) if bias else None, i_bias=randn(g, C) if bias and inp else None, h_in=randn(g, rows_in or b, C) if hist else None)
    return t, dict(dy=randn(g, b, n, C, io=io), dh_out=randn(g, b, C))


def _behind(t, lens, fill=float("nan")):
    """What lies behind a sequence's tokens must not matter."""
    if lens is None or t is None:
        return t
    t = t.clone()
    for i, m in enumerate(lens.tolist()):
        t[i, max(m, 0):] = fill
    return t


def _space(n):
    return torch.full((n // 4,), float("nan"), device="cuda") if n else None


def _call(t, b, n, C, io, form, src=None, lens=None, wide=None, rows_in=0, in_place=False, states=True):
    """The forward call: (y, h_out, states)."""
    lay = (lambda v: cuda(strided(v, *wide))) if wide else cuda
    d = {k: (lay(_behind(v, lens)) if v is not None and v.dim() == 3 else cuda(v)) for k, v in t.items()}
    st = lambda v: 0 if v is None else v.stride(1) if n > 1 or wide else 0
    y = strided(torch.full((b, n, C), 7.0, dtype=IO[io], device="cuda"), *(wide or (0, 0)), fill=5.0)
    h = d["h_in"] if in_place else torch.full((b, C), 7.0, device="cuda")
    s = torch.full((b, (n + TILE - 1) // TILE, C), 7.0, device="cuda") if states else None
    ssmv.ssm_gated_recurrence(x=d["x"], f=d["f"], i=d["i"], z=d["z"], A=d["A"], f_bias=d["f_bias"], i_bias=d["i_bias"], h_in=d["h_in"], src_row=cuda(src), seq_len=cuda(lens),
                              rows_in=rows_in, y_out=y, h_out=h, states=s, batch=b, channels=C, L=n, io=io, form=form, x_stride=st(d["x"]), f_stride=st(d["f"]),
                              i_stride=st(d["i"]), z_stride=st(d["z"]), y_stride=st(y), workspace=_space(ssmv.ssm_gated_recurrence_workspace(b, C, n)))
    torch.cuda.synchronize()
    return y, h, s, d


def _check_forward(b, n, C, io, form, seed=0, src=None, lens=None, wide=None, rows_in=None, in_place=False, **flags):
    src = None if src is None else torch.tensor(src, dtype=torch.int32)
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32)
    t, _ = _inputs(b, n, C, io, form, seed, rows_in=rows_in, **flags)
    want_y, before, want_h, _ = gated_forward(**t, src=src, lens=lens)
    y, h, s, _ = _call(t, b, n, C, io, form, src, lens, wide, rows_in or 0, in_place)
    check(h, want_h, "f32", "h")
    got = y.cpu()
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        part = lambda q: type(q)(q.v[i, :m], q.e[i, :m])
        check(got[i, :m], part(want_y), io, "y of sequence %d" % i)
        assert bool((got[i, m:] == 7).all()), "written behind the sequence's tokens"
        places = max((m + TILE - 1) // TILE, 1)
        check(s[i, :(m + TILE - 1) // TILE], type(before)(before.v[i, :m:TILE], before.e[i, :m:TILE]), "f32", "states of sequence %d" % i)
        if m == 0 and src is None:
            assert torch.equal(s[i, 0].cpu(), t["h_in"][i] if t["h_in"] is not None else torch.zeros(C))
        assert bool((s[i, places:] == 7).all())
    if wide:
        parent = y._base.cpu()
        assert bool((parent[..., :wide[0]] == 5).all()) and bool((parent[..., wide[0] + C:] == 5).all())


def _check_backward(b, n, C, io, form, seed=0, lens=None, wide=None, only=None, dh=True, **flags):
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32)
    t, up = _inputs(b, n, C, io, form, seed, **flags)
    if not dh:
        up["dh_out"] = None
    want = gated_backward(**t, **up, lens=lens)
    _, _, s, d = _call(t, b, n, C, io, form, None, lens, wide)
    lay = (lambda v: cuda(strided(v, *wide))) if wide else cuda
    dy = lay(_behind(up["dy"], lens))
    if lens is not None:                                            # states of tokens that are none
        for i, m in enumerate(lens.tolist()):
            s[i, max((m + TILE - 1) // TILE, 1):] = float("nan")
    st = lambda v: 0 if v is None else v.stride(1)
    out = {}
    for k, w in want.items():
        if only is None or k in only:
            out[k] = strided(torch.full((b, n, C), 7.0, dtype=IO[io], device="cuda"), *(wide or (0, 0)), fill=5.0) if w.v.dim() == 3 else torch.full(w.v.shape, 7.0, device="cuda")
    o = out.get
    ssmv.ssm_gated_recurrence_backward(x=d["x"], f=d["f"], i=d["i"], z=d["z"], A=d["A"], f_bias=d["f_bias"], i_bias=d["i_bias"], states=s, seq_len=cuda(lens), dy=dy,
                                       dh_out=cuda(up["dh_out"]), dx=o("dx"), df=o("df"), di=o("di"), dz=o("dz"), dA=o("dA"), df_bias=o("df_bias"), di_bias=o("di_bias"),
                                       dh_in=o("dh_in"), batch=b, channels=C, L=n, io=io, form=form, x_stride=st(d["x"]), f_stride=st(d["f"]), i_stride=st(d["i"]),
                                       z_stride=st(d["z"]), dy_stride=st(dy), dx_stride=st(o("dx")), df_stride=st(o("df")), di_stride=st(o("di")), dz_stride=st(o("dz")),
                                       workspace=_space(ssmv.ssm_gated_recurrence_backward_workspace(b, C, n)))
    torch.cuda.synchronize()
    for k, v in out.items():
        if v.dim() == 3:
            got = v.cpu()
            for i in range(b):
                m = n if lens is None else min(max(int(lens[i]), 0), n)
                check(got[i, :m], type(want[k])(want[k].v[i, :m], want[k].e[i, :m]), io, "%s of sequence %d" % (k, i))
                assert bool((got[i, m:] == 7).all()), "written behind the sequence's tokens"
        else:
            check(v, want[k], "f32", k)
    return out


FORMS = ["lru", "mix"]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 64, 65, 130, 519])
def test_lengths(io, form, n):
    _check_forward(3, n, 72, io, form, seed=n)
    _check_backward(3, n, 72, io, form, seed=n)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("C", [1, 2, 5, 16, 17, 63, 130, 257])
def test_channel_counts(io, form, C):
    _check_forward(2, 70, C, io, form, seed=C)
    _check_forward(4, 1, C, io, form, seed=C + 1)
    _check_backward(2, 70, C, io, form, seed=C)
    _check_backward(4, 1, C, io, form, seed=C + 1)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("flags", [dict(inp=0), dict(gate=0), dict(inp=0, gate=0), dict(bias=0), dict(hist=0), dict(inp=0, gate=0, bias=0, hist=0)])
def test_parts(io, form, flags):
    for n in (1, 100):
        _check_forward(2, n, 40, io, form, seed=4, **flags)
        _check_backward(2, n, 40, io, form, seed=4, **flags)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("b,n,C", [(2, 70, 40000), (600, 70, 34), (300, 150, 60), (40, 300, 150), (1, 700, 5200), (3, 333, 1001), (1, 1100, 1030), (5, 900, 33)])
def test_widths(form, b, n, C):
    """Workgroups of both widths, sequences whole and cut, tails of tokens and channels in each."""
    for io in ("bf16", "f32"):
        _check_forward(b, n, C, io, form, seed=1)
        _check_backward(b, n, C, io, form, seed=1)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_long_sequences_in_segments(io, form):
    n, C = 8 * 512 * 2 + 77, 10
    assert ssmv.ssm_gated_recurrence_workspace(2, C, n) > 0
    _check_forward(2, n, C, io, form, seed=2, lens=[n, 4500], slow=True)
    _check_forward(2, n, C, io, form, seed=3, in_place=True, slow=True)
    _check_backward(2, n, C, io, form, seed=2, lens=[n, 4500], slow=True)
    _check_backward(3, n, C, io, form, seed=3, lens=[0, n - 1, 1])
    _check_backward(1, n, C, io, form, seed=3, dh=False)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_ragged_and_empty_sequences(io, form):
    for n in (1, 150):
        lens = [n, 0, 1, min(n, 64), min(n, 65), n - 1, -4, 999]
        _check_forward(8, n, 40, io, form, lens=lens)
        _check_forward(8, n, 40, io, form, lens=lens, in_place=True)
        _check_backward(8, n, 40, io, form, lens=lens)
    _check_backward(3, 20, 40, io, form, lens=[0, 0, 0])
    _check_backward(70, 20, 12, io, form, lens=[k % 21 for k in range(70)])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 90])
def test_rows_of_other_beams(io, n):
    _check_forward(6, n, 48, io, "lru", src=[2, 2, 0, -1, 3, 77], rows_in=4)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("wide", [(0, 8), (8, 8), (3, 2), (1, 0)])
def test_strides(io, wide):
    _check_forward(2, 80, 33, io, "lru", wide=wide)
    _check_forward(4, 1, 32, io, "mix", wide=wide)
    _check_backward(2, 80, 33, io, "lru", wide=wide)
    _check_backward(2, 80, 32, io, "mix", wide=wide)


def test_gradients_not_wanted():
    names = ("dx", "df", "di", "dz", "dA", "df_bias", "di_bias", "dh_in")
    for k in names:
        _check_backward(2, 100, 24, "bf16", "lru", only=(k,))
    _check_backward(2, 100, 24, "f32", "mix", dh=False)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_gates_far_from_the_middle(io, form):
    """Sigmoids that are 0 or 1 in fp32 or near it, decays that are 1 or 0: finite everywhere, and within the bounds."""
    b, n, C = 2, 66, 24
    t, up = _inputs(b, n, C, io, form, 7)
    far = torch.tensor([-200.0, -90.0, -60.0, -20.0, -12.0, 12.0, 20.0, 60.0, 90.0, 200.0])
    g = gen(9)
    for k in ("f", "i", "z"):
        t[k] = far[torch.randint(0, len(far), (b, n, C), generator=g)].to(IO[io])
    if form == "lru":
        t["A"][:6] = torch.tensor([-1e-8, -1e-30, -50.0, -1e4, -1e-3, -1.0])
    want_y, _, want_h, _ = gated_forward(**t)
    y, h, s, d = _call(t, b, n, C, io, form)
    check(h, want_h, "f32", "h")
    check(y, want_y, io, "y")
    want = gated_backward(**t, **up)
    out = {k: torch.empty(w.v.shape, dtype=IO[io] if w.v.dim() == 3 else torch.float32, device="cuda") for k, w in want.items()}
    ssmv.ssm_gated_recurrence_backward(**{k: v for k, v in d.items() if k != "h_in"}, states=s, dy=cuda(up["dy"]), dh_out=cuda(up["dh_out"]), **out, batch=b, channels=C, L=n, io=io,
                                       form=form, workspace=_space(ssmv.ssm_gated_recurrence_backward_workspace(b, C, n)))
    for k, v in out.items():
        assert bool(torch.isfinite(v.float()).all()), k
        check(v, want[k], io if v.dim() == 3 else "f32", k)


def test_decays_of_zero_and_infinity():
    """A = 0 keeps the state and takes nothing in; A = -inf forgets at every token."""
    b, n, C = 2, 70, 4
    t, up = _inputs(b, n, C, "f32", "lru", 3, gate=0, inp=0)
    t["A"] = torch.tensor([0.0, -float("inf"), 0.0, -float("inf")])
    y, h, s, d = _call(t, b, n, C, "f32", "lru")
    assert torch.equal(h[:, ::2].cpu(), t["h_in"][:, ::2]) and torch.equal(y[..., ::2].cpu(), t["h_in"][:, None, ::2].expand(b, n, 2))
    assert torch.equal(y[..., 1::2].cpu(), t["x"][..., 1::2])
    out = dict(dx=torch.empty(b, n, C, device="cuda"), df=torch.empty(b, n, C, device="cuda"), dA=torch.empty(C, device="cuda"), dh_in=torch.empty(b, C, device="cuda"))
    ssmv.ssm_gated_recurrence_backward(x=d["x"], f=d["f"], A=d["A"], f_bias=d["f_bias"], states=s, dy=cuda(up["dy"]), dh_out=cuda(up["dh_out"]), **out, batch=b, channels=C, L=n,
                                       io="f32", form="lru", workspace=_space(ssmv.ssm_gated_recurrence_backward_workspace(b, C, n)))
    assert all(bool(torch.isfinite(v).all()) for v in out.values())
    assert bool((out["dA"] == 0).all()) and bool((out["df"] == 0).all()) and bool((out["dx"][..., ::2] == 0).all()) and bool((out["dh_in"][:, 1::2] == 0).all())
    up["dy"][:, -1] += up["dh_out"]
    assert torch.equal(out["dx"][..., 1::2].cpu(), up["dy"][..., 1::2])


@pytest.mark.parametrize("form", FORMS)
def test_two_calls_continue_one(form):
    """Pieces of a sequence one after the other, the last of them single tokens, forwards, and backwards by dh_in and dh_out: within twice the bound of one call."""
    b, C, n = 2, 50, 200
    t, up = _inputs(b, n, C, "f32", form, 5)
    want_y, _, want_h, _ = gated_forward(**t)
    want = gated_backward(**t, **up)
    d = {k: cuda(v) for k, v in t.items()}
    cut, at, h, parts = [64, 33, 1, 70, 31, 1], 0, d["h_in"], []
    for m in cut:
        piece = {k: d[k][:, at:at + m].contiguous() for k in ("x", "f", "i", "z")}
        y, nxt, s = torch.empty(b, m, C, device="cuda"), torch.empty(b, C, device="cuda"), torch.empty(b, (m + 63) // 64, C, device="cuda")
        vec = {k: d[k] for k in ("A", "f_bias", "i_bias")}
        ssmv.ssm_gated_recurrence(**piece, **vec, h_in=h, h_out=nxt, states=s, y_out=y, batch=b, channels=C, L=m, io="f32", form=form)
        parts.append((at, m, piece, vec, s, y))
        h, at = nxt, at + m
    for q in (want_y, want_h, *want.values()):
        q.e *= 2
    check(torch.cat([p[5] for p in parts], 1), want_y, "f32", "y")
    check(h, want_h, "f32", "h")
    dh, grads = cuda(up["dh_out"]), []
    for at, m, piece, vec, s, _ in reversed(parts):
        out = dict(dx=torch.empty(b, m, C, device="cuda"), df=torch.empty(b, m, C, device="cuda"), di=torch.empty(b, m, C, device="cuda"), dz=torch.empty(b, m, C, device="cuda"),
                   dh_in=torch.empty(b, C, device="cuda"), df_bias=torch.empty(C, device="cuda"))
        ssmv.ssm_gated_recurrence_backward(**piece, **vec, states=s, dy=cuda(up["dy"][:, at:at + m].contiguous()), dh_out=dh, **out, batch=b, channels=C, L=m, io="f32", form=form,
                                           workspace=_space(ssmv.ssm_gated_recurrence_backward_workspace(b, C, m)))
        dh = out["dh_in"]
        grads.insert(0, out)
    check(dh, want["dh_in"], "f32", "dh_in")
    for k in ("dx", "df", "di", "dz"):
        check(torch.cat([o[k] for o in grads], 1), want[k], "f32", k)
    check(sum(o["df_bias"] for o in grads), want["df_bias"], "f32", "df_bias")


def test_gradient_against_differences():
    """Differences of fp32 forward calls along random directions: the loss, of 4200 terms of size 1 that are each off by at most 2e-5, is off by 4e-2 at the very most over a
    step of 2^-4 both ways, and by far less in the mean: 0.7; the step's square / 6 times the third derivative adds less than 0.3."""
    b, n, C = 2, 70, 30
    t, up = _inputs(b, n, C, "f32", "lru", 6)
    got = _check_backward(b, n, C, "f32", "lru", seed=6)
    names = dict(dx="x", df="f", di="i", dz="z", dA="A", df_bias="f_bias", di_bias="i_bias", dh_in="h_in")

    def loss(moved):
        y, h, _, _ = _call(moved, b, n, C, "f32", "lru", states=False)
        return float((y.cpu().double() * up["dy"]).sum() + (h.cpu().double() * up["dh_out"]).sum())

    g = gen(12)
    for k, name in names.items():
        way = torch.randn(t[name].shape, generator=g)
        way = way / way.norm() * (4 if k != "dA" else t["A"].abs().min() * 8)
        step = 2.0 ** -4
        diff = (loss({**t, name: t[name] + step * way}) - loss({**t, name: t[name] - step * way})) / (2 * step)
        assert abs(diff - float((got[k].cpu().double() * way).sum())) < 1.0, k


def test_same_bits_again():
    one, two = (_check_backward(5, 200, 64, "bf16", "lru", seed=8) for _ in range(2))
    assert all(torch.equal(one[k], two[k]) for k in one)


@pytest.mark.parametrize("n,C", [(1, 96), (150, 96), (8300, 6)])
def test_captured_and_on_another_stream(n, C):
    b = 2
    t, up = _inputs(b, n, C, "bf16", "lru", 8)
    d, u = {k: cuda(v) for k, v in t.items()}, {k: cuda(v) for k, v in up.items()}
    s, y, h = torch.zeros(b, (n + 63) // 64, C, device="cuda"), torch.zeros_like(d["x"]), torch.zeros(b, C, device="cuda")
    out = dict(dx=torch.zeros_like(y), df=torch.zeros_like(y), di=torch.zeros_like(y), dz=torch.zeros_like(y), dA=torch.zeros(C, device="cuda"), df_bias=torch.zeros(C, device="cuda"),
               di_bias=torch.zeros(C, device="cuda"), dh_in=torch.zeros(b, C, device="cuda"))
    w1, w2 = _space(ssmv.ssm_gated_recurrence_workspace(b, C, n)), _space(ssmv.ssm_gated_recurrence_backward_workspace(b, C, n))

    def both():
        ssmv.ssm_gated_recurrence(**d, h_out=h, states=s, y_out=y, batch=b, channels=C, L=n, io="bf16", form="lru", workspace=w1)
        ssmv.ssm_gated_recurrence_backward(**{k: v for k, v in d.items() if k != "h_in"}, **u, states=s, **out, batch=b, channels=C, L=n, io="bf16", form="lru", workspace=w2)

    every = dict(out, y=y, h=h, s=s)
    both()
    torch.cuda.synchronize()
    eager = {k: v.clone() for k, v in every.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(every[k], eager[k]) for k in every)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(3):
        d["x"].copy_(cuda(t["x"]) * (turn + 1))
        for v in every.values():
            v.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in every.items()}
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(every[k], got[k]) for k in every), turn
