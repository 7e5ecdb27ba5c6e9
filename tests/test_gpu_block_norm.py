"""ssmv_block_norm and its gradients on the GPU against the formulas in 64 bits."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _layers import EPS, IO, Num, check, cuda, gen, norm_backward, norm_forward, randn, strided

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]
ALL = dict(x=1, gate=1, post=1, scale=1, pre=1, residual=1)


def _inputs(rows, C, io, res_io, seed, x=1, gate=1, post=1, scale=1, pre=1, residual=1, alpha=0.5):
    g = gen(seed)
    vec = lambda on: 1 + randn(g, C) / 4 if on else None
    t = dict(x=randn(g, rows, C, io=io) if x else None, z=randn(g, rows, C, io=io) if x and gate else None, res=2 * randn(g, rows, C, io=res_io) if residual else None,
             post=vec(x and post), scale=vec(x and scale), pre=vec(pre))
    return t, dict(alpha=alpha), dict(dr=randn(g, rows, C, io=res_io), dn=randn(g, rows, C, io=io))


def _forward(rows, C, io, res_io, seed=0, wide=None, in_place=False, want=("r", "n"), **flags):
    t, kw, _ = _inputs(rows, C, io, res_io, seed, **flags)
    a, sigma, p, r, rho, n = norm_forward(**t, **kw)
    lay = (lambda v: cuda(strided(v, *wide))) if wide else cuda
    st = lambda v: 0 if v is None else v.stride(0)
    d = {k: (lay(v) if k in ("x", "z", "res") and v is not None else cuda(v)) for k, v in t.items()}
    out = lambda io: strided(torch.full((rows, C), 7.0, dtype=IO[io], device="cuda"), *(wide or (0, 0)), fill=5.0)
    r_out = (d["res"] if in_place else out(res_io)) if "r" in want else None
    n_out = out(io) if "n" in want else None
    ssmv.ssmv_block_norm(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], r_out=r_out, n_out=n_out, rows=rows, channels=C, io=io,
                         res_io=res_io, eps=EPS, res_scale=kw["alpha"], x_stride=st(d["x"]), z_stride=st(d["z"]), res_stride=st(d["res"]), r_stride=st(r_out), n_stride=st(n_out))
    torch.cuda.synchronize()
    if r_out is not None:
        check(r_out, r, res_io, "r")
    if n_out is not None:
        check(n_out, n, io, "n")
    if wide and n_out is not None:
        parent = n_out._base.cpu()
        assert bool((parent[:, :wide[0]] == 5).all()) and bool((parent[:, wide[0] + C:] == 5).all())


def _backward(rows, C, io, res_io, seed=0, wide=None, dr=True, dn=True, in_place=False, only=None, **flags):
    t, kw, up = _inputs(rows, C, io, res_io, seed, **flags)
    up = dict(dr=up["dr"] if dr else None, dn=up["dn"] if dn else None)
    want = norm_backward(**t, **kw, **up)
    lay = (lambda v: cuda(strided(v, *wide))) if wide else cuda
    st = lambda v: 0 if v is None else v.stride(0)
    d = {k: (lay(v) if v is not None and v.dim() == 2 else cuda(v)) for k, v in {**t, **up}.items()}
    out = {}
    for k in want:
        if only and k not in only:
            continue
        if k in ("dx", "dz", "dres"):
            out[k] = strided(torch.full((rows, C), 7.0, dtype=IO[res_io if k == "dres" else io], device="cuda"), *(wide or (0, 0)), fill=5.0)
        else:
            out[k] = torch.full((C,), 7.0, device="cuda")
    if in_place:
        out["dres"], out["dx"] = d["dr"], d["dn"]
    work = torch.full((ssmv.ssmv_block_norm_backward_workspace(rows, C) // 4,), float("nan"), device="cuda")
    ssmv.ssmv_block_norm_backward(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], dr=d["dr"], dn=d["dn"], dx=out.get("dx"),
                                  dz=out.get("dz"), dres=out.get("dres"), dpost_wgt=out.get("dpost"), dch_scale=out.get("dscale"), dpre_wgt=out.get("dpre"), rows=rows,
                                  channels=C, io=io, res_io=res_io, eps=EPS, res_scale=kw["alpha"], x_stride=st(d["x"]), z_stride=st(d["z"]), res_stride=st(d["res"]),
                                  dr_stride=st(d["dr"]), dn_stride=st(d["dn"]), dx_stride=st(out.get("dx")), dz_stride=st(out.get("dz")), dres_stride=st(out.get("dres")),
                                  workspace=work)
    torch.cuda.synchronize()
    for k, v in out.items():
        check(v, want[k], "f32" if v.dim() == 1 else res_io if k == "dres" else io, k)
    return out


@pytest.mark.parametrize("io,res_io", TYPES)
@pytest.mark.parametrize("C", [1, 5, 8, 63, 264, 511, 513, 1001, 4096])
def test_channel_counts(io, res_io, C):
    _forward(5, C, io, res_io, seed=C)
    _backward(5, C, io, res_io, seed=C)


@pytest.mark.parametrize("io,res_io", TYPES)
@pytest.mark.parametrize("C", [8192, 8197, 16384])
def test_wide_rows(io, res_io, C):
    _forward(3, C, io, res_io, seed=C)
    _backward(3, C, io, res_io, seed=C)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 511, 513, 1100, 2051])
def test_row_counts(rows):
    """Below, at and above the rows that workgroups of the backward pass walk over."""
    for C in (40, 600):
        _forward(rows, C, "bf16", "f32", seed=rows)
        _backward(rows, C, "bf16", "f32", seed=rows)


@pytest.mark.parametrize("flags", [dict(gate=0), dict(post=0), dict(scale=0), dict(pre=0), dict(residual=0), dict(gate=0, post=0, scale=0), dict(gate=0, post=0, scale=0, pre=0),
                                   dict(x=0), dict(post=0, scale=0, alpha=1.0), dict(alpha=0.0)])
@pytest.mark.parametrize("C", [72, 700])
def test_parts(flags, C):
    for io, res_io in TYPES:
        _forward(9, C, io, res_io, seed=1, **flags, want=("n",) if flags.get("x") == 0 else ("r", "n"))
        _backward(9, C, io, res_io, seed=1, **flags)


@pytest.mark.parametrize("io,res_io", TYPES)
@pytest.mark.parametrize("wide", [(0, 8), (8, 8), (3, 2), (1, 0)])
def test_strides(io, res_io, wide):
    for C in (33, 520):
        _forward(6, C, io, res_io, wide=wide)
        _backward(6, C, io, res_io, wide=wide)


@pytest.mark.parametrize("io,res_io", TYPES)
def test_in_place_and_outputs_not_wanted(io, res_io):
    for C in (100, 1000):
        _forward(7, C, io, res_io, in_place=True)
        _forward(7, C, io, res_io, want=("r",))
        _forward(7, C, io, res_io, want=("n",))
        _backward(700, C, io, res_io, in_place=True)
        _backward(7, C, io, res_io, dr=False)
        _backward(7, C, io, res_io, dn=False)
        for k in ("dx", "dz", "dres", "dpost", "dscale", "dpre"):
            _backward(7, C, io, res_io, only=(k,))


def test_gradient_against_differences():
    """The loss sum(r dr) + sum(n dn) of fp32 forward calls, moved both ways along a random direction of every input: of 2400 terms about 2 in size, each off by about 1e-6 of
    itself (a row's norm: 64 roundings), the sums are off by 5e-3 at the very most, over a step of 2^-6 both ways: 0.16 for each of the difference's ends; the third derivative
    times the step's square / 6 (4e-5) adds less than 0.03."""
    rows, C = 6, 200
    t, kw, up = _inputs(rows, C, "f32", "f32", 4)
    got = _backward(rows, C, "f32", "f32", seed=4)
    names = dict(dx="x", dz="z", dres="res", dpost="post", dscale="scale", dpre="pre")

    def loss(moved):
        d = {k: cuda(v) for k, v in moved.items()}
        r, n = torch.empty(rows, C, device="cuda"), torch.empty(rows, C, device="cuda")
        ssmv.ssmv_block_norm(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], r_out=r, n_out=n, rows=rows, channels=C, io="f32", eps=EPS,
                             res_scale=kw["alpha"])
        return float((r.cpu().double() * up["dr"]).sum() + (n.cpu().double() * up["dn"]).sum())

    g = gen(11)
    for k, name in names.items():
        way = torch.randn(t[name].shape, generator=g)
        way = way / way.norm() * 4
        step = 2.0 ** -6
        diff = (loss({**t, name: t[name] + step * way}) - loss({**t, name: t[name] - step * way})) / (2 * step)
        assert abs(diff - float((got[k].cpu().double() * way).sum())) < 0.35, k


def test_same_bits_again_and_rows_alone():
    """A row does not depend on its neighbours, and no sum on the order in which workgroups run."""
    rows, C = 1500, 320
    one, two = _backward(rows, C, "bf16", "bf16", seed=2), _backward(rows, C, "bf16", "bf16", seed=2)
    assert all(torch.equal(one[k], two[k]) for k in one)


def test_rows_that_are_no_numbers_stay_alone():
    C, rows = 130, 9
    t, kw, _ = _inputs(rows, C, "f32", "f32", 3)
    clean = {k: cuda(v) for k, v in t.items()}
    t["x"][2, 5], t["res"][4, 0], t["z"][6, 1] = float("nan"), float("inf"), float("nan")
    bad = {k: cuda(v) for k, v in t.items()}
    outs = []
    for d in (clean, bad):
        r, n = torch.empty(rows, C, device="cuda"), torch.empty(rows, C, device="cuda")
        ssmv.ssmv_block_norm(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], r_out=r, n_out=n, rows=rows, channels=C, io="f32", eps=EPS,
                             res_scale=kw["alpha"])
        outs.append((r, n))
    keep = [i for i in range(rows) if i not in (2, 4, 6)]
    for a, b in zip(*outs):
        assert torch.equal(a[keep], b[keep])
    assert all(bool(torch.isnan(outs[1][1][i]).any()) for i in (2, 4, 6))


def test_rows_of_zeros():
    C = 48
    zeros, n, r = torch.zeros(3, C, device="cuda"), torch.empty(3, C, device="cuda"), torch.empty(3, C, device="cuda")
    ssmv.ssmv_block_norm(x=zeros, post_wgt=zeros[0], res=zeros, r_out=r, n_out=n, rows=3, channels=C, io="f32")
    assert bool((n == 0).all()) and bool((r == 0).all())


def test_captured_and_on_another_stream():
    rows, C = 900, 256
    t, kw, up = _inputs(rows, C, "bf16", "f32", 6)
    d = {k: cuda(v) for k, v in {**t, **up}.items()}
    out = dict(r=torch.zeros(rows, C, device="cuda"), n=torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda"), dx=torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda"),
               dz=torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda"), dres=torch.zeros(rows, C, device="cuda"), dpost=torch.zeros(C, device="cuda"),
               dscale=torch.zeros(C, device="cuda"), dpre=torch.zeros(C, device="cuda"))
    work = torch.empty(ssmv.ssmv_block_norm_backward_workspace(rows, C), dtype=torch.uint8, device="cuda")

    def both():
        ssmv.ssmv_block_norm(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], r_out=out["r"], n_out=out["n"], rows=rows, channels=C,
                             io="bf16", res_io="f32", eps=EPS, res_scale=kw["alpha"])
        ssmv.ssmv_block_norm_backward(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], dr=d["dr"], dn=d["dn"], dx=out["dx"],
                                      dz=out["dz"], dres=out["dres"], dpost_wgt=out["dpost"], dch_scale=out["dscale"], dpre_wgt=out["dpre"], rows=rows, channels=C, io="bf16",
                                      res_io="f32", eps=EPS, res_scale=kw["alpha"], workspace=work)

    both()
    torch.cuda.synchronize()
    eager = {k: v.clone() for k, v in out.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    assert all(torch.equal(out[k], eager[k]) for k in out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for turn in range(3):
        d["x"].copy_(cuda(t["x"]) * (turn + 1))                    # eager work between the replays
        for v in out.values():
            v.fill_(3.0)
        work.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], got[k]) for k in out), turn
