"""The backward pass of ssmv_block_norm in every shape of its workgroups - several rows to one, a row to one, 9 to 12 waves, two vectors a thread, 9 to 16 waves -, with one row and with several rows for
every workgroup to walk over.  The launches are looked at, so that a size that another rule lays out in another way fails here."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _harness import launches
from _layers import EPS, check, cuda, norm_backward
from test_gpu_block_norm import TYPES, _inputs

pytestmark = pytest.mark.gpu


def _call(t, up, rows, C, io, res_io, spare=0):
    """(the call, what it writes, its workspace)."""
    d = {k: cuda(v) for k, v in {**t, **up}.items()}
    like = lambda v: None if v is None else torch.full_like(v, 7.0)
    out = dict(dx=like(d["x"]), dz=like(d["z"]), dres=like(d["res"]), dpost=like(d["post"]), dscale=like(d["scale"]), dpre=like(d["pre"]))
    work = torch.full((ssmv.ssmv_block_norm_backward_workspace(rows, C) + spare,), 0xFF, dtype=torch.uint8, device="cuda")      # NaN
    call = lambda: ssmv.ssmv_block_norm_backward(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], dr=d["dr"], dn=d["dn"], dx=out["dx"],
                                                 dz=out["dz"], dres=out["dres"], dpost_wgt=out["dpost"], dch_scale=out["dscale"], dpre_wgt=out["dpre"], rows=rows, channels=C, io=io,
                                                 res_io=res_io, eps=EPS, res_scale=0.5, workspace=work)
    return call, {k: v for k, v in out.items() if v is not None}, work


def _check(rows, C, io, res_io, workgroups, waves, seed=0):
    t, kw, up = _inputs(rows, C, io, res_io, seed)
    call, out, work = _call(t, up, rows, C, io, res_io)
    assert launches(call) == [(workgroups, 64 * waves), (3 * -(-C // 32), 1024)]
    call()
    torch.cuda.synchronize()
    want = norm_backward(**t, **kw, **up)
    assert set(want) == set(out)
    for k, v in out.items():
        check(v, want[k], "f32" if v.dim() == 1 else res_io if k == "dres" else io, k)


# channels, waves of a row, workgroups at most
WIDE = [(2056, 5, 512), (4096, 8, 512), (4104, 9, 256), (5120, 10, 256), (5121, 11, 256), (6144, 12, 256), (6152, 7, 256), (8192, 8, 256), (8200, 9, 256), (12301, 13, 256), (16384, 16, 256)]


@pytest.mark.parametrize("io,res_io", TYPES)
@pytest.mark.parametrize("C,waves,most", WIDE)
def test_a_row_to_a_workgroup(io, res_io, C, waves, most):
    _check(4, C, io, res_io, 4, waves, seed=C)


@pytest.mark.parametrize("io,res_io", TYPES)
@pytest.mark.parametrize("C,waves,most", [w for w in WIDE if w[0] in (2056, 4096, 5120, 6144, 8192, 8200)])
def test_rows_one_after_the_other(io, res_io, C, waves, most):
    """Three rows for some workgroups and two for the others: the buffers that even and odd rows change between are used again, and the sums go on from row to row."""
    _check(2 * most + 37, C, io, res_io, most, waves, seed=C)


def test_the_widest_rows_one_after_the_other():
    _check(2 * 256 + 5, 16384, "bf16", "f32", 256, 16)


@pytest.mark.parametrize("io,res_io", TYPES)
@pytest.mark.parametrize("C,per_wg,waves", [(40, 8, 8), (513, 4, 8), (1025, 2, 6), (1600, 2, 8)])
def test_several_rows_to_a_workgroup(io, res_io, C, per_wg, waves):
    """Three groups of rows for some workgroups, two for the others, the last one not whole."""
    _check(2 * 512 * per_wg + 3 * per_wg + 1, C, io, res_io, 512, waves, seed=C)


@pytest.mark.parametrize("io,res_io", TYPES)
@pytest.mark.parametrize("C", [40, 600, 1100, 5120, 8200])
def test_a_row_depends_on_no_other(io, res_io, C):
    """The gradients of rows next to rows of NaN and infinities, and of some of the rows alone: the same bits."""
    rows, bad = 21, [2, 7, 12, 20]
    t, _, up = _inputs(rows, C, io, res_io, C)
    def run(t, up, n):
        call, out, _ = _call(t, up, n, C, io, res_io)
        call()
        torch.cuda.synchronize()
        return {k: out[k].cpu() for k in ("dx", "dz", "dres")}
    clean = run(t, up, rows)
    part = {k: v[3:14] if v is not None and v.dim() == 2 else v for k, v in t.items()}
    alone = run({k: None if v is None else v.contiguous() for k, v in part.items()}, {k: v[3:14].contiguous() for k, v in up.items()}, 11)
    assert all(torch.equal(alone[k], clean[k][3:14]) for k in clean)
    t, up = {k: None if v is None else v.clone() for k, v in t.items()}, {k: v.clone() for k, v in up.items()}
    t["x"][2, 5], t["res"][7, 0], up["dn"][12, C - 1], up["dr"][20, 1] = float("nan"), float("inf"), float("nan"), float("-inf")
    mixed = run(t, up, rows)
    keep = [i for i in range(rows) if i not in bad]
    assert all(torch.equal(mixed[k][keep], clean[k][keep]) for k in clean)
    assert all(not bool(torch.isfinite(mixed["dx"][i].float()).all()) for i in bad)


@pytest.mark.parametrize("rows,C", [(1, 5), (9, 40), (700, 600), (3, 2056), (600, 5120), (300, 8200)])
def test_workspaces_are_not_left(rows, C):
    """What lies behind the bytes that a call asks for is left as it was."""
    t, _, up = _inputs(rows, C, "bf16", "f32", 1)
    call, _, work = _call(t, up, rows, C, "bf16", "f32", spare=4096)
    work[-4096:] = 0x5A
    call()
    torch.cuda.synchronize()
    assert bool((work[-4096:] == 0x5A).all())
