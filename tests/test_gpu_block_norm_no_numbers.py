"""Infinities in the backward pass of ssmv_block_norm: the gradients of vectors, which are added up over rows, may only hold what rows that are there bring.  A workgroup of several rows goes through
the last ones with waves that have none; 0 times what those hold would be no number where it is infinite."""
import math

import pytest
import torch

import paper_2408_15237_amd as ssmv
from _layers import EPS, IO, check, cuda, norm_backward
from test_gpu_block_norm import _inputs as norm_inputs

pytestmark = pytest.mark.gpu
INF = float("inf")


def _norm_gradients(t, up, rows, C, io, in_place=False):
    """dpost, dscale and dpre, and dx and dres as stored."""
    d = {k: cuda(v) for k, v in {**t, **up}.items()}
    like = lambda v: torch.full_like(v, 7.0)
    dx, dres = (d["dn"], d["dr"]) if in_place else (like(d["x"]), like(d["res"]))
    vec = {k: torch.full((C,), 7.0, device="cuda") for k in ("post", "scale", "pre") if d[k] is not None}
    work = torch.full((ssmv.ssmv_block_norm_backward_workspace(rows, C) // 4,), float("nan"), device="cuda")
    ssmv.ssmv_block_norm_backward(x=d["x"], z=d["z"], res=d["res"], post_wgt=d["post"], ch_scale=d["scale"], pre_wgt=d["pre"], dr=d["dr"], dn=d["dn"], dx=dx, dres=dres,
                                  dpost_wgt=vec.get("post"), dch_scale=vec.get("scale"), dpre_wgt=vec.get("pre"), rows=rows, channels=C, io=io, eps=EPS, res_scale=0.5, workspace=work)
    torch.cuda.synchronize()
    return {k: v.cpu() for k, v in vec.items()}, dx.cpu(), dres.cpu()


# rows that leave waves of the last workgroup without one, and that leave none: 8 rows a workgroup, 4, and 1
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", [(1, 40), (9, 40), (16, 40), (9, 3), (4097, 40), (5, 600), (8, 600), (2049, 600), (3, 2100)])
def test_an_infinite_gradient_of_the_last_row(io, rows, C):
    """An infinite dr makes that channel's sums infinite, by the sign of what it is multiplied with; the other channels' stay as they are.  The same of dn and the norm ahead."""
    at = C // 2
    t, _, up = norm_inputs(rows, C, io, io, rows + C)
    want = norm_backward(**t, alpha=0.5, dr=up["dr"].clone().index_put_((torch.tensor(rows - 1), torch.tensor(at)), torch.tensor(0.0, dtype=IO[io])), dn=None)
    p_sign = math.copysign(1.0, float(t["x"][-1, at]) * float(t["z"][-1, at]))
    others = torch.arange(C) != at
    up["dr"][-1, at] = INF
    got, _, _ = _norm_gradients(t, dict(dr=up["dr"], dn=None), rows, C, io)
    for k, sign in (("post", math.copysign(1.0, float(t["scale"][at])) * p_sign), ("scale", math.copysign(1.0, float(t["post"][at])) * p_sign)):
        assert float(got[k][at]) == sign * INF, (k, float(got[k][at]))
        check(got[k][others], type(want["dpost"])(want["d" + k].v[others], want["d" + k].e[others]), "f32", k)
    assert bool((got["pre"] == 0).all())
    t = dict(t, z=None, post=None, scale=None)
    want = norm_backward(**t, alpha=0.5, dr=None, dn=up["dn"].clone().index_put_((torch.tensor(rows - 1), torch.tensor(at)), torch.tensor(0.0, dtype=IO[io])))
    up["dn"][-1, at] = INF
    got, _, _ = _norm_gradients(t, dict(dr=None, dn=up["dn"]), rows, C, io)
    r = float(t["res"][-1, at]) + 0.5 * float(t["x"][-1, at])
    assert float(got["pre"][at]) == math.copysign(INF, r)
    check(got["pre"][others], type(want["dpre"])(want["dpre"].v[others], want["dpre"].e[others]), "f32", "pre")


@pytest.mark.parametrize("rows,C", [(9, 40), (4097, 40), (5, 600), (2049, 600)])
def test_gradients_that_overflow_in_place(rows, C):
    """dx over dn and dres over dr, both stored as infinities in the last row: the gradient of pre_wgt, which is finite, has the bits of the call that is not in place."""
    t, _, up = norm_inputs(rows, C, "bf16", "bf16", rows + C, gate=0, post=0, scale=0)
    t["x"][-1] *= 1e-3
    t["res"][-1] *= 1e-3
    up["dn"][-1] *= 1e37                                            # times rho, about 200: beyond fp32
    apart, dx, dres = _norm_gradients(t, up, rows, C, "bf16")
    over, dx2, dres2 = _norm_gradients(t, up, rows, C, "bf16", in_place=True)
    assert bool(torch.isinf(dx[-1]).any()) and bool(torch.isfinite(dx[:-1]).all())
    assert bool(torch.isfinite(apart["pre"]).all()) and torch.equal(apart["pre"], over["pre"])
    for a, b in ((dx, dx2), (dres, dres2)):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    want = norm_backward(**t, alpha=0.5, **up)
    check(apart["pre"], want["dpre"], "f32", "pre")
