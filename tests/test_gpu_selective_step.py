"""ssm_selective_step on the GPU against one token of the recurrence in 64 bits."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _decode import IO, check_within, cuda, gen, randn, scan_reference, strided

pytestmark = pytest.mark.gpu


def _run(io, mode, rows, H, P, N, G=1, soft=True, gate=True, src=None, rows_in=None, in_place=False, no_state=False, wide=None, seed=0):
    g = gen(seed)
    A = -(torch.arange(1, N + 1) + (torch.rand(H, N, generator=g) - 0.5) * 0.5) if mode == "diag" else -torch.exp(torch.rand(H, generator=g) * 2.7)
    dt = randn(g, rows, H) - 4.0
    s = dict(x=randn(g, rows, H * P, io=io), dt=(dt if soft else torch.nn.functional.softplus(dt)).to(IO[io]), B=(randn(g, rows, G * N) / N ** 0.5).to(IO[io]),
             C=(randn(g, rows, G * N) / N ** 0.5).to(IO[io]), z=randn(g, rows, H * P, io=io) if gate else None)
    D, bias = randn(g, H), torch.rand(H, generator=g) - 0.5 if soft else None
    h_in = None if no_state else randn(g, rows_in or rows, H, P, N) * 0.3
    src = None if src is None else torch.tensor(src, dtype=torch.int32)
    y_ref, ey, h_ref, eh = scan_reference(s["x"].view(rows, 1, H, P), s["dt"].view(rows, 1, H), A, s["B"].view(rows, 1, G, N), s["C"].view(rows, 1, G, N), D, io,
                                          bias, soft, s["z"].view(rows, 1, H, P) if gate else None, h_in, src)
    y = torch.full((rows, H * P), 7.0, dtype=IO[io], device="cuda")
    strides = {}
    if wide:
        s = {k: None if v is None else strided(v, *(wide if k not in "BC" else (2, 4))) for k, v in s.items()}
        y = strided(y, *wide, fill=5.0)
        strides = {k + "_stride": v.stride(0) for k, v in (("x", s["x"]), ("dt", s["dt"]), ("b", s["B"]), ("c", s["C"]), ("y", y))}
        strides["z_stride"] = s["z"].stride(0) if gate else 0
    d = {k: cuda(v) for k, v in s.items()}
    dh = cuda(h_in)
    h_out = dh if in_place else torch.full((rows, H, P, N), 7.0, device="cuda")
    ssmv.ssm_selective_step(x=d["x"], dt=d["dt"], A=A.cuda(), Bm=d["B"], Cm=d["C"], D=D.cuda(), y_out=y, h_in=dh, h_out=h_out, rows=rows, nheads=H, headdim=P,
                            dstate=N, ngroups=G, io=io, a_mode=mode, dt_bias=cuda(bias), dt_softplus=soft, z=d["z"], src_row=cuda(src), **strides)
    torch.cuda.synchronize()
    check_within(y, y_ref.reshape(rows, H * P), ey.reshape(rows, H * P), "y")
    check_within(h_out, h_ref, eh, "state")
    if wide:
        parent = y._base.cpu()
        assert bool((parent[..., :wide[0]] == 5.0).all()) and bool((parent[..., wide[0] + H * P:] == 5.0).all())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("N", [16, 32, 64])
@pytest.mark.parametrize("rows", [1, 3, 8, 21])
def test_diagonal(io, N, rows):
    _run(io, "diag", rows, 200, 1, N, seed=N + rows)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,P,N,G", [(4, 16, 16, 1), (6, 5, 32, 3), (8, 64, 64, 2), (5, 48, 128, 5), (2, 33, 256, 1), (1, 1, 16, 1)])
@pytest.mark.parametrize("rows", [1, 10])
def test_one_decay_per_head(io, H, P, N, G, rows):
    _run(io, "scalar", rows, H, P, N, G, seed=H + P)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("mode,H,P,N", [("diag", 90, 1, 16), ("scalar", 3, 20, 64)])
def test_rows_strides_and_pieces(io, mode, H, P, N):
    for rows in (6, 9):
        _run(io, mode, rows, H, P, N, src=[2, 2, 0, -1, 3, 77, 1, 1, 0][:rows], rows_in=4)
        _run(io, mode, rows, H, P, N, in_place=True)
        _run(io, mode, rows, H, P, N, no_state=True)
        _run(io, mode, rows, H, P, N, soft=False, gate=False)
        for wide in ((0, 8), (3, 2)):
            _run(io, mode, rows, H, P, N, wide=wide)


def test_steps_follow_a_prompt():
    """A prompt by the scan and its tokens one by one end in the same state."""
    g = gen(4)
    b, n, C, N = 2, 20, 96, 16
    x, dt, B, Cm = randn(g, b, n, C).cuda(), (randn(g, b, n, C) - 4).cuda(), randn(g, b, n, N).cuda() / 4, randn(g, b, n, N).cuda() / 4
    A, D = (-torch.rand(C, N, generator=g) * 16 - 0.5).cuda(), randn(g, C).cuda()
    y, h = torch.empty_like(x), torch.empty(b, C, N, device="cuda")
    size = ssmv.ssm_selective_scan_workspace(b, C, N, n)
    ssmv.ssm_selective_scan(x=x, dt=dt, A=A, Bm=B, Cm=Cm, D=D, y_out=y, batch=b, channels=C, dstate=N, L=n, io="f32", dt_softplus=True, h_out=h,
                            workspace=torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
    hs, ys = torch.zeros_like(h), torch.empty_like(y)
    for t in range(n):
        out = torch.empty(b, C, device="cuda")
        ssmv.ssm_selective_step(x=x[:, t].contiguous(), dt=dt[:, t].contiguous(), A=A, Bm=B[:, t].contiguous(), Cm=Cm[:, t].contiguous(), D=D, y_out=out, h_in=hs,
                                h_out=hs, rows=b, nheads=C, headdim=1, dstate=N, io="f32", a_mode="diag", dt_softplus=True)
        ys[:, t] = out
    _, ey, _, eh = scan_reference(x.cpu()[..., None], dt.cpu(), A.cpu(), B.cpu()[:, :, None], Cm.cpu()[:, :, None], D.cpu(), "f32", None, True)
    check_within(ys, y.cpu().double(), 2 * ey[..., 0], "y")
    check_within(hs, h.cpu().double(), 2 * eh[:, :, 0], "state")


@pytest.mark.parametrize("mode,H,P,N", [("diag", 90, 1, 16), ("scalar", 6, 20, 64)])
def test_a_decay_that_forgets_everything(mode, H, P, N):
    """A of -inf: what a step > 0 finds is gone to the last bit, and a step of 0 leaves the state as it is."""
    g = gen(8)
    rows, C = 5, H * P
    h = randn(g, rows, H, P, N).cuda()
    A = torch.full((H, N) if mode == "diag" else (H,), -float("inf"), device="cuda")
    dt = torch.rand(rows, H, generator=g) + 0.1
    dt[:, ::2] = 0.0
    x, B, Cm = randn(g, rows, C).cuda(), randn(g, rows, N).cuda(), randn(g, rows, N).cuda()
    out = {}
    for name, start in (("kept", h), ("empty", None)):
        y, to = torch.empty(rows, C, device="cuda"), torch.empty_like(h)
        ssmv.ssm_selective_step(x=x, dt=dt.cuda(), A=A, Bm=B, Cm=Cm, D=torch.zeros(H, device="cuda"), y_out=y, h_in=start, h_out=to, rows=rows, nheads=H, headdim=P,
                                dstate=N, io="f32", a_mode=mode)
        out[name] = to.cpu()
    assert torch.equal(out["kept"][:, ::2], h.cpu()[:, ::2])
    assert torch.equal(out["kept"][:, 1::2], out["empty"][:, 1::2]) and bool(torch.isfinite(out["empty"]).all())


@pytest.mark.parametrize("mode,H,P,N", [("diag", 90, 1, 16), ("scalar", 6, 20, 64)])
def test_the_least_step_that_forgets(mode, H, P, N):
    """A of -inf and a step of 2^-120: nothing of the start is left, to the last bit."""
    g = gen(9)
    rows, C = 5, H * P
    h = randn(g, rows, H, P, N).cuda()
    A = torch.full((H, N) if mode == "diag" else (H,), -float("inf"), device="cuda")
    x, B, Cm = randn(g, rows, C).cuda(), randn(g, rows, N).cuda(), randn(g, rows, N).cuda()
    out = []
    for start in (h, None):
        y, to = torch.empty(rows, C, device="cuda"), torch.empty_like(h)
        ssmv.ssm_selective_step(x=x, dt=torch.full((rows, H), 2.0 ** -120, device="cuda"), A=A, Bm=B, Cm=Cm, D=torch.zeros(H, device="cuda"), y_out=y, h_in=start, h_out=to,
                                rows=rows, nheads=H, headdim=P, dstate=N, io="f32", a_mode=mode)
        out.append((y.cpu(), to.cpu()))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
