"""ssm_selective_scan on the GPU against the token-by-token recurrence in 64 bits, with bounds that follow the arithmetic."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _decode import IO, check_within, cuda, gen, randn, scan_reference, strided

pytestmark = pytest.mark.gpu


def _inputs(io, b, n, C, N, soft=True, gate=True, rows_in=None, resume=True, seed=0):
    g = gen(seed)
    dt = randn(g, b, n, C) - 4.0
    dt = (dt if soft else torch.nn.functional.softplus(dt)).to(IO[io])
    A = -(torch.arange(1, N + 1) + (torch.rand(C, N, generator=g) - 0.5) * 0.5)
    return dict(x=randn(g, b, n, C, io=io), dt=dt, A=A, B=(randn(g, b, n, N) / N ** 0.5).to(IO[io]), C=(randn(g, b, n, N) / N ** 0.5).to(IO[io]), D=randn(g, C),
                dt_bias=torch.rand(C, generator=g) - 0.5 if soft else None, z=randn(g, b, n, C, io=io) if gate else None,
                h_in=randn(g, rows_in or b, C, N) * 0.1 if resume else None)


def _reference(s, io, soft, src=None, lens=None):
    b, n, C = s["x"].shape
    y, ey, h, eh = scan_reference(s["x"][..., None], s["dt"], s["A"], s["B"][:, :, None], s["C"][:, :, None], s["D"], io, s["dt_bias"], soft,
                                  None if s["z"] is None else s["z"][..., None],
                                  None if s["h_in"] is None else s["h_in"][:, :, None, :], src, lens)
    return y[..., 0], ey[..., 0], h[:, :, 0], eh[:, :, 0]


def call(d, io, b, n, C, N, soft, y, h_out, src=None, lens=None, **strides):
    size = ssmv.ssm_selective_scan_workspace(b, C, N, n)
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda") if size else None       # as NaN as bytes can be
    ssmv.ssm_selective_scan(x=d["x"], dt=d["dt"], A=d["A"], Bm=d["B"], Cm=d["C"], D=d["D"], y_out=y, batch=b, channels=C, dstate=N, L=n, io=io,
                            dt_bias=d["dt_bias"], dt_softplus=soft, z=d["z"], h_in=d["h_in"], h_out=h_out, src_row=src, seq_len=lens, workspace=ws, **strides)


def _run(io, b, n, C, N, soft=True, gate=True, resume=True, src=None, rows_in=None, lens=None, in_place=False, wide=None, seed=0):
    s = _inputs(io, b, n, C, N, soft, gate, rows_in, resume, seed)
    src = None if src is None else torch.tensor(src, dtype=torch.int32)
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32)
    y_ref, ey, h_ref, eh = _reference(s, io, soft, src, lens)
    if lens is not None:                                          # what lies behind a sequence's tokens must not matter
        for i, m in enumerate(lens.tolist()):
            for k in ("x", "dt", "B", "C", "z"):
                if s[k] is not None:
                    s[k][i, max(m, 0):] = float("nan")
    y = torch.full((b, n, C), 7.0, dtype=IO[io], device="cuda")
    strides = {}
    if wide:
        for k in ("x", "dt", "z"):
            if s[k] is not None:
                s[k] = strided(s[k], *wide)
        s["B"], s["C"], y = strided(s["B"], 4, N + 2), strided(s["C"], N + 2, 4), strided(y, *wide, fill=5.0)
        strides = dict(x_stride=C + sum(wide), dt_stride=C + sum(wide), z_stride=C + sum(wide) if gate else 0, y_stride=C + sum(wide), b_stride=2 * N + 6, c_stride=2 * N + 6)
    d = {k: cuda(v) for k, v in s.items()}
    h_out = d["h_in"] if in_place else torch.full((b, C, N), 7.0, device="cuda")
    call(d, io, b, n, C, N, soft, y, h_out, cuda(src), cuda(lens), **strides)
    torch.cuda.synchronize()
    got = y.cpu()
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        check_within(got[i, :m], y_ref[i, :m], ey[i, :m], "y of sequence %d" % i)
        assert torch.equal(got[i, m:], torch.full_like(got[i, m:], 7.0)), "written behind the sequence's tokens"
    check_within(h_out, h_ref, eh, "state")
    if wide:
        parent = y._base.cpu()
        assert bool((parent[..., :wide[0]] == 5.0).all()) and bool((parent[..., wide[0] + C:] == 5.0).all())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 31, 32, 33, 64, 95, 200])
def test_lengths(io, n):
    _run(io, 2, n, 72, 16, seed=n)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("N", [16, 32, 64])
@pytest.mark.parametrize("C", [1, 7, 64, 68, 130])
def test_channel_counts_and_state_sizes(io, N, C):
    _run(io, 2, 37, C, N, seed=C + N)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("soft", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("resume", [False, True])
def test_optional_pieces(io, soft, gate, resume):
    _run(io, 1, 41, 64, 16, soft, gate, resume, seed=3)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("N", [16, 64])
def test_ragged_and_empty_prompts(io, N):
    _run(io, 7, 70, 72, N, lens=[70, 0, 1, 32, 33, 64, -3])
    _run(io, 3, 70, 72, N, lens=[99, 5, 40], in_place=True)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_rows_of_other_sequences(io):
    _run(io, 6, 34, 72, 16, src=[2, 2, 0, -1, 3, 77], rows_in=4)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("wide", [(0, 8), (8, 8), (3, 2), (1, 0)])
def test_strides(io, wide):
    _run(io, 2, 45, 72, 16, wide=wide)
    _run(io, 2, 45, 72, 64, wide=wide)


@pytest.mark.parametrize("io,b,n,C,N", [("bf16", 1, 1500, 192, 16), ("f32", 1, 1027, 72, 16), ("bf16", 2, 700, 72, 32), ("f32", 1, 2050, 8, 64), ("bf16", 1, 640, 70, 64)])
def test_long_prompts_of_few_channels(io, b, n, C, N):
    _run(io, b, n, C, N, seed=n)
    _run(io, b, n, C, N, seed=n + 1, in_place=True)
    _run(io, b, n, C, N, seed=n + 2, resume=False, lens=[n // 3 + 1] * (b - 1) + [n - 1])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_strong_and_vanishing_steps(io):
    """Steps whose decay underflows to zero, and steps so small that softplus is its argument's exponential."""
    b, n, C, N = 1, 66, 64, 16
    s = _inputs(io, b, n, C, N, seed=11)
    g = gen(12)
    s["dt"] = (randn(g, b, n, C) * 30).to(IO[io])
    y_ref, ey, h_ref, eh = _reference(s, io, True)
    d = {k: cuda(v) for k, v in s.items()}
    y, h = torch.empty_like(d["x"]), torch.empty(b, C, N, device="cuda")
    call(d, io, b, n, C, N, True, y, h)
    check_within(y, y_ref, ey, "y")
    check_within(h, h_ref, eh, "state")


def test_two_calls_continue_one_and_the_same_call_gives_the_same_bits():
    io, b, n, C, N = "f32", 2, 150, 72, 16
    s = _inputs(io, b, n, C, N, resume=False, seed=21)
    y_ref, ey, h_ref, eh = _reference(s, io, True)
    d = {k: cuda(v) for k, v in s.items()}
    ys = [torch.empty(b, n, C, device="cuda") for _ in range(2)]
    hs = [torch.empty(b, C, N, device="cuda") for _ in range(2)]
    for y, h in zip(ys, hs):
        call(d, io, b, n, C, N, True, y, h)
    assert torch.equal(ys[0], ys[1]) and torch.equal(hs[0], hs[1])
    parts, h, at = [], None, 0
    for m in (1, 33, 64, 52):
        part = {k: v[:, at:at + m].contiguous() if k in ("x", "dt", "B", "C", "z") else v for k, v in d.items()}
        part["h_in"] = h
        y, h = torch.empty(b, m, C, device="cuda"), torch.empty(b, C, N, device="cuda")
        call(part, io, b, m, C, N, True, y, h)
        parts.append(y)
        at += m
    check_within(torch.cat(parts, 1), y_ref, ey, "y in pieces")
    check_within(h, h_ref, eh, "state in pieces")


def test_on_another_stream_and_in_a_graph():
    io, b, n, C, N = "bf16", 1, 700, 72, 16
    s = _inputs(io, b, n, C, N, seed=31)
    y_ref, ey, h_ref, eh = _reference(s, io, True)
    d = {k: cuda(v) for k, v in s.items()}
    y, h = torch.zeros_like(d["x"]), torch.zeros(b, C, N, device="cuda")
    size = ssmv.ssm_selective_scan_workspace(b, C, N, n)
    ws = torch.zeros(max(size, 16), dtype=torch.uint8, device="cuda")
    kw = dict(x=d["x"], dt=d["dt"], A=d["A"], Bm=d["B"], Cm=d["C"], D=d["D"], y_out=y, batch=b, channels=C, dstate=N, L=n, io=io, dt_bias=d["dt_bias"],
              dt_softplus=True, z=d["z"], h_in=d["h_in"], h_out=h, workspace=ws)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        ssmv.ssm_selective_scan(**kw)
    side.synchronize()
    check_within(y, y_ref, ey, "y on a side stream")
    with torch.cuda.stream(side):
        graph.capture_begin()
        ssmv.ssm_selective_scan(**kw)
        graph.capture_end()
    for _ in range(3):
        y.zero_(), h.zero_(), ws.fill_(0x7F)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_within(y, y_ref, ey, "y of a replay")
        check_within(h, h_ref, eh, "state of a replay")


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("b,n,C,N,lens", [(4, 39, 72, 16, [13, 0, 39, 38]), (2, 21, 9, 64, None), (1, 1333, 64, 32, None)])
def test_a_decay_that_forgets_everything(io, b, n, C, N, lens):
    """A of -inf: exp(dt' A) is 0 at every token, and tokens that fill up the last tile must still leave the state as it is."""
    if n > 1000:
        assert ssmv.ssm_selective_scan_workspace(b, C, N, n) > 0
    s = _inputs(io, b, n, C, N, seed=5)
    s["A"][:, ::3] = -float("inf")
    s["A"][2] = -float("inf")
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32)
    y_ref, ey, h_ref, eh = _reference(s, io, True, None, lens)
    assert bool(torch.isfinite(h_ref).all()) and bool(torch.isfinite(ey).all())
    d = {k: cuda(v) for k, v in s.items()}
    y, h = torch.zeros(b, n, C, dtype=IO[io], device="cuda"), torch.full((b, C, N), 7.0, device="cuda")
    call(d, io, b, n, C, N, True, y, h, None, cuda(lens))
    for i in range(b):
        m = n if lens is None else int(lens[i])
        check_within(y[i, :m], y_ref[i, :m], ey[i, :m], "y of sequence %d" % i)
    check_within(h, h_ref, eh, "state")


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("N", [16, 32, 64])
def test_enough_channels_to_fill_the_chip(io, N):
    """In the widest workgroups: the last one's channels are not whole, nor are the last tokens."""
    _run(io, 64, 11, 1000, N, lens=[11, 3, 0, 10, 1, 7, 11, 8] * 8, seed=N)


@pytest.mark.parametrize("C,N", [(72, 16), (5, 32), (70, 64)])
def test_the_least_step_that_forgets(C, N):
    """A of -inf and steps of 2^-120: nothing of the start is left, to the last bit; after a step of 0 all of it."""
    b, n = 2, 21
    s = _inputs("f32", b, n, C, N, soft=False, gate=False, seed=6)
    s["A"][:] = -float("inf")
    for step, forgets in ((2.0 ** -120, True), (0.0, False)):
        s["dt"][:] = step
        out = []
        for start in (s["h_in"], torch.zeros_like(s["h_in"])):
            d = {k: cuda(v) for k, v in dict(s, h_in=start).items()}
            y, h = torch.zeros(b, n, C, device="cuda"), torch.full((b, C, N), 7.0, device="cuda")
            call(d, "f32", b, n, C, N, False, y, h)
            out.append((y.cpu(), h.cpu()))
        if forgets:
            assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
        else:
            assert torch.equal(out[0][1], s["h_in"])
