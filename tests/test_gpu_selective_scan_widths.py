"""ssm_selective_scan in every width of workgroup (64, 32, 16 channels), whole and cut into segments, over several tiles and a part of one:
against the recurrence in 64 bits on a sample of the channels, which are independent of each other.  Every call's launches are looked at, so
that a case that another plan runs in another width fails here."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _decode import IO, check_within, cuda, strided
from _harness import launches
from test_gpu_selective_scan import _inputs, _reference

pytestmark = pytest.mark.gpu

# (dstate, channels of a workgroup, segments of the longest prompt, batch, channels, tokens)
CASES = [(16, 16, 1, 3, 9, 200), (16, 16, 5, 3, 9, 300), (16, 32, 1, 3, 1530, 131), (16, 32, 9, 3, 201, 515), (16, 64, 1, 5, 5001, 75), (16, 64, 11, 3, 777, 700),
         (32, 16, 1, 3, 9, 200), (32, 16, 5, 3, 9, 300), (32, 32, 1, 3, 1530, 131), (32, 32, 5, 3, 501, 300), (32, 64, 1, 5, 5001, 75), (32, 64, 11, 3, 777, 700),
         (64, 16, 1, 3, 501, 200), (64, 16, 4, 3, 9, 200), (64, 32, 1, 3, 1530, 131), (64, 32, 5, 3, 333, 300), (64, 64, 1, 5, 5001, 75), (64, 64, 9, 3, 2999, 515)]
IDS = ["N%d-w%d-%dseg" % c[:3] for c in CASES]


def _sample(C, width):
    """Channels at the ends of the first and last workgroups and in between."""
    last = (C - 1) // width * width
    return sorted({c for c in (0, 1, 5, width - 1, width, width + 7, 2 * width + 18, C // 2, last - 1, last, last + 2, C - 2, C - 1) if 0 <= c < C})


def _run(case, io, soft=True, gate=True, resume=True, src=None, rows_in=None, lens=None, in_place=False, wide=None, seed=0):
    N, width, segments, b, C, n = case
    s = _inputs(io, b, n, C, N, soft, gate, rows_in, resume, seed)
    at = _sample(C, width)
    src = None if src is None else torch.tensor(src, dtype=torch.int32)
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32)
    part = {k: None if v is None else v if k in "BC" else v[at] if k in ("A", "D", "dt_bias") else v[:, at] if k == "h_in" else v[..., at] for k, v in s.items()}
    y_ref, ey, h_ref, eh = _reference(part, io, soft, src, lens)
    if lens is not None:                                          # what lies behind a sequence's tokens must not matter
        for i, m in enumerate(lens.tolist()):
            for k in ("x", "dt", "B", "C", "z"):
                if s[k] is not None:
                    s[k][i, max(m, 0):] = float("nan")
    y, strides = torch.full((b, n, C), 7.0, dtype=IO[io], device="cuda"), {}
    if wide:
        for k in ("x", "dt", "z"):
            if s[k] is not None:
                s[k] = strided(s[k], *wide)
        s["B"], s["C"], y = strided(s["B"], 4, N + 2), strided(s["C"], N + 2, 4), strided(y, *wide, fill=5.0)
        strides = dict([(k, C + sum(wide)) for k in ("x_stride", "dt_stride", "y_stride")], z_stride=C + sum(wide) if gate else 0, b_stride=2 * N + 6, c_stride=2 * N + 6)
    d = {k: cuda(v) for k, v in s.items()}
    h_out = d["h_in"] if in_place else torch.full((b, C, N), 7.0, device="cuda")
    size = ssmv.ssm_selective_scan_workspace(b, C, N, n)
    ws = torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda") if size else None       # as NaN as bytes can be
    src_d, lens_d = cuda(src), cuda(lens)
    call = lambda: ssmv.ssm_selective_scan(x=d["x"], dt=d["dt"], A=d["A"], Bm=d["B"], Cm=d["C"], D=d["D"], y_out=y, batch=b, channels=C, dstate=N, L=n, io=io,
                                           dt_bias=d["dt_bias"], dt_softplus=soft, z=d["z"], h_in=d["h_in"], h_out=h_out, src_row=src_d, seq_len=lens_d, workspace=ws, **strides)
    groups = b * -(-C // width)
    assert launches(call) == ([(groups * (segments - 1), 512)] if segments > 1 else []) + [(groups * segments, 512)]
    call()
    torch.cuda.synchronize()
    got = y.cpu()
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        check_within(got[i, :m][:, at], y_ref[i, :m], ey[i, :m], "y of sequence %d" % i)
        assert torch.equal(got[i, m:], torch.full_like(got[i, m:], 7.0)), "written behind the sequence's tokens"
    check_within(h_out[:, at], h_ref, eh, "state")
    assert bool(torch.isfinite(h_out).all())
    if wide:
        parent = y._base.cpu()
        assert bool((parent[..., :wide[0]] == 5.0).all()) and bool((parent[..., wide[0] + C:] == 5.0).all())
    return got, h_out.cpu()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_whole_prompts(case, io):
    y, h = _run(case, io, seed=1)
    y2, h2 = _run(case, io, in_place=True, seed=1)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    _run(case, io, soft=False, gate=False, resume=False, seed=2)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_ragged_prompts_of_other_rows(case, io):
    b, n = case[3], case[5]
    seg = -(-(-(-n // 64)) // case[2]) * 64                       # tokens of a segment
    _run(case, io, lens=[n // 2 + 1, 0, n, 1, 17][:b], src=[1, 1, -1, 0, 9][:b], rows_in=2, seed=3)
    _run(case, io, lens=[min(seg, n - 2), n - 1, n + 40, 16, 33][:b], in_place=True, seed=4)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_strides(case, io):
    _run(case, io, wide=(3, 2), seed=5)
    _run(case, io, wide=(0, 8), lens=[case[5] - 5, case[5], 40, 2, 70][:case[3]], seed=6)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(16, 16, 1, 70, 9, 90), (32, 32, 1, 70, 66, 75), (16, 64, 1, 130, 400, 41)], ids=["w16", "w32", "w64"])
def test_more_prompts_than_are_put_in_order(case, io):
    """Beyond 64 prompts they start in the order of their indexes."""
    b, n = case[3], case[5]
    _run(case, io, lens=[(n * (i * 37 % 101)) // 100 for i in range(b)], seed=7)
