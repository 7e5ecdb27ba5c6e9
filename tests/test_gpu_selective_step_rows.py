"""ssm_selective_step where four rows of the batch share a workgroup: against the recurrence in 64 bits, and beyond 2^32 bytes against the
kernel of one row.  Every call's launch is looked at, so that another rule of choosing between the two kernels shows here."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
import test_gpu_selective_step as one_row
from _harness import launches
from test_gpu_decode_large import _randn

pytestmark = pytest.mark.gpu


def _workgroups(rows, channels, N, together):
    return -(-channels * N // 1024) * -(-rows // together)


@pytest.fixture
def four_rows(monkeypatch):
    """The test's calls have to be ones of four rows to a workgroup."""
    call = ssmv.ssm_selective_step

    def checked(**kw):
        assert launches(lambda: call(**kw)) == [(_workgroups(kw["rows"], kw["nheads"] * kw["headdim"], kw["dstate"], 4), 256)]
        call(**kw)

    monkeypatch.setattr(ssmv, "ssm_selective_step", checked)


# (mode, nheads, headdim, dstate, groups, rows): the last workgroup is neither full of channels nor of rows
SHAPES = [("diag", 8200, 1, 16, 1, 33), ("diag", 4100, 1, 32, 1, 34), ("diag", 2060, 1, 64, 1, 35), ("scalar", 41, 200, 16, 1, 34), ("scalar", 10, 410, 32, 2, 35),
          ("scalar", 9, 229, 64, 3, 33), ("scalar", 5, 206, 128, 5, 34), ("scalar", 3, 171, 256, 1, 35)]


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("mode,H,P,N,G,rows", SHAPES)
def test_against_the_recurrence(four_rows, io, mode, H, P, N, G, rows):
    one_row._run(io, mode, rows, H, P, N, G, seed=H + N)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("mode,H,P,N,G,rows", [SHAPES[0], SHAPES[5]])
def test_rows_strides_and_pieces(four_rows, io, mode, H, P, N, G, rows):
    src = ([2, 2, 0, -1, 3, 77, 1, 1, 0] * 4)[:rows]
    one_row._run(io, mode, rows, H, P, N, G, src=src, rows_in=4, seed=1)
    one_row._run(io, mode, rows + 1, H, P, N, G, in_place=True, seed=2)
    one_row._run(io, mode, rows + 2, H, P, N, G, no_state=True, seed=3)
    one_row._run(io, mode, rows + 3, H, P, N, G, soft=False, gate=False, seed=4)
    one_row._run(io, mode, rows, H, P, N, G, wide=(3, 2), seed=5)
    one_row._run(io, mode, rows, H, P, N, G, src=src, rows_in=4, wide=(0, 8), gate=False, seed=6)


def test_the_kernel_of_one_row_beyond_32_bits():
    rows, H, P, N = 2102, 32, 128, 128                            # 4.4 GB of states in, and out
    h_in = _randn(10, rows, H, P, N, dtype=torch.float32)
    tok = dict(x=_randn(11, rows, H * P), dt=_randn(12, rows, H), Bm=_randn(13, rows, 1, N), Cm=_randn(14, rows, 1, N), z=_randn(16, rows, H * P))
    A, D = -torch.rand(H, device="cuda", generator=torch.Generator(device="cuda").manual_seed(15)), torch.ones(H, device="cuda")
    src = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")
    y, h = torch.empty_like(tok["x"]), torch.empty_like(h_in)
    kw = dict(A=A, D=D, nheads=H, headdim=P, dstate=N, io="bf16", a_mode="scalar", dt_softplus=True)
    call = lambda: ssmv.ssm_selective_step(**tok, y_out=y, h_in=h_in, h_out=h, rows=rows, src_row=src, **kw)
    assert launches(call) == [(_workgroups(rows, H * P, N, 4), 256)]
    call()
    for a in (0, 1045, rows - 7):
        part = {k: v[a:a + 7].contiguous() for k, v in tok.items()}
        y7, h7, start = torch.empty_like(part["x"]), torch.empty(7, H, P, N, device="cuda"), h_in[src[a:a + 7].long()].contiguous()
        few = lambda: ssmv.ssm_selective_step(**part, y_out=y7, h_in=start, h_out=h7, rows=7, **kw)
        assert launches(few) == [(_workgroups(7, H * P, N, 1), 256)]
        few()
        assert torch.equal(y[a:a + 7], y7) and torch.equal(h[a:a + 7], h7)
