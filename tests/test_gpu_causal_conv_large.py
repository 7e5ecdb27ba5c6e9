"""ssm_causal_conv where the outputs are stored past the caches (128 MiB of them or more; fp32: eight tokens of a thread), against the
convolution in 64 bits on a sample of the channels, which are independent of each other.  Every call's launch is looked at."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _decode import IO, check_within, conv_reference
from _harness import launches

pytestmark = pytest.mark.gpu

# (type, batch, tokens, channels): numbers of tokens that neither 8 nor 4 divides, channels that a vector divides and that it does not
CASES = [("f32", 1, 4203, 8192), ("f32", 1, 4203, 8197), ("f32", 3, 1403, 8197), ("f32", 7, 1501, 3333), ("bf16", 1, 8403, 8192), ("bf16", 3, 2805, 8197), ("bf16", 7, 3002, 3333)]


def _workgroups(io, b, n, C):
    """Of the kernel for large outputs: vectors of 16 bytes, 64 of a row side by side, 8 (fp32) or 4 tokens of a thread, 256 threads."""
    chunks, tokens = -(-C // (4 if io == "f32" else 8)), 8 if io == "f32" else 4
    return b * -(-chunks // 64) * -(-(-(-n // tokens)) // 4)


def _run(io, b, n, C, act, hist=True, bias=True, src=None, rows_in=None, lens=None, wide=None, in_place=False, seed=0):
    assert b * n * C * IO[io].itemsize > 128 << 20
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda").to(IO[io])
    before, after = wide or (0, 0)
    x = randn(b, n, before + C + after)[..., before:before + C]
    w, bv = randn(C, 4) / 2, randn(C) * 0.1 if bias else None
    conv_in = randn(rows_in or b, 3, C) if hist else None
    src = None if src is None else torch.tensor(src, dtype=torch.int32)
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32)
    at = sorted({0, 1, 3, 4, 7, 8, 255, 256, 511, 513, C // 2, C - 9, C - 8, C - 5, C - 4, C - 2, C - 1})
    cpu = lambda t: None if t is None else t[..., at].cpu()
    ref, bound, _ = conv_reference(cpu(x), w[at].cpu(), cpu(bv), cpu(conv_in), act, io, src, lens)
    start = None if conv_in is None else conv_in.clone()
    if lens is not None:                                          # what lies behind a sequence's tokens must not matter
        for i, m in enumerate(lens.tolist()):
            x[i, max(m, 0):] = float("nan")
    out = torch.full((b, n, before + C + after), 7.0, dtype=IO[io], device="cuda")[..., before:before + C]
    conv_out = conv_in if in_place else torch.full((b, 3, C), 7.0, dtype=IO[io], device="cuda")
    src_d, lens_d = None if src is None else src.cuda(), None if lens is None else lens.cuda()
    call = lambda: ssmv.ssm_causal_conv(x=x, wgt=w, bias=bv, conv_in=conv_in, src_row=src_d, seq_len=lens_d, out=out, conv_out=conv_out, batch=b, channels=C, L=n, io=io,
                                        act=act, x_stride=x.stride(1), out_stride=out.stride(1))
    assert launches(call) == [(_workgroups(io, b, n, C), 256)]
    call()
    torch.cuda.synchronize()
    got = out[..., at].cpu()
    for i in range(b):
        m = n if lens is None else min(max(int(lens[i]), 0), n)
        check_within(got[i, :m], ref[i, :m], bound[i, :m], "out of sequence %d" % i)
        assert bool((out[i, m:] == 7.0).all()), "written behind the sequence's tokens"
        assert bool(torch.isfinite(out[i, :m]).all())
        r = i if src is None else int(src[i])
        old = start[r] if start is not None and 0 <= r < start.shape[0] else torch.zeros(3, C, dtype=IO[io], device="cuda")
        assert torch.equal(conv_out[i], torch.cat([old, x[i, max(0, m - 3):m]])[-3:]), "history of sequence %d" % i
    if wide:
        parent = out._base
        assert bool((parent[..., :before] == 7.0).all()) and bool((parent[..., before + C:] == 7.0).all())


@pytest.mark.parametrize("io,b,n,C", CASES)
def test_whole_prompts(io, b, n, C):
    _run(io, b, n, C, "silu", seed=1)
    _run(io, b, n, C, "none", hist=False, bias=False, wide=(3, 2), seed=2)


@pytest.mark.parametrize("io,b,n,C", [c for c in CASES if c[1] > 1])
def test_ragged_prompts(io, b, n, C):
    lens = [n, 0, 9, 1, n - 1, 2, 1000]
    _run(io, b, n, C, "silu", lens=lens[:b], in_place=True, seed=3)
    _run(io, b, n, C, "silu", lens=[n // 2 + 3, n + 5, -2, 3, 8, 12, n - 6][:b], src=[1, 1, -1, 0, 9, 0, 1][:b], rows_in=2, wide=(0, 8), seed=4)
