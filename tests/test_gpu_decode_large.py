"""The state-to-state operators on tensors beyond 2^32 bytes, on outputs that are stored past the caches, and on rows of logits of several
pieces and chunks: against the same call on a part of the tensors, which the other tests hold to the definition."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _decode import gen
from test_gpu_beam_select import _check, _select

pytestmark = pytest.mark.gpu


def _randn(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _conv(x, w, **kw):
    b, n, C = x.shape
    out, state = torch.empty(b, n, C, dtype=x.dtype, device="cuda"), torch.empty(b, 3, C, dtype=x.dtype, device="cuda")
    ssmv.ssm_causal_conv(x=x, wgt=w, out=out, conv_out=state, batch=b, channels=C, L=n, io="bf16", act="silu", **kw)
    return out, state


def test_conv_beyond_32_bits():
    n, C, cut = 140000, 16384, 139950                             # 4.6 GB in, 4.6 GB out
    x, w = _randn(1, 1, n, C), _randn(2, C, 4)
    whole, state = _conv(x, w)
    tail, tail_state = _conv(x[:, cut:].contiguous(), w, conv_in=x[:, cut - 3:cut].contiguous())
    assert torch.equal(whole[:, cut:], tail) and torch.equal(state, tail_state)
    head, _ = _conv(x[:, :64].contiguous(), w)
    assert torch.equal(whole[:, :64], head)


@pytest.mark.parametrize("C", [8192, 8197])
def test_conv_outputs_past_the_caches(C):
    n = 8300                                                      # 136 MB
    x, w = _randn(3, 1, n, C), _randn(4, C, 4)
    whole, _ = _conv(x, w)
    for a in (0, 1000, 8000):
        part, _ = _conv(x[:, a:a + 300].contiguous(), w, conv_in=x[:, a - 3:a].contiguous() if a else None)
        assert torch.equal(whole[:, a:a + 300], part)


def _scan(d, a, b, h_in, C, N):
    n = b - a
    need = ssmv.ssm_selective_scan_workspace(1, C, N, n)
    y, h = torch.empty(1, n, C, dtype=torch.bfloat16, device="cuda"), torch.empty(1, C, N, device="cuda")
    ssmv.ssm_selective_scan(x=d["x"][:, a:b], dt=d["dt"][:, a:b], A=d["A"], Bm=d["B"][:, a:b], Cm=d["C"][:, a:b], D=d["D"], y_out=y, batch=1, channels=C,
                            dstate=N, L=n, io="bf16", dt_softplus=True, h_in=h_in, h_out=h,
                            workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
    return y, h


def test_scan_beyond_32_bits():
    n, C, N, cut = 140000, 16384, 16, 139000
    d = dict(x=_randn(5, 1, n, C), dt=_randn(6, 1, n, C) - 4, B=_randn(7, 1, n, N) / 4, C=_randn(8, 1, n, N) / 4, D=_randn(9, C, dtype=torch.float32),
             A=-torch.arange(1, N + 1, device="cuda", dtype=torch.float32).repeat(C, 1))
    y, h = _scan(d, 0, n, None, C, N)
    _, mid = _scan(d, 0, cut, None, C, N)
    y_tail, h_tail = _scan(d, cut, n, mid, C, N)
    # the two are cut differently: states agree to a few roundings of 32 bits, outputs to one of bf16
    scale = float(h_tail.abs().max())
    assert float((h - h_tail).abs().max()) <= 1e-5 * scale
    off = (y[:, cut:].float() - y_tail.float()).abs()
    assert bool((off <= 2.0 ** -7 * y_tail.float().abs() + 1e-5 * float(y_tail.float().abs().max())).all())


def test_step_beyond_32_bits():
    rows, H, P, N = 2100, 32, 128, 128                            # 4.4 GB of states in, and out
    h_in = _randn(10, rows, H, P, N, dtype=torch.float32)
    tok = dict(x=_randn(11, rows, H * P), dt=_randn(12, rows, H), Bm=_randn(13, rows, 1, N), Cm=_randn(14, rows, 1, N))
    A, D = -torch.rand(H, device="cuda", generator=torch.Generator(device="cuda").manual_seed(15)), torch.ones(H, device="cuda")
    src = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")
    y, h = torch.empty_like(tok["x"]), torch.empty_like(h_in)
    kw = dict(A=A, D=D, nheads=H, headdim=P, dstate=N, io="bf16", a_mode="scalar", dt_softplus=True)
    ssmv.ssm_selective_step(**tok, y_out=y, h_in=h_in, h_out=h, rows=rows, src_row=src, **kw)
    for a in (0, 1040, rows - 8):
        part = {k: v[a:a + 8].contiguous() for k, v in tok.items()}
        y8, h8 = torch.empty_like(part["x"]), torch.empty(8, H, P, N, device="cuda")
        ssmv.ssm_selective_step(**part, y_out=y8, h_in=h_in[src[a:a + 8].long()].contiguous(), h_out=h8, rows=8, **kw)
        assert torch.equal(y[a:a + 8], y8) and torch.equal(h[a:a + 8], h8)


def _select_gpu(logits, scores, batch, K):
    W, V = logits.shape[0] // batch, logits.shape[1]
    parent, token = (torch.empty(batch * K, dtype=torch.int32, device="cuda") for _ in range(2))
    out = torch.empty(batch * K, device="cuda")
    ws = torch.empty(ssmv.ssmv_beam_workspace(batch, W, K, V), dtype=torch.uint8, device="cuda")
    ssmv.ssmv_beam_select(logits=logits, scores=scores, parent=parent, token=token, scores_out=out, batch=batch, beams_in=W, beams_out=K, vocab=V, io="bf16", workspace=ws)
    return [t.view(batch, K) for t in (parent, token, out)]


def test_selection_beyond_32_bits():
    batch, W, V, K = 4200, 4, 131101, 4                           # 4.4 GB of logits
    logits, scores = _randn(16, batch * W, V), _randn(17, batch * W, dtype=torch.float32)
    parent, token, out = _select_gpu(logits, scores, batch, K)
    for s in (0, 2100, 4199):
        p1, t1, o1 = _select_gpu(logits[s * W:(s + 1) * W], scores[s * W:(s + 1) * W], 1, K)
        # (pieces of another size: a row's sum may differ in its last bits, and with it only what is nearer than that)
        assert torch.allclose(out[s], o1[0], rtol=0, atol=1e-5)
        assert torch.equal(parent[s] - s * W, p1[0]) and torch.equal(token[s], t1[0])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_rows_of_several_chunks(io):
    """Many rows: a piece takes several chunks one after the other."""
    g = gen(18)
    dtype = torch.bfloat16 if io == "bf16" else torch.float32
    batch, W, V = 130, 4, 33001
    logits = (3 * torch.randn(batch * W, V, generator=g)).to(dtype)
    logits[0:4] = 1.0                                             # nothing but ties
    logits[4:8, :30000] = float("-inf")                           # nothing in the first chunks
    logits[8:12, 5:] = float("-inf")                              # nothing in the last ones
    logits[12] = float("-inf")
    logits[16:20] = torch.linspace(-9, 9, V).to(dtype)            # every chunk better than the ones before
    logits[20:24] = torch.linspace(9, -9, V).to(dtype)
    logits[24:28, ::2] = 7.0                                      # thousands of ties below the best
    scores = -(20 + 2 * torch.randn(batch * W, generator=g).abs())
    scores[0:4], scores[24:28] = -5.0, -6.0
    few = 12                                                      # the reference sorts in 64 bits: the sequences with something about them
    parent, token, out, _ = _select(logits, scores, batch, 40, io)
    _check(logits[:4 * few], scores[:4 * few], few, 40, io)
    assert parent[0].tolist() == [0] * 40 and token[0].tolist() == list(range(40))
    alone = _select(logits[:4 * few], scores[:4 * few], few, 40, io)
    for s in range(few):
        assert torch.allclose(out[s], alone[2][s], rtol=0, atol=1e-5, equal_nan=True)
        assert parent[s].tolist() == alone[0][s].tolist() and token[s].tolist() == alone[1][s].tolist()
