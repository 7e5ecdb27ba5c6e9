"""The layer operators as they are used: a step of training through two gated layers, and a beam search whose logits go through the rules."""
import os
import sys

import pytest
import torch

import paper_2408_15237_amd as ssmv
from _layers import gen

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import beam_decode  # noqa: E402

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _weights(g, layers, D, C):
    r = lambda *s: torch.randn(*s, generator=g)
    return [dict(w_in=r(D, 4 * C) / D ** 0.5, w_out=r(C, D) / C ** 0.5, A=-8 * torch.rand(C, generator=g) * 0.1 - 1e-3, f_bias=r(C), i_bias=r(C), post=1 + r(D) / 8, scale=1 + r(D) / 8,
                 pre=1 + r(D) / 8) for _ in range(layers)]


def _definition(x, start, ws, first):
    """Hidden states after every layer's residual sum and norm, from the definitions; the weights' type."""
    norm = lambda v, w: v / (v.square().mean(-1, keepdim=True) + EPS).sqrt() * w
    r, n, ends = x, norm(x, first), []
    for w, h in zip(ws, start):
        px, pf, pi, pz = (n @ w["w_in"]).chunk(4, -1)
        a = torch.exp(w["A"] * torch.sigmoid(pf + w["f_bias"]))
        v = (1 - a * a).sqrt() * torch.sigmoid(pi + w["i_bias"]) * px
        hs = []
        for t in range(x.shape[1]):
            h = a[:, t] * h + v[:, t]
            hs.append(h)
        ends.append(h)
        o = (torch.stack(hs, 1) * torch.nn.functional.silu(pz)) @ w["w_out"]
        r = r + 0.5 * w["scale"] * norm(o, w["post"])
        n = norm(r, w["pre"])
    return n, ends


def test_a_training_step():
    """Gradients of all weights and inputs through two layers against automatic differentiation in 64 bits.  A product over 48 values is off by 50 roundings (3e-6) of the sizes
    it adds, an operator by about as much; some dozen of them follow each other, and no norm here magnifies by more than ten: 5e-4 of a gradient's largest entry."""
    g = gen(21)
    b, n, D, C, layers = 3, 90, 48, 40, 2
    ws, first, x, G = _weights(g, layers, D, C), 1 + torch.randn(D, generator=g) / 8, torch.randn(b, n, D, generator=g), torch.randn(b, n, D, generator=g)
    start = [torch.randn(b, C, generator=g) for _ in range(layers)]
    leaf = lambda t: t.double().requires_grad_()
    ref = [{k: leaf(v) for k, v in w.items()} for w in ws]
    rx, rfirst, rstart = leaf(x), leaf(first), [leaf(h) for h in start]
    out, _ = _definition(rx, rstart, ref, rfirst)
    leaves = [rx, rfirst] + rstart + [v for w in ref for v in w.values()]
    want = torch.autograd.grad((out * G).sum(), leaves)

    rows, cu = b * n, lambda t: t.cuda()
    E = lambda *s: torch.empty(*s, device="cuda")
    W = [{k: cu(v) for k, v in w.items()} for w in ws]
    r = cu(x).view(rows, D)
    nrm = E(rows, D)
    ssmv.ssmv_block_norm(res=r, pre_wgt=cu(first), n_out=nrm, rows=rows, channels=D, io="f32", eps=EPS)
    kept = []
    for w, h0 in zip(W, start):
        p = nrm @ w["w_in"]
        px, pf, pi, pz = p.split(C, -1)
        y, states, h0 = E(b, n, C), E(b, (n + 63) // 64, C), cu(h0)
        st = dict(x_stride=4 * C, f_stride=4 * C, i_stride=4 * C, z_stride=4 * C)
        ssmv.ssm_gated_recurrence(x=px, f=pf, i=pi, z=pz, A=w["A"], f_bias=w["f_bias"], i_bias=w["i_bias"], h_in=h0, states=states, y_out=y, batch=b, channels=C, L=n, io="f32", **st)
        o = y.view(rows, C) @ w["w_out"]
        r2, n2 = E(rows, D), E(rows, D)
        ssmv.ssmv_block_norm(x=o, res=r, post_wgt=w["post"], ch_scale=w["scale"], pre_wgt=w["pre"], r_out=r2, n_out=n2, rows=rows, channels=D, io="f32", eps=EPS, res_scale=0.5)
        kept.append((nrm, p, states, y, o, r, st))
        r, nrm = r2, n2
    assert torch.allclose(nrm.view(b, n, D).cpu().double(), out.detach(), rtol=0, atol=5e-4 * float(out.detach().abs().max()))
    got_w, got_h = [None] * layers, [None] * layers
    dr, dn = None, cu(G).view(rows, D).contiguous()
    work = torch.empty(ssmv.ssmv_block_norm_backward_workspace(rows, D), dtype=torch.uint8, device="cuda")
    work2 = torch.empty(ssmv.ssm_gated_recurrence_backward_workspace(b, C, n), dtype=torch.uint8, device="cuda")
    for k in reversed(range(layers)):
        w, (nin, p, states, y, o, res, st) = W[k], kept[k]
        d = dict(post=E(D), scale=E(D), pre=E(D))
        do, dres = E(rows, D), E(rows, D)
        ssmv.ssmv_block_norm_backward(x=o, res=res, post_wgt=w["post"], ch_scale=w["scale"], pre_wgt=w["pre"], dr=dr, dn=dn, dx=do, dres=dres, dpost_wgt=d["post"], dch_scale=d["scale"],
                                      dpre_wgt=d["pre"], rows=rows, channels=D, io="f32", eps=EPS, res_scale=0.5, workspace=work)
        d["w_out"] = y.view(rows, C).T.contiguous() @ do
        dy = (do @ w["w_out"].T.contiguous()).view(b, n, C)
        dp = E(rows, 4 * C)
        parts = dp.split(C, -1)
        px, pf, pi, pz = p.split(C, -1)
        d.update(A=E(C), f_bias=E(C), i_bias=E(C))
        dh = E(b, C)
        ssmv.ssm_gated_recurrence_backward(x=px, f=pf, i=pi, z=pz, A=w["A"], f_bias=w["f_bias"], i_bias=w["i_bias"], states=states, dy=dy, dx=parts[0], df=parts[1], di=parts[2],
                                           dz=parts[3], dA=d["A"], df_bias=d["f_bias"], di_bias=d["i_bias"], dh_in=dh, batch=b, channels=C, L=n, io="f32", dx_stride=4 * C,
                                           df_stride=4 * C, di_stride=4 * C, dz_stride=4 * C, workspace=work2, **st)
        d["w_in"] = nin.T.contiguous() @ dp
        dn, dr = dp @ w["w_in"].T.contiguous(), dres
        got_w[k], got_h[k] = d, dh
    dfirst, dx = E(D), E(rows, D)
    ssmv.ssmv_block_norm_backward(res=cu(x).view(rows, D), pre_wgt=cu(first), dr=dr, dn=dn, dres=dx, dpre_wgt=dfirst, rows=rows, channels=D, io="f32", eps=EPS, workspace=work)
    got = [dx.view(b, n, D), dfirst] + got_h + [d[k] for d, w in zip(got_w, ws) for k in w]
    for i, (a, q) in enumerate(zip(got, want)):
        assert float((a.cpu().double() - q).abs().max()) <= 5e-4 * float(q.abs().max()), i


def test_single_tokens_continue_a_prompt():
    """A prompt by whole calls, then tokens one at a time from rows that beams chose: the hidden states of the definition over every beam's own text."""
    g = gen(22)
    rows, n, D, C, steps = 4, 70, 48, 40, 3
    ws, first = _weights(g, 2, D, C), 1 + torch.randn(D, generator=g) / 8
    W = [{k: v.cuda() for k, v in w.items()} for w in ws]
    text = torch.randn(rows, n, D, generator=g)

    def forward(x, h, src):
        b, m = x.shape[:2]
        r = x.cuda().reshape(b * m, D)
        nrm, ends = torch.empty_like(r), []
        ssmv.ssmv_block_norm(res=r, pre_wgt=first.cuda(), n_out=nrm, rows=b * m, channels=D, io="f32", eps=EPS)
        for w, h0 in zip(W, h):
            px, pf, pi, pz = (nrm @ w["w_in"]).split(C, -1)
            y, h1 = torch.empty(b, m, C, device="cuda"), torch.empty(b, C, device="cuda")
            ssmv.ssm_gated_recurrence(x=px, f=pf, i=pi, z=pz, A=w["A"], f_bias=w["f_bias"], i_bias=w["i_bias"], h_in=h0, src_row=src, h_out=h1, y_out=y, batch=b, channels=C, L=m,
                                      io="f32", x_stride=4 * C, f_stride=4 * C, i_stride=4 * C, z_stride=4 * C)
            o = y.view(b * m, C) @ w["w_out"]
            n2 = torch.empty_like(r)
            ssmv.ssmv_block_norm(x=o, res=r, post_wgt=w["post"], ch_scale=w["scale"], pre_wgt=w["pre"], r_out=r, n_out=n2, rows=b * m, channels=D, io="f32", eps=EPS, res_scale=0.5)
            nrm = n2
            ends.append(h1)
        return nrm.view(b, m, D), ends

    hidden, h = forward(text, [None, None], None)
    for _ in range(steps):
        src = torch.randint(0, rows, (rows,), generator=g, dtype=torch.int32)
        new = torch.randn(rows, 1, D, generator=g)
        text = torch.cat([text[src.long()], new], 1)
        hidden, h = forward(new, h, src.cuda())
    dbl = [{k: v.double() for k, v in w.items()} for w in ws]
    want, ends = _definition(text.double(), [torch.zeros(rows, C, dtype=torch.float64)] * 2, dbl, first.double())
    # a forward pass alone: 1e-4 of the largest entry (see the training step)
    assert float((hidden[:, 0].cpu().double() - want[:, -1]).abs().max()) <= 1e-4 * float(want.abs().max())
    for a, q in zip(h, ends):
        assert float((a.cpu().double() - q).abs().max()) <= 1e-4 * float(q.abs().max())


def test_a_beam_search_with_a_penalty():
    """examples/beam_decode.py: a penalty of 1 changes nothing; a very large one keeps tokens that occurred (their logits positive or not) from being said again."""
    w = beam_decode.make_weights(layers=2, width=64, inner=96, dstate=16, dt_rank=6, vocab=200, io="f32", seed=3)
    g = torch.Generator().manual_seed(5)
    lengths = torch.tensor([11, 1, 40], dtype=torch.int32).cuda()
    prompts = torch.randint(3, 200, (3, 40), generator=g, dtype=torch.int32).cuda()
    run = lambda repetition: beam_decode.beam_search(beam_decode.Model(w), prompts, lengths, 4, 9, eos=2, repetition=repetition)
    plain, same, strict = run(None), run(1.0), run(1e6)
    assert torch.equal(plain[0], same[0]) and torch.equal(plain[1], same[1])
    for s in range(3):
        seen = set(prompts[s, :int(lengths[s])].tolist())
        for beam in strict[0][s].tolist():
            said = beam[:beam.index(2)] if 2 in beam else beam
            assert len(set(said)) == len(said) and not seen & set(said), (s, beam)
