"""A model with one decay per head decoded without a cache from where a cache stands: the prompt by ssm_prefill_block, its state by
ssmv_materialize_block and ssmv_conv_history, then tokens of beams by ssm_causal_conv and ssm_selective_step, rows continuing from other rows; and back
into a cache.  Against the recurrence in 64 bits over every row's own line of tokens."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _decode import IO, conv_reference, scan_reference
from _harness import TOL, rel_err, to_host

pytestmark = pytest.mark.gpu

H, P, N, G, L = 4, 64, 64, 2, 37
Cx = H * P


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_prompt_in_a_cache_then_beams_without(io):
    g, lens, t = torch.Generator().manual_seed(17), [L, 20], IO[io]
    rnd = lambda *s: torch.randn(*s, generator=g).to(t)
    tokens = lambda rows, n: dict(x=rnd(rows, n, Cx), dt=(torch.randn(rows, n, H, generator=g) - 2).to(t), B=(rnd(rows, n, G, N).float() / N ** 0.5).to(t),
                                  C=(rnd(rows, n, G, N).float() / N ** 0.5).to(t), z=rnd(rows, n, Cx))
    w, bias, D = (rnd(Cx, 4).float() / 2).to(t), (rnd(Cx).float() * 0.1).to(t), torch.randn(H, generator=g)
    A, dtb = -torch.exp(torch.rand(H, generator=g) * 2), torch.rand(H, generator=g) - 0.5
    dev = {k: v.cuda() for k, v in dict(w=w, bias=bias, D=D, A=A, dtb=dtb).items()}

    def reference(line):
        """y and state at the end of a line of tokens: dict of [1][n][..]."""
        xc, _, _ = conv_reference(line["x"], w, bias, None, "silu", io)
        y, _, h, _ = scan_reference(xc.to(t).view(1, -1, H, P), line["dt"], A, line["B"], line["C"], D, io, dtb, True, line["z"].view(1, -1, H, P))
        return y.reshape(1, -1, Cx), h[0]

    prompt = tokens(2, L)
    dims = ssmv.make_dims(2, H, P, N, ngroups=G, kmax=4, io=io, conv_act="silu")
    cache = ssmv.LayerCache.allocate(dims)
    ssmv.ssmv_cache_reset(dims, cache.c)
    y = torch.zeros(2, L, Cx, dtype=t, device="cuda")
    p = {k: v.cuda() for k, v in prompt.items()}
    ssmv.ssm_prefill_block(dims, cache.c, x_raw=p["x"], conv_wgt=dev["w"], conv_bias=dev["bias"], dt=p["dt"], dt_bias=dev["dtb"], dt_softplus=True, Bm=p["B"], Cm=p["C"],
                           z=p["z"], A=dev["A"], D=dev["D"], L=L, y_out=y, seq_len=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    h, conv = torch.empty(2, H, P, N, device="cuda"), torch.empty(2, 3, Cx, dtype=t, device="cuda")
    ssmv.ssmv_materialize_block(dims, cache.c, dev["A"], dev["dtb"], True, h)
    ssmv.ssmv_conv_history(dims, cache.c, conv)
    lines = [{k: v[i:i + 1, :lens[i]] for k, v in prompt.items()} for i in range(2)]
    for i in range(2):
        assert torch.equal(conv[i].cpu(), prompt["x"][i, lens[i] - 3:lens[i]])
        y_ref, h_ref = reference(lines[i])
        assert rel_err(to_host(y[i:i + 1, :lens[i]]), y_ref.numpy()) <= TOL[io] and rel_err(to_host(h[i]), h_ref.numpy()) <= TOL[io]

    for parents in ([0, 0, 1, 1, 0], [1, 0, 3, 3, 4], [4, 2, 1, 0, 3], [0, 1, 2, 2, 2]):
        rows = len(parents)
        new = tokens(rows, 1)
        d, src = {k: v.cuda() for k, v in new.items()}, torch.tensor(parents, dtype=torch.int32, device="cuda")
        xc, conv2 = torch.empty(rows, 1, Cx, dtype=t, device="cuda"), torch.empty(rows, 3, Cx, dtype=t, device="cuda")
        ssmv.ssm_causal_conv(x=d["x"], wgt=dev["w"], bias=dev["bias"], conv_in=conv, conv_out=conv2, src_row=src, out=xc, batch=rows, channels=Cx, L=1, io=io, act="silu")
        y, h2 = torch.empty(rows, Cx, dtype=t, device="cuda"), torch.empty(rows, H, P, N, device="cuda")
        ssmv.ssm_selective_step(x=xc, dt=d["dt"], A=dev["A"], Bm=d["B"], Cm=d["C"], D=dev["D"], z=d["z"], y_out=y, h_in=h, h_out=h2, src_row=src, rows=rows, nheads=H,
                                headdim=P, dstate=N, ngroups=G, io=io, a_mode="scalar", dt_bias=dev["dtb"], dt_softplus=True)
        lines = [{k: torch.cat([lines[r][k], new[k][i:i + 1]], 1) for k in new} for i, r in enumerate(parents)]
        h, conv = h2, conv2
        for i in range(rows):
            y_ref, h_ref = reference(lines[i])
            assert torch.equal(conv[i].cpu(), lines[i]["x"][0, -3:])
            assert rel_err(to_host(y[i]), y_ref[0, -1].numpy()) <= TOL[io] and rel_err(to_host(h[i]), h_ref.numpy()) <= TOL[io]

    # and back: caches that start from the rows' states go on with the next token
    dims = ssmv.make_dims(rows, H, P, N, ngroups=G, kmax=4, io=io, conv_act="silu")
    cache = ssmv.LayerCache.allocate(dims)
    ssmv.ssmv_cache_reset(dims, cache.c, h, conv)
    new = tokens(rows, 1)
    d, y = {k: v.cuda() for k, v in new.items()}, torch.zeros(rows, 1, Cx, dtype=t, device="cuda")
    ssmv.ssm_prefill_block(dims, cache.c, x_raw=d["x"], conv_wgt=dev["w"], conv_bias=dev["bias"], dt=d["dt"], dt_bias=dev["dtb"], dt_softplus=True, Bm=d["B"], Cm=d["C"],
                           z=d["z"], A=dev["A"], D=dev["D"], L=1, y_out=y)
    for i in range(rows):
        y_ref, _ = reference({k: torch.cat([lines[i][k], new[k][i:i + 1]], 1) for k in new})
        assert rel_err(to_host(y[i, 0]), y_ref[0, -1].numpy()) <= TOL[io]
