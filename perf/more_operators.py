"""The operators around a gated recurrent layer, as cases that can be timed and compared.

Five kinds of pass, together what such a layer does in training and what a model of them does with every new token:

* "norm": gate and norm behind a block, the residual sum, the norm ahead of the next block (ssmv_block_norm).
* "norm_grad": its gradients, of weights too (ssmv_block_norm_backward).
* "rec": the gated linear recurrence over a prompt, or over one new token of every beam (ssm_gated_recurrence).
* "rec_grad": its gradients, from the states that the forward pass leaves every 64 tokens (ssm_gated_recurrence_backward).
* "rules": penalties for repeated tokens, biases and grammar masks on the logits of every beam (ssmv_logit_rules).

`own` False computes them in elementary torch operations.  Distributions: activations, their gradients and raw gates ~ N(0,1), the residual
stream ~ 2 N(0,1), norm weights ~ 1 + N(0,1)/10; decays A = 8 ln U(0.9, 0.999) per channel (form lru) or forget biases U(1, 4) (form mix);
logits ~ 3 N(0,1), histories with repeated tokens, grammar states that allow few tokens.
"""
from __future__ import annotations

import math

import torch

own = False

IO = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
TILE = 64            # tokens between two states that the forward pass leaves for the backward pass

_NORM = dict(kind="norm", io="bf16", res="bf16", rows=4, channels=4096, gate=True, post=True, scale=True, residual=True, split=False)
_REC = dict(kind="rec", io="bf16", form="lru", batch=1, length=2048, channels=4096, inp=True, gate=True, resume=False, ragged=False, beams=False,
            split=True)
_RULES = dict(kind="rules", io="bf16", rows=4, vocab=32000, pad=0, history=300, penalties="all", bias=0, grammar=0, beams=False, in_place=False)


def listed():
    return [
        # a new token of one user's four beams
        dict(_NORM, name="norm_token_b4", channels=8192, scale=False),
        # the prompts of a serving batch: residual sum and pre-norm alone
        dict(_NORM, name="norm_prompt_b8", rows=16384, gate=False, post=False, scale=False),
        # a training step's micro-batch with everything: gate (half of a projection's output), norm behind the block, residual scale, fp32 stream
        dict(_NORM, name="norm_grad_b4", kind="norm_grad", res="f32", rows=8192, channels=5120, split=True),
        # fp32, channels that no vector divides
        dict(_NORM, name="norm_grad_odd", kind="norm_grad", io="f32", res="f32", rows=999, channels=1001, gate=False),
        # one user's four beams: a token each, from the states of the beams that they descend from
        dict(_REC, name="rec_token_b4", batch=4, length=1, channels=8192, beams=True, resume=True),
        # one user's prompt
        dict(_REC, name="rec_prompt_b1", channels=8192),
        # a training step's batch
        dict(_REC, name="rec_grad_b8", kind="rec_grad", batch=8, channels=5120),
        # one long document through few channels
        dict(_REC, name="rec_grad_long", kind="rec_grad", form="mix", length=32768, channels=1024, inp=False),
        # fp32, odd sizes, sequences of different lengths that go on from a state
        dict(_REC, name="rec_grad_odd", kind="rec_grad", io="f32", batch=3, length=333, channels=1001, resume=True, ragged=True, split=False),
        # one user's next token, penalties alone
        dict(_RULES, name="rules_first", io="f32", rows=1),
        # a serving batch of 16 requests with eight beams each over a large vocabulary: everything, rows padded to whole lines
        dict(_RULES, name="rules_serving", rows=128, vocab=128011, pad=53, history=1000, bias=100, grammar=16, beams=True),
        # grammars alone, in place, an odd vocabulary
        dict(_RULES, name="rules_grammar", rows=64, vocab=49999, history=0, penalties="none", grammar=24, in_place=True),
    ]


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _channels(rng):
    """Mostly whole vectors of channels, sometimes any number."""
    return 16 * _log_int(rng, 4, 512) if rng.random() < 0.75 else _log_int(rng, 64, 8192)


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "norm_grad", "rec", "rec", "rec_grad", "rec_grad", "rules", "rules"])
    io = rng.choice(["bf16", "bf16", "f32"])
    flag = lambda p=0.5: rng.random() < p
    if kind in ("norm", "norm_grad"):
        channels, most = _channels(rng), 8192 * 5120 // (2 if io == "f32" else 1)
        rows = _log_int(rng, 1, max(1, min(32768, most // channels)))
        return dict(_NORM, kind=kind, io=io, res="f32" if io == "f32" else rng.choice(["bf16", "f32"]), rows=rows, channels=channels, gate=flag(), post=flag(),
                    scale=flag(), residual=flag(0.8), split=flag())
    if kind in ("rec", "rec_grad"):
        channels, most = _channels(rng), 8 * 2048 * 5120 // (2 if io == "f32" else 1)
        beams = kind == "rec" and flag(0.35)
        length = 1 if beams else _log_int(rng, 1, min(32768, most // channels))
        batch = _log_int(rng, 1, max(1, min(256 if beams else 32, most // (length * channels))))
        return dict(_REC, kind=kind, io=io, form=rng.choice(["lru", "mix"]), batch=batch, length=length, channels=channels, inp=flag(0.6), gate=flag(0.6),
                    resume=beams or flag(), ragged=batch > 1 and not beams and flag(), beams=beams, split=flag())
    vocab = _log_int(rng, 500, 160000)
    rows = _log_int(rng, 1, max(1, min(256, 128 * 128011 // (2 if io == "f32" else 1) // vocab)))
    in_place = flag(0.25)
    return dict(_RULES, io=io, rows=rows, vocab=vocab, pad=rng.choice([0, 0, -vocab % 64]), history=0 if in_place else _log_int(rng, 1, 8192),
                penalties="none" if in_place else rng.choice(["all", "all", "repetition"]), bias=0 if in_place else rng.choice([0, _log_int(rng, 1, 500)]),
                grammar=rng.choice([8, 64]) if in_place else rng.choice([0, 0, 8, 64]), beams=not in_place and flag(), in_place=in_place)


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _rng(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + what) % (1 << 62))
    return lambda *s: torch.randn(*s, generator=g, device="cuda"), lambda *s: torch.rand(*s, generator=g, device="cuda"), g


def _lengths(c, seed):
    """Lengths of the sequences: the longest is c["length"]; ragged ones from one token up."""
    g = torch.Generator().manual_seed(int(seed) * 17 + 5)
    n = torch.randint(1, c["length"] + 1, (c["batch"],), generator=g)
    n[0] = c["length"]
    return n.int().cuda() if c["ragged"] else None


def _prepare_norm(c, seed):
    randn, _, _ = _rng(seed, 11)
    n, C, io, res = c["rows"], c["channels"], IO[c["io"]], IO[c["res"]]
    wide = randn(n, 2 * C if c["split"] else C).to(io)             # the gate is the second half of a projection's output where that is so
    s = dict(case=c, x=randn(n, C).to(io), z=wide[:, -C:] if c["gate"] else None, res=(2 * randn(n, C)).to(res) if c["residual"] else None,
             post=1 + randn(C) / 10 if c["post"] else None, scale=0.5 + randn(C) / 10 if c["scale"] else None, pre=1 + randn(C) / 10,
             alpha=0.25 if c["scale"] else 1.0)
    if c["kind"] == "norm":
        s.update(r=torch.zeros(n, C, dtype=res, device="cuda"), n=torch.zeros(n, C, dtype=io, device="cuda"))
        return s
    s.update(dr=randn(n, C).to(res), dn=randn(n, C).to(io), dx=torch.zeros(n, C, dtype=io, device="cuda"),
             dz=torch.zeros(n, C, dtype=io, device="cuda") if c["gate"] else None,
             dres=torch.zeros(n, C, dtype=res, device="cuda") if c["residual"] else None, dpre=torch.zeros(C, device="cuda"),
             dpost=torch.zeros(C, device="cuda") if c["post"] else None, dscale=torch.zeros(C, device="cuda") if c["scale"] else None)
    return s


def _prepare_rec(c, seed):
    randn, rand, g = _rng(seed, 12)
    b, n, C, io = c["batch"], c["length"], c["channels"], IO[c["io"]]
    # x and z, f and i lie side by side as their projections leave them where that is so ("split")
    xz = randn(b, n, 2 * C if c["split"] else C).to(io)
    fi = randn(b, n, 2 * C if c["split"] else C).to(io)
    apart = lambda: randn(b, n, C).to(io)
    s = dict(case=c, x=xz[..., :C], f=fi[..., :C], i=(fi[..., C:] if c["split"] else apart()) if c["inp"] else None,
             z=(xz[..., C:] if c["split"] else apart()) if c["gate"] else None,
             A=8 * torch.log(0.9 + 0.099 * rand(C)) if c["form"] == "lru" else None,
             f_bias=rand(C) - 0.5 if c["form"] == "lru" else 1 + 3 * rand(C), i_bias=rand(C) - 0.5 if c["inp"] else None,
             h_in=randn(b, C) if c["resume"] else None, lens=_lengths(c, seed),
             src=torch.randint(0, b, (b,), generator=g, device="cuda", dtype=torch.int32) if c["beams"] else None)
    like = lambda on=True: torch.zeros(b, n, C, dtype=io, device="cuda") if on else None
    if c["kind"] == "rec":
        s.update(y=like(), h_out=torch.zeros(b, C, device="cuda"))
        return s
    # what the forward pass leaves: the state ahead of every 64th token
    a, v = _coefficients(s, torch.float64)
    h = _scan(a, v, s["h_in"])
    start = torch.zeros(b, 1, C, dtype=torch.float64, device="cuda") if s["h_in"] is None else s["h_in"].double()[:, None]
    s["states"] = torch.cat([start, h[:, TILE - 1:n - 1:TILE]], dim=1).float().contiguous()
    s.update(dy=apart(), dh_out=randn(b, C), dx=like(), df=like(), di=like(c["inp"]), dz=like(c["gate"]), dh_in=torch.zeros(b, C, device="cuda"),
             dA=torch.zeros(C, device="cuda") if c["form"] == "lru" else None, df_bias_out=torch.zeros(C, device="cuda"),
             di_bias_out=torch.zeros(C, device="cuda") if c["inp"] else None)
    return s


def _prepare_rules(c, seed):
    randn, rand, g = _rng(seed, 13)
    b, V, n = c["rows"], c["vocab"], c["history"]
    ints = lambda hi, *s: torch.randint(0, hi, s, generator=g, device="cuda", dtype=torch.int32)
    s = dict(case=c, logits=(3 * randn(b, V + c["pad"])).to(IO[c["io"]])[:, :V], rep=None, freq=None, pres=None, hist=None)
    if n:
        # frequent tokens occur many times; the histories are of different lengths, with room for more
        room = n + 32
        s["hist"] = (V * rand(b, room) ** 3).int().clamp(max=V - 1)
        s["hist_len"] = 1 + ints(n, b)
        s["hist_len"][0] = n
        s["prompt"] = ints(n, b)
        s["token"] = ints(V, b)
        s["src"] = ints(b, b) if c["beams"] else None
        s["hist_out"], s["hist_len_out"] = torch.zeros(b, room, dtype=torch.int32, device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda")
        s["rep"] = 1 + 0.3 * rand(b)
    if c["penalties"] == "all":
        s["freq"], s["pres"] = rand(b), rand(b)
    if c["bias"]:
        s["bias_token"], s["bias"] = ints(V, b, c["bias"]), 5 * randn(b, c["bias"])
        s["bias"][rand(b, c["bias"]) < 0.2] = -math.inf            # words that a request rules out
    if c["grammar"]:
        # a few states of a grammar allow most tokens (inside a text), the others some hundred
        words = (V + 31) // 32
        loose = rand(c["grammar"], 1) < 0.25
        bits = rand(c["grammar"], words, 32) < torch.where(loose, 0.9, 200 / V)[..., None]
        s["mask"] = (bits.long() << torch.arange(32, device="cuda")).sum(-1).to(torch.int64).bitwise_and(0xFFFFFFFF)
        s["mask"] = torch.where(s["mask"] >= 2 ** 31, s["mask"] - 2 ** 32, s["mask"]).int()
        s["mask_row"] = ints(c["grammar"] + 1, b) - 1              # -1: a request without a grammar
    s["out"] = s["logits"] if c["in_place"] else torch.zeros(b, V + c["pad"], dtype=IO[c["io"]], device="cuda")[:, :V]
    return s


def prepare(case, seed):
    return dict(norm=_prepare_norm, norm_grad=_prepare_norm, rec=_prepare_rec, rec_grad=_prepare_rec, rules=_prepare_rules)[case["kind"]](case, seed)


# ---- plain forms --------------------------------------------------------------------------------------------------------


def _norm_parts(s):
    """a, its scale, p, r, its scale; all in 32 bits."""
    a = s["x"].float()
    if s["z"] is not None:
        z = s["z"].float()
        a = a * z * torch.sigmoid(z)
    at = torch.rsqrt((a * a).mean(-1, keepdim=True) + EPS) if s["post"] is not None else None
    p = a if at is None else a * at * s["post"]
    r = s["alpha"] * p
    if s["scale"] is not None:
        r = r * s["scale"]
    if s["res"] is not None:
        r = r + s["res"].float()
    return a, at, p, r, torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS)


def _plain_norm(s):
    c = s["case"]
    _, _, _, r, rt = _norm_parts(s)
    return dict(r=r.to(IO[c["res"]]), n=(r * rt * s["pre"]).to(IO[c["io"]]))


def _plain_norm_grad(s):
    c, io = s["case"], IO[s["case"]["io"]]
    a, at, p, r, rt = _norm_parts(s)
    dn = s["dn"].float()
    g, out = dn * s["pre"], dict(dpre=(dn * r * rt).sum(0))
    d = s["dr"].float() + rt * (g - r * rt * rt * (g * r).mean(-1, keepdim=True))
    if s["res"] is not None:
        out["dres"] = d.to(IO[c["res"]])
    d = d * s["alpha"]
    if s["scale"] is not None:
        out["dscale"] = (d * p).sum(0)
        d = d * s["scale"]
    if s["post"] is not None:
        out["dpost"] = (d * a * at).sum(0)
        g = d * s["post"]
        d = at * (g - a * at * at * (g * a).mean(-1, keepdim=True))
    if s["z"] is not None:
        z = s["z"].float()
        sg = torch.sigmoid(z)
        out["dz"] = (d * s["x"].float() * sg * (1 + z * (1 - sg))).to(io)
        d = d * z * sg
    out["dx"] = d.to(io)
    return out


def _coefficients(s, dtype=torch.float32):
    """Decay a and what a token adds to the state."""
    r = torch.sigmoid(s["f"].to(dtype) + s["f_bias"].to(dtype))
    v = s["x"].to(dtype)
    if s["i"] is not None:
        v = v * torch.sigmoid(s["i"].to(dtype) + s["i_bias"].to(dtype))
    if s["A"] is None:
        return r, torch.sigmoid(-(s["f"].to(dtype) + s["f_bias"].to(dtype))) * v
    e = s["A"].to(dtype) * r
    return torch.exp(e), torch.sqrt(-torch.expm1(2 * e)) * v


def _scan(a, v, start):
    """All states of h <- a h + v at once by doubling: (a, v) stands for the tokens that a position has taken in so far."""
    n, reach = a.shape[1], 1
    v = v.clone()
    if start is not None:
        v[:, 0] += a[:, 0] * start.to(v.dtype)
    while reach < n:
        v = torch.cat([v[:, :reach], v[:, reach:] + a[:, reach:] * v[:, :-reach]], dim=1)
        if 2 * reach < n:
            a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], dim=1)
        reach *= 2
    return v


def _plain_rec(s):
    c, io = s["case"], IO[s["case"]["io"]]
    start = s["h_in"] if s["src"] is None else s["h_in"][s["src"].long()]
    a, v = _coefficients(s)
    h = _scan(a, v, start)
    y = h
    if s["z"] is not None:
        z = s["z"].float()
        y = h * z * torch.sigmoid(z)
    y = y.to(io)
    if s["lens"] is None:
        return dict(y=y, h=h[:, -1].clone())
    y = torch.where(torch.arange(c["length"], device="cuda")[None, :, None] < s["lens"][:, None, None], y, torch.zeros((), dtype=io, device="cuda"))
    return dict(y=y, h=h[torch.arange(c["batch"], device="cuda"), s["lens"].long() - 1])


def _plain_rec_grad(s):
    c, io = s["case"], IO[s["case"]["io"]]
    n = c["length"]
    live = last = None
    if s["lens"] is not None:
        at = torch.arange(n, device="cuda")[None, :, None]
        live, last = at < s["lens"][:, None, None], at == s["lens"][:, None, None] - 1
    a, v = _coefficients(s)
    start = s["states"][:, 0]
    before = torch.cat([start[:, None], _scan(a, v, start)[:, :-1]], dim=1)      # the state ahead of every token
    h = a * before + v
    dy, out = s["dy"].float(), {}
    g = dy
    if s["z"] is not None:
        z = s["z"].float()
        sg = torch.sigmoid(z)
        g = dy * z * sg
        out["dz"] = dy * h * sg * (1 + z * (1 - sg))
    if live is None:
        g = g.clone()
        g[:, -1] += s["dh_out"]
    else:
        g = torch.where(live, g, torch.zeros_like(g)) + torch.where(last, s["dh_out"][:, None], torch.zeros_like(g))
    # gradients of the states: the same recurrence from the last token to the first, with the decay of the token behind
    back = torch.cat([torch.zeros_like(a[:, :1]), a.flip(1)[:, :-1]], dim=1)
    G = _scan(back, g.flip(1), None).flip(1)
    out["dh_in"] = a[:, 0] * G[:, 0]
    r = torch.sigmoid(s["f"].float() + s["f_bias"])
    x = s["x"].float()
    i = 1.0 if s["i"] is None else torch.sigmoid(s["i"].float() + s["i_bias"])
    if s["A"] is None:
        m = torch.sigmoid(-(s["f"].float() + s["f_bias"]))
        out["df"] = G * (before - i * x) * r * m
    else:
        e = s["A"] * r                                              # log of the decay; its gradient times itself stays finite as it goes to 0
        m = torch.sqrt(-torch.expm1(2 * e))
        de = G * (a * before - i * x * a * a / m)
        out["df"] = de * e * torch.sigmoid(-(s["f"].float() + s["f_bias"]))
        dA = de * r
        out["dA"] = (dA if live is None else torch.where(live, dA, torch.zeros_like(dA))).sum((0, 1))
    out["dx"] = G * m * i
    if s["i"] is not None:
        out["di"] = G * m * x * i * torch.sigmoid(-(s["i"].float() + s["i_bias"]))
    for k in ("dx", "df", "di", "dz"):
        if k in out and live is not None:
            out[k] = torch.where(live, out[k], torch.zeros_like(out[k]))
    out["df_bias"] = out["df"].sum((0, 1))
    if s["i"] is not None:
        out["di_bias"] = out["di"].sum((0, 1))
    for k in ("dx", "df", "di", "dz"):
        if k in out:
            out[k] = out[k].to(io)
    return out


def _plain_rules(s):
    c = s["case"]
    b, V = c["rows"], c["vocab"]
    l, out = s["logits"].float(), {}
    if s["hist"] is not None:
        src = torch.arange(b, device="cuda") if s["src"] is None else s["src"].long()
        hist, length = s["hist"][src], s["hist_len"][src].long()
        at = torch.arange(hist.shape[1], device="cuda")
        hist = torch.where(at == length[:, None], s["token"][:, None], hist)      # there is room for one more
        hist = torch.where(at <= length[:, None], hist, torch.zeros_like(hist))
        out.update(hist=hist, hist_len=(length + 1).int())
        tokens, seen = hist.long(), at <= length[:, None]
        occurs = torch.zeros(b, V, dtype=torch.int32, device="cuda").scatter_add_(1, tokens, seen.int()) > 0
        l = torch.where(occurs, torch.where(l > 0, l / s["rep"][:, None], l * s["rep"][:, None]), l)
        if s["freq"] is not None:
            said = seen & (at >= s["prompt"][:, None])
            count = torch.zeros(b, V, dtype=torch.int32, device="cuda").scatter_add_(1, tokens, said.int())
            l = l - s["freq"][:, None] * count - s["pres"][:, None] * (count > 0)
    if c["bias"]:
        l = l.scatter_add(1, s["bias_token"].long(), s["bias"])
    if c["grammar"]:
        bits = (s["mask"][s["mask_row"].clamp(min=0).long()][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        allowed = (bits.reshape(b, -1)[:, :V] != 0) | (s["mask_row"] < 0)[:, None]
        l = torch.where(allowed, l, torch.full_like(l, -math.inf))
    out["logits"] = l.to(IO[c["io"]])
    return out


# ---- the library's operators --------------------------------------------------------------------------------------------


def _stride(t, d):
    return 0 if t is None else t.stride(d)


def _own_norm(s, ssmv):
    c = s["case"]
    ssmv.ssmv_block_norm(x=s["x"], z=s["z"], res=s["res"], post_wgt=s["post"], ch_scale=s["scale"], pre_wgt=s["pre"], r_out=s["r"], n_out=s["n"],
                         rows=c["rows"], channels=c["channels"], io=c["io"], res_io=c["res"], eps=EPS, res_scale=s["alpha"], z_stride=_stride(s["z"], 0))
    return dict(r=s["r"], n=s["n"])


def _own_norm_grad(s, ssmv):
    c = s["case"]
    if "workspace" not in s:                                                 # kept by the program, like its outputs
        s["workspace"] = torch.empty(ssmv.ssmv_block_norm_backward_workspace(c["rows"], c["channels"]), dtype=torch.uint8, device="cuda")
    ssmv.ssmv_block_norm_backward(x=s["x"], z=s["z"], res=s["res"], post_wgt=s["post"], ch_scale=s["scale"], pre_wgt=s["pre"], dr=s["dr"], dn=s["dn"],
                                  dx=s["dx"], dz=s["dz"], dres=s["dres"], dpost_wgt=s["dpost"], dch_scale=s["dscale"], dpre_wgt=s["dpre"],
                                  rows=c["rows"], channels=c["channels"], io=c["io"], res_io=c["res"], eps=EPS, res_scale=s["alpha"],
                                  z_stride=_stride(s["z"], 0), workspace=s["workspace"])
    return {k: s[k] for k in ("dpre", "dres", "dscale", "dpost", "dz", "dx") if s[k] is not None}


def _own_rec(s, ssmv):
    c = s["case"]
    if "workspace" not in s:
        n = ssmv.ssm_gated_recurrence_workspace(c["batch"], c["channels"], c["length"])
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    ssmv.ssm_gated_recurrence(x=s["x"], f=s["f"], i=s["i"], z=s["z"], A=s["A"], f_bias=s["f_bias"], i_bias=s["i_bias"], h_in=s["h_in"], src_row=s["src"],
                              seq_len=s["lens"], y_out=s["y"], h_out=s["h_out"], batch=c["batch"], channels=c["channels"], L=c["length"], io=c["io"],
                              form=c["form"], x_stride=s["x"].stride(1), f_stride=s["f"].stride(1), i_stride=_stride(s["i"], 1),
                              z_stride=_stride(s["z"], 1), workspace=s["workspace"])
    return dict(y=s["y"], h=s["h_out"])


def _own_rec_grad(s, ssmv):
    c = s["case"]
    if "workspace" not in s:
        n = ssmv.ssm_gated_recurrence_backward_workspace(c["batch"], c["channels"], c["length"])
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    ssmv.ssm_gated_recurrence_backward(x=s["x"], f=s["f"], i=s["i"], z=s["z"], A=s["A"], f_bias=s["f_bias"], i_bias=s["i_bias"], states=s["states"],
                                       seq_len=s["lens"], dy=s["dy"], dh_out=s["dh_out"], dx=s["dx"], df=s["df"], di=s["di"], dz=s["dz"], dA=s["dA"],
                                       df_bias=s["df_bias_out"], di_bias=s["di_bias_out"], dh_in=s["dh_in"], batch=c["batch"], channels=c["channels"],
                                       L=c["length"], io=c["io"], form=c["form"], x_stride=s["x"].stride(1), f_stride=s["f"].stride(1),
                                       i_stride=_stride(s["i"], 1), z_stride=_stride(s["z"], 1), workspace=s["workspace"])
    out = {k: s[k] for k in ("dz", "dh_in", "df", "dA", "dx", "di") if s[k] is not None}
    out["df_bias"] = s["df_bias_out"]
    if s["di_bias_out"] is not None:
        out["di_bias"] = s["di_bias_out"]
    return out


def _own_rules(s, ssmv):
    c = s["case"]
    more = {}
    if s["hist"] is not None:
        more.update(hist=s["hist"], hist_len=s["hist_len"], prompt_len=s["prompt"], src_row=s["src"], token=s["token"], hist_out=s["hist_out"],
                    hist_len_out=s["hist_len_out"], repetition=s["rep"], frequency=s["freq"], presence=s["pres"])
    if c["bias"]:
        more.update(bias_token=s["bias_token"], bias=s["bias"])
    if c["grammar"]:
        more.update(mask=s["mask"], mask_row=s["mask_row"])
    ssmv.ssmv_logit_rules(logits=s["logits"], out=s["out"], rows=c["rows"], vocab=c["vocab"], io=c["io"], row_stride=s["logits"].stride(0),
                          out_stride=s["out"].stride(0), **more)
    out = dict(hist=s["hist_out"], hist_len=s["hist_len_out"]) if s["hist"] is not None else {}
    out["logits"] = s["out"]
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2408_15237_amd as ssmv
        return dict(norm=_own_norm, norm_grad=_own_norm_grad, rec=_own_rec, rec_grad=_own_rec_grad, rules=_own_rules)[kind](state, ssmv)
    return dict(norm=_plain_norm, norm_grad=_plain_norm_grad, rec=_plain_rec, rec_grad=_plain_rec_grad, rules=_plain_rules)[kind](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------


def work(case):
    c = case
    e = 2 if c["io"] == "bf16" else 4
    if c["kind"] in ("norm", "norm_grad"):
        n, C, w = c["rows"] * c["channels"], c["channels"], 2 if c["res"] == "bf16" else 4
        weights = 1 + c["post"] + c["scale"]
        by = n * (e * (1 + c["gate"]) + w * c["residual"]) + 4 * C * weights
        if c["kind"] == "norm":
            return {"bytes": by + n * (w + e), "flops": n * (7 + 5 * c["gate"] + 4 * c["post"] + c["scale"])}
        return {"bytes": by + n * (w + e) + n * (e * (1 + c["gate"]) + w * c["residual"]) + 4 * C * weights,
                "flops": n * (18 + 14 * c["gate"] + 12 * c["post"] + 4 * c["scale"])}
    if c["kind"] in ("rec", "rec_grad"):
        C, lru = c["channels"], c["form"] == "lru"
        tokens = c["length"] * ((c["batch"] + 1) / 2 if c["ragged"] else c["batch"])      # mean length of ragged sequences: half the longest
        ins = 2 + c["inp"] + c["gate"]
        vectors = 4 * C * (lru + 1 + c["inp"])
        if c["kind"] == "rec":
            return {"bytes": tokens * C * e * (ins + 1) + vectors + 4 * c["batch"] * C * (1 + c["resume"]),
                    "flops": tokens * C * (8 + 9 * lru + 6 * c["inp"] + 5 * c["gate"])}
        return {"bytes": tokens * C * (e * (2 * ins + 1) + 4 / TILE) + 2 * vectors + 8 * c["batch"] * C,
                "flops": tokens * C * (22 + 16 * lru + 12 * c["inp"] + 14 * c["gate"])}
    b, V, n = c["rows"], c["vocab"], c["history"]
    by = b * V * e * (1 if c["in_place"] else 2) + (b + c["grammar"]) * ((V + 31) // 32) * 4 * (c["grammar"] > 0)
    return {"bytes": by + 8 * b * n + 8 * b * c["bias"] + 40 * b, "flops": 2 * b * V}


# ---- the same in 64 bits, from the definitions ----------------------------------------------------------------------------


def _leaf(t, grads):
    """An input in 64 bits; for the gradients a leaf of its own."""
    return None if t is None else t.double().detach().clone().requires_grad_(grads)


def _exact_norm(c, s):
    grads = c["kind"] == "norm_grad"
    v = {k: _leaf(s[k], grads) for k in ("x", "z", "res", "post", "scale", "pre")}
    unit = lambda t: t / torch.sqrt(t.square().sum(-1, keepdim=True) / c["channels"] + EPS)
    p = v["x"] if v["z"] is None else v["x"] * v["z"] / (1 + torch.exp(-v["z"]))
    if v["post"] is not None:
        p = unit(p) * v["post"]
    r = p * s["alpha"] if v["scale"] is None else p * s["alpha"] * v["scale"]
    if v["res"] is not None:
        r = v["res"] + r
    n = unit(r) * v["pre"]
    if not grads:
        return dict(r=r, n=n)
    names = [k for k in v if v[k] is not None]
    got = torch.autograd.grad([r, n], [v[k] for k in names], [s["dr"].double(), s["dn"].double()])
    return {"d" + k: t for k, t in zip(names, got)}


def _exact_rec(c, s):
    grads = c["kind"] == "rec_grad"
    b, n = c["batch"], c["length"]
    v = {k: _leaf(s[k], grads) for k in ("x", "f", "i", "z", "A", "f_bias", "i_bias")}
    start = s["states"][:, 0] if grads else s["h_in"] if s["src"] is None else s["h_in"].index_select(0, s["src"])
    h = first = torch.zeros(b, c["channels"], dtype=torch.float64, device="cuda").requires_grad_(grads) if start is None else _leaf(start, grads)
    gate = 1 / (1 + torch.exp(-(v["f"] + v["f_bias"])))
    keep = gate if v["A"] is None else torch.exp(v["A"] * gate)
    take = 1 / (1 + torch.exp(v["f"] + v["f_bias"])) if v["A"] is None else torch.sqrt((1 - keep) * (1 + keep))
    new = take * v["x"] if v["i"] is None else take * v["x"] / (1 + torch.exp(-(v["i"] + v["i_bias"])))
    if s["lens"] is not None:                                      # tokens that are none leave the state as it is
        live = (torch.arange(n, device="cuda") < s["lens"][:, None])[..., None]
        keep, new = torch.where(live, keep, torch.ones_like(keep)), torch.where(live, new, torch.zeros_like(new))
    states = []
    for a, u in zip(keep.unbind(1), new.unbind(1)):
        h = torch.addcmul(u, a, h)
        states.append(h)
    y = torch.stack(states, 1)
    if v["z"] is not None:
        y = y * v["z"] / (1 + torch.exp(-v["z"]))
    if s["lens"] is not None:
        y = torch.where(live, y, torch.zeros_like(y))
    if not grads:
        return dict(y=y, h=h)
    names = [k for k in v if v[k] is not None]
    got = torch.autograd.grad([y, h], [v[k] for k in names] + [first], [s["dy"].double(), s["dh_out"].double()])
    return {"d" + k: t for k, t in zip(names + ["h_in"], got)}


def _exact_rules(c, s):
    rows = []
    for k in range(c["rows"]):
        l = s["logits"][k].double().clone()
        if s["hist"] is not None:
            j = k if s["src"] is None else int(s["src"][k])
            said = torch.cat([s["hist"][j, :int(s["hist_len"][j])], s["token"][k:k + 1]]).long()
            once = said.unique()
            p = s["rep"][k].double()
            l[once] = torch.where(l[once] > 0, l[once] / p, l[once] * p)
            if s["freq"] is not None:
                some, times = said[int(s["prompt"][k]):].unique(return_counts=True)
                l[some] -= s["freq"][k].double() * times + s["pres"][k].double()
        if c["bias"]:
            l.index_put_((s["bias_token"][k].long(),), s["bias"][k].double(), accumulate=True)
        if c["grammar"] and int(s["mask_row"][k]) >= 0:
            words = s["mask"][int(s["mask_row"][k])].long()
            bit = torch.arange(c["vocab"], device="cuda")
            l[(words[bit // 32] >> (bit % 32)) % 2 == 0] = -math.inf
        rows.append(l)
    out = dict(hist=None, hist_len=None) if s["hist"] is not None else {}
    return dict(out, logits=torch.stack(rows))


def exact(case, seed):
    s = prepare(case, seed)
    return dict(norm=_exact_norm, norm_grad=_exact_norm, rec=_exact_rec, rec_grad=_exact_rec, rules=_exact_rules)[case["kind"]](case, s)
