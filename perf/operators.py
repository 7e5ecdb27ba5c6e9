"""The operators of plain decoding with a selective state-space model, as cases that can be timed and compared.

Four kinds of pass, together what a beam search over such a model does:

* "conv": the width-4 causal convolution over a prompt, or over one new token of every beam, from a history of raw inputs to the
  newest one (ssm_causal_conv).
* "scan": a prompt through the recurrence with a decay per channel and state index (ssm_selective_scan).
* "step": one token of every row through the recurrence, diagonal or with one decay per head, each row continuing the state of
  the beam that it descends from (ssm_selective_step).
* "beam": the choice of the best continuations over all beams and the vocabulary (ssmv_beam_select).

`own` False computes them in elementary torch operations.  Distributions are those of `workload`: x ~ N(0,1), B, C ~
N(0,1)/sqrt(dstate), raw step sizes N(0,1) - 4, A = -(n+1) + U(-1/4, 1/4) per channel or -exp(U(0, ln 16)) per head; logits
~ 3 N(0,1), a few of them masked.
"""
from __future__ import annotations

import math

import torch

own = False

IO = {"bf16": torch.bfloat16, "f32": torch.float32}
EOS = 2

_CONV = dict(kind="conv", io="bf16", batch=1, length=2048, channels=8192, act="silu", ragged=False, beams=False, split=True)
_SCAN = dict(kind="scan", io="bf16", batch=1, length=2048, channels=8192, dstate=16, softplus=True, gate=True, ragged=False, resume=False)
_STEP = dict(kind="step", io="bf16", mode="diag", rows=4, heads=8192, headdim=1, dstate=16, groups=1, softplus=True, gate=True, beams=True)
_BEAM = dict(kind="beam", io="bf16", batch=1, beams_in=4, beams_out=4, vocab=32000, pad=0, done=True, masked=True)


def listed():
    return [
        # one user's four beams: a new token each, the histories in the order that the last selection left
        dict(_CONV, name="conv_token_b4", batch=4, length=1, beams=True),
        # the prompts of a serving batch, of different lengths; x is one half of a projection's output
        dict(_CONV, name="conv_prompt_b8", batch=8, channels=5120, ragged=True),
        # fp32 tensors, a channel count that no vector divides, a continued prompt
        dict(_CONV, name="conv_f32_odd", io="f32", batch=3, length=333, channels=1001, act="none", split=False),
        # one user's prompt through the Mamba-1 style layer
        dict(_SCAN, name="scan_prompt_b1"),
        # the prompts of a serving batch, of different lengths
        dict(_SCAN, name="scan_prompt_b8", batch=8, channels=5120, ragged=True),
        # fp32 tensors, a short continuation of two sequences, a larger state
        dict(_SCAN, name="scan_f32_short", io="f32", batch=2, length=37, channels=1000, dstate=32, softplus=False, gate=False, resume=True),
        # one user's four beams, one token each
        dict(_STEP, name="step_b4"),
        # a serving batch: 64 requests of four beams
        dict(_STEP, name="step_b256", rows=256, heads=5120),
        # a serving batch of the 8B shape, one decay per head
        dict(_STEP, name="step_heads_b48", mode="scalar", rows=48, heads=32, headdim=128, dstate=64),
        # the first choice after one user's prompt: one beam becomes four
        dict(_BEAM, name="beam_first", io="f32", beams_in=1, done=False, masked=False),
        # a serving batch with eight beams each over a large vocabulary, rows padded to whole lines
        dict(_BEAM, name="beam_serving", batch=16, beams_in=8, beams_out=8, vocab=128011, pad=53),
        # twice as many candidates as beams, an odd vocabulary
        dict(_BEAM, name="beam_wide_odd", batch=5, beams_in=3, beams_out=6, vocab=49999),
    ]


def _log_int(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _channels(rng):
    """Mostly whole vectors of channels, sometimes any number."""
    return 16 * _log_int(rng, 4, 512) if rng.random() < 0.75 else _log_int(rng, 64, 8192)


def draw(rng):
    kind = rng.choice(["conv", "scan", "scan", "step", "step", "beam", "beam"])
    io = rng.choice(["bf16", "bf16", "f32"])
    if kind == "conv":
        channels, most = _channels(rng), 8 * 2048 * 5120 // (2 if io == "f32" else 1)
        beams = rng.random() < 0.4
        length = 1 if beams else _log_int(rng, 1, 4096)
        batch = _log_int(rng, 1, max(1, min(256 if beams else 32, most // (length * channels))))
        return dict(_CONV, io=io, batch=batch, length=length, channels=channels, act=rng.choice(["silu", "silu", "none"]),
                    ragged=batch > 1 and not beams and rng.random() < 0.5, beams=beams, split=rng.random() < 0.5)
    if kind == "scan":
        channels, dstate = _channels(rng), rng.choice([16, 16, 16, 32, 64])
        most = 8 * 2048 * 5120 * 16 // (2 if io == "f32" else 1)
        length = _log_int(rng, 1, min(4096, most // (channels * dstate)))
        batch = _log_int(rng, 1, max(1, min(32, most // (length * channels * dstate))))
        return dict(_SCAN, io=io, batch=batch, length=length, channels=channels, dstate=dstate, softplus=rng.random() < 0.7,
                    gate=rng.random() < 0.7, ragged=batch > 1 and rng.random() < 0.5, resume=rng.random() < 0.5)
    if kind == "step":
        mode = rng.choice(["diag", "scalar"])
        if mode == "diag":
            heads, headdim, groups, dstate = _channels(rng), 1, 1, rng.choice([16, 16, 16, 32, 64])
        else:
            heads, headdim, dstate = _log_int(rng, 4, 80), rng.choice([32, 48, 64, 64, 128, 128]), rng.choice([16, 32, 64, 64, 128, 256])
            groups = rng.choice([g for g in (1, 1, 2, 4, 8) if heads % g == 0])
        rows = _log_int(rng, 1, max(1, min(256, 256 * 5120 * 16 // (heads * headdim * dstate))))
        return dict(_STEP, io=io, mode=mode, rows=rows, heads=heads, headdim=headdim, dstate=dstate, groups=groups,
                    softplus=rng.random() < 0.7, gate=rng.random() < 0.7, beams=rng.random() < 0.7)
    beams_in = rng.choice([1, 2, 3, 4, 4, 5, 8, 16])
    beams_out = rng.choice([beams_in, beams_in, 2 * beams_in, rng.randint(1, 16)])
    vocab = _log_int(rng, 500, 160000)
    batch = _log_int(rng, 1, max(1, min(64, 16 * 8 * 128011 // (2 if io == "f32" else 1) // (beams_in * vocab))))
    return dict(_BEAM, io=io, batch=batch, beams_in=beams_in, beams_out=beams_out, vocab=vocab, pad=rng.choice([0, 0, -vocab % 64]),
                done=rng.random() < 0.5, masked=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------------------------------


def _rng(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + what) % (1 << 62))
    return lambda *s: torch.randn(*s, generator=g, device="cuda"), lambda *s: torch.rand(*s, generator=g, device="cuda"), g


def _lengths(c, seed):
    """Prompt lengths: the longest is c["length"]; ragged prompts from one token up."""
    g = torch.Generator().manual_seed(int(seed) * 17 + 3)
    n = torch.randint(1, c["length"] + 1, (c["batch"],), generator=g)
    n[0] = c["length"]
    return n.int().cuda() if c["ragged"] else None


def _prepare_conv(c, seed):
    randn, rand, g = _rng(seed, 1)
    b, n, C, io = c["batch"], c["length"], c["channels"], IO[c["io"]]
    # a prompt's x is the first half of a projection's output where that is so ("split")
    proj = randn(b, n, 2 * C if c["split"] else C).to(io)
    return dict(case=c, x=proj[..., :C], w=(randn(C, 4) / 2).to(io), bias=(randn(C) * 0.1).to(io), conv_in=randn(b, 3, C).to(io),
                src=torch.randint(0, b, (b,), generator=g, device="cuda", dtype=torch.int32) if c["beams"] else None, lens=_lengths(c, seed),
                out=torch.zeros(b, n, C, dtype=io, device="cuda"), conv_out=torch.zeros(b, 3, C, dtype=io, device="cuda"))


def _step_size(c, raw):
    """The raw step size where the operator takes its softplus, the positive one otherwise."""
    return raw if c["softplus"] else torch.nn.functional.softplus(raw)


def _diagonal(rand, H, N):
    return -(torch.arange(1, N + 1, device="cuda", dtype=torch.float32) + (rand(H, N) - 0.5) * 0.5)


def _prepare_scan(c, seed):
    randn, rand, _ = _rng(seed, 2)
    b, n, C, N, io = c["batch"], c["length"], c["channels"], c["dstate"], IO[c["io"]]
    proj = randn(b, n, 2 * C).to(io) if c["gate"] else None        # the input projection's output: z is its second half
    bc = (randn(b, n, 2 * N) / N ** 0.5).to(io)                    # B and C lie side by side, as their projection leaves them
    return dict(case=c, x=randn(b, n, C).to(io), dt=_step_size(c, randn(b, n, C) - 4.0).to(io), B=bc[..., :N], C=bc[..., N:],
                z=proj[..., C:] if c["gate"] else None, A=_diagonal(rand, C, N), D=randn(C), dt_bias=rand(C) - 0.5 if c["softplus"] else None,
                h_in=randn(b, C, N) * 0.1 if c["resume"] else None, lens=_lengths(c, seed),
                y=torch.zeros(b, n, C, dtype=io, device="cuda"), h_out=torch.zeros(b, C, N, device="cuda"))


def _prepare_step(c, seed):
    randn, rand, g = _rng(seed, 3)
    b, H, P, N, G, io = c["rows"], c["heads"], c["headdim"], c["dstate"], c["groups"], IO[c["io"]]
    A = _diagonal(rand, H, N) if c["mode"] == "diag" else -torch.exp(rand(H) * math.log(16.0))
    return dict(case=c, x=randn(b, H * P).to(io), dt=_step_size(c, randn(b, H) - 4.0).to(io), B=(randn(b, G, N) / N ** 0.5).to(io),
                C=(randn(b, G, N) / N ** 0.5).to(io), z=randn(b, H * P).to(io) if c["gate"] else None, A=A, D=randn(H),
                dt_bias=rand(H) - 0.5 if c["softplus"] else None, h_in=randn(b, H, P, N) * 0.1,
                src=torch.randint(0, b, (b,), generator=g, device="cuda", dtype=torch.int32) if c["beams"] else None,
                y=torch.zeros(b, H * P, dtype=io, device="cuda"), h_out=torch.zeros(b, H, P, N, device="cuda"))


def _prepare_beam(c, seed):
    randn, rand, _ = _rng(seed, 4)
    b, W, K, V = c["batch"], c["beams_in"], c["beams_out"], c["vocab"]
    logits = (3 * randn(b * W, V + c["pad"])).to(IO[c["io"]])
    if c["masked"]:                                                # tokens that the request does not allow
        logits[rand(*logits.shape) < 0.05] = -math.inf
    done = (rand(b * W) < 0.15).int() if c["done"] else None
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(case=c, logits=logits[:, :V], scores=-(20.0 + 2.0 * randn(b * W).abs()), done=done, parent=torch.zeros(b * K, **i32),
                token=torch.zeros(b * K, **i32), scores_out=torch.zeros(b * K, device="cuda"), done_out=torch.zeros(b * K, **i32))


def prepare(case, seed):
    return dict(conv=_prepare_conv, scan=_prepare_scan, step=_prepare_step, beam=_prepare_beam)[case["kind"]](case, seed)


# ---- plain forms --------------------------------------------------------------------------------------------------------


def _silu(v):
    return v * torch.sigmoid(v)


def _softplus(v):
    return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-v.abs()))


def _plain_conv(s):
    c, io = s["case"], IO[s["case"]["io"]]
    n = c["length"]
    hist = s["conv_in"] if s["src"] is None else s["conv_in"][s["src"].long()]
    raw = torch.cat([hist, s["x"]], dim=1)
    f, w = raw.float(), s["w"].float()
    out = s["bias"].float() + f[:, 0:n] * w[:, 0] + f[:, 1:n + 1] * w[:, 1] + f[:, 2:n + 2] * w[:, 2] + f[:, 3:n + 3] * w[:, 3]
    out = (_silu(out) if c["act"] == "silu" else out).to(io)
    if s["lens"] is None:
        return dict(out=out, conv=raw[:, n:].clone())
    out = torch.where(torch.arange(n, device="cuda")[None, :, None] < s["lens"][:, None, None], out, torch.zeros((), dtype=io, device="cuda"))
    at = s["lens"].long()[:, None] + torch.arange(3, device="cuda")
    return dict(out=out, conv=torch.gather(raw, 1, at[:, :, None].expand(-1, -1, c["channels"])))


def _plain_scan(s):
    """All prefixes at once by doubling: (a, v) stands for h -> a h + v over the tokens that a position has taken in so far."""
    c, io = s["case"], IO[s["case"]["io"]]
    n = c["length"]
    x, dt = s["x"].float(), s["dt"].float()
    if c["softplus"]:
        dt = _softplus(dt + s["dt_bias"])
    a = torch.exp(dt[..., None] * s["A"])
    v = (dt * x)[..., None] * s["B"].float()[:, :, None, :]
    if c["resume"]:
        v[:, 0] += a[:, 0] * s["h_in"]
    reach = 1
    while reach < n:
        v = torch.cat([v[:, :reach], v[:, reach:] + a[:, reach:] * v[:, :-reach]], dim=1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], dim=1)
        reach *= 2
    y = (v * s["C"].float()[:, :, None, :]).sum(-1) + s["D"] * x
    if c["gate"]:
        y = y * _silu(s["z"].float())
    y = y.to(io)
    if s["lens"] is None:
        return dict(y=y, h=v[:, -1].contiguous())
    y = torch.where(torch.arange(n, device="cuda")[None, :, None] < s["lens"][:, None, None], y, torch.zeros((), dtype=io, device="cuda"))
    return dict(y=y, h=v[torch.arange(c["batch"], device="cuda"), s["lens"].long() - 1])


def _plain_step(s):
    c, io = s["case"], IO[s["case"]["io"]]
    b, H, P, N, G = c["rows"], c["heads"], c["headdim"], c["dstate"], c["groups"]
    h = s["h_in"] if s["src"] is None else s["h_in"][s["src"].long()]
    x, dt = s["x"].float().view(b, H, P), s["dt"].float()
    if c["softplus"]:
        dt = _softplus(dt + s["dt_bias"])
    A = s["A"] if c["mode"] == "diag" else s["A"][:, None]
    B, C = (s[k].float().repeat_interleave(H // G, dim=1) if c["mode"] == "scalar" else s[k].float() for k in ("B", "C"))
    h = h * torch.exp(dt[:, :, None] * A)[:, :, None, :] + (dt[:, :, None] * x)[..., None] * B[:, :, None, :]
    y = (h * C[:, :, None, :]).sum(-1) + s["D"][:, None] * x
    y = y.reshape(b, H * P)
    return dict(y=(y * _silu(s["z"].float()) if c["gate"] else y).to(io), h=h)


def _plain_beam(s):
    """Scores in 64 bits: two candidates of different beams may lie as near to each other as they like."""
    c = s["case"]
    b, W, K, V = c["batch"], c["beams_in"], c["beams_out"], c["vocab"]
    # NaN is a masked token, +inf the largest finite logit
    logits = torch.nan_to_num(s["logits"].float(), nan=-math.inf, posinf=torch.finfo(torch.float32).max, neginf=-math.inf)
    best = logits.max(-1, keepdim=True).values.clamp(min=torch.finfo(torch.float32).min).double()
    total = torch.exp(logits.double() - best).sum(-1).clamp(min=1e-300)       # 0 where every token is masked: all its scores are -inf
    # a row's candidates in the order of their logits, equal ones by index: both in one whole number
    bits = logits.contiguous().view(torch.int32)
    bits = torch.where(bits == -2 ** 31, torch.zeros_like(bits), bits)       # -0 is 0
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    index = torch.arange(V, device="cuda")
    keys = torch.topk(order * 2 ** 32 + (2 ** 32 - 1 - index), min(K, V), dim=-1).values
    token = 2 ** 32 - 1 - (keys & (2 ** 32 - 1))
    score = s["scores"].double()[:, None] + (torch.gather(logits, 1, token).double() - best - torch.log(total)[:, None])
    if c["done"]:                                                            # a finished beam continues as it is, and in no other way
        done = s["done"] != 0
        first = torch.arange(min(K, V), device="cuda") == 0
        score = torch.where(done[:, None], torch.where(first, s["scores"].double()[:, None], -math.inf), score)
        token = torch.where(done[:, None], EOS, token)
    k = min(K, V)
    at = torch.sort(score.view(b, W * k), dim=1, descending=True, stable=True).indices[:, :K]
    parent = at // k + torch.arange(b, device="cuda")[:, None] * W
    token = torch.gather(token.view(b, W * k), 1, at)
    out = dict(parent=parent.reshape(-1).int(), token=token.reshape(-1).int(), scores=torch.gather(score.view(b, W * k), 1, at).reshape(-1).float())
    if c["done"]:
        out["done"] = ((s["done"][out["parent"].long()] != 0) | (out["token"] == EOS)).int()
    return out


# ---- the library's operators --------------------------------------------------------------------------------------------


def _own_conv(s, ssmv):
    c = s["case"]
    ssmv.ssm_causal_conv(x=s["x"], wgt=s["w"], bias=s["bias"], out=s["out"], batch=c["batch"], channels=c["channels"], L=c["length"], io=c["io"],
                         act=c["act"], conv_in=s["conv_in"], conv_out=s["conv_out"], src_row=s["src"], seq_len=s["lens"],
                         x_stride=s["x"].stride(1))
    return dict(out=s["out"], conv=s["conv_out"])


def _own_scan(s, ssmv):
    c = s["case"]
    if "workspace" not in s:                                                 # kept by the program, like its outputs
        n = ssmv.ssm_selective_scan_workspace(c["batch"], c["channels"], c["dstate"], c["length"])
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    ssmv.ssm_selective_scan(x=s["x"], dt=s["dt"], A=s["A"], Bm=s["B"], Cm=s["C"], D=s["D"], y_out=s["y"], batch=c["batch"],
                            channels=c["channels"], dstate=c["dstate"], L=c["length"], io=c["io"], dt_bias=s["dt_bias"],
                            dt_softplus=c["softplus"], z=s["z"], h_in=s["h_in"], h_out=s["h_out"], seq_len=s["lens"],
                            b_stride=s["B"].stride(1), c_stride=s["C"].stride(1), z_stride=s["z"].stride(1) if c["gate"] else 0,
                            workspace=s["workspace"])
    return dict(y=s["y"], h=s["h_out"])


def _own_step(s, ssmv):
    c = s["case"]
    ssmv.ssm_selective_step(x=s["x"], dt=s["dt"], A=s["A"], Bm=s["B"], Cm=s["C"], D=s["D"], y_out=s["y"], h_in=s["h_in"], h_out=s["h_out"],
                            rows=c["rows"], nheads=c["heads"], headdim=c["headdim"], dstate=c["dstate"], ngroups=c["groups"], io=c["io"],
                            a_mode=c["mode"], dt_bias=s["dt_bias"], dt_softplus=c["softplus"], z=s["z"], src_row=s["src"])
    return dict(y=s["y"], h=s["h_out"])


def _own_beam(s, ssmv):
    c = s["case"]
    if "workspace" not in s:
        s["workspace"] = torch.empty(ssmv.ssmv_beam_workspace(c["batch"], c["beams_in"], c["beams_out"], c["vocab"]), dtype=torch.uint8, device="cuda")
    ssmv.ssmv_beam_select(logits=s["logits"], scores=s["scores"], parent=s["parent"], token=s["token"], scores_out=s["scores_out"],
                          batch=c["batch"], beams_in=c["beams_in"], beams_out=c["beams_out"], vocab=c["vocab"], io=c["io"],
                          row_stride=s["logits"].stride(0), done=s["done"], done_out=s["done_out"] if c["done"] else None, eos=EOS,
                          workspace=s["workspace"])
    out = dict(parent=s["parent"], token=s["token"], scores=s["scores_out"])
    if c["done"]:
        out["done"] = s["done_out"]
    return out


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2408_15237_amd as ssmv
        return dict(conv=_own_conv, scan=_own_scan, step=_own_step, beam=_own_beam)[kind](state, ssmv)
    return dict(conv=_plain_conv, scan=_plain_scan, step=_plain_step, beam=_plain_beam)[kind](state)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------


def work(case):
    c = case
    e = 2 if c["io"] == "bf16" else 4
    if c["kind"] == "conv":
        tokens = c["length"] * ((c["batch"] + 1) / 2 if c["ragged"] else c["batch"])      # mean length of ragged prompts: half the longest
        n = tokens * c["channels"]
        return {"bytes": 2 * n * e + c["channels"] * (5 + 6 * c["batch"]) * e, "flops": n * (9 if c["act"] == "none" else 13)}
    if c["kind"] == "scan":
        C, N = c["channels"], c["dstate"]
        tokens = c["length"] * ((c["batch"] + 1) / 2 if c["ragged"] else c["batch"])
        by = tokens * ((4 if c["gate"] else 3) * C + 2 * N) * e + C * (N + 2) * 4 + c["batch"] * C * N * 4 * (2 if c["resume"] else 1)
        return {"bytes": by, "flops": tokens * C * (7 * N + 4 + (4 if c["softplus"] else 0) + (5 if c["gate"] else 0))}
    if c["kind"] == "step":
        b, H, P, N = c["rows"], c["heads"], c["headdim"], c["dstate"]
        tok = (3 if c["gate"] else 2) * H * P + H + 2 * c["groups"] * N
        return {"bytes": 8 * b * H * P * N + b * tok * e + 4 * H * ((N if c["mode"] == "diag" else 1) + 2),
                "flops": b * H * P * (N * (7 if c["mode"] == "diag" else 5) + 8)}
    rows = c["batch"] * c["beams_in"]
    return {"bytes": rows * (c["vocab"] * e + 8) + 16 * c["batch"] * c["beams_out"], "flops": rows * c["vocab"] * 4}


# ---- the same in 64 bits, from the definitions ----------------------------------------------------------------------------


def _exact_conv(s):
    c = s["case"]
    b, n = c["batch"], c["length"]
    start = list(range(b)) if s["src"] is None else s["src"].tolist()
    lens = [n] * b if s["lens"] is None else s["lens"].tolist()
    w, out, conv = s["w"].double(), torch.zeros(b, n, c["channels"], dtype=torch.float64, device="cuda"), []
    for i in range(b):
        raw = torch.cat([s["conv_in"][start[i]].double(), s["x"][i, :lens[i]].double()])
        v = s["bias"].double() + sum(raw[k:k + lens[i]] * w[:, k] for k in range(4))
        out[i, :lens[i]] = v / (1 + torch.exp(-v)) if c["act"] == "silu" else v
        conv.append(raw[-3:])
    return dict(out=out, conv=torch.stack(conv))


def _exact_scan(s):
    c = s["case"]
    b, n, C, N = c["batch"], c["length"], c["channels"], c["dstate"]
    lens = torch.full((b,), n, device="cuda") if s["lens"] is None else s["lens"]
    h = torch.zeros(b, C, N, dtype=torch.float64, device="cuda") if s["h_in"] is None else s["h_in"].double()
    A, D, y = s["A"].double(), s["D"].double(), torch.zeros(b, n, C, dtype=torch.float64, device="cuda")
    for t in range(n):
        dt, x = s["dt"][:, t].double(), s["x"][:, t].double()
        if c["softplus"]:
            dt = torch.logaddexp(dt + s["dt_bias"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        new = torch.exp(dt[:, :, None] * A) * h + (dt * x)[:, :, None] * s["B"][:, t, None].double()
        at = torch.matmul(new, s["C"][:, t, :, None].double())[..., 0] + D * x
        if c["gate"]:
            z = s["z"][:, t].double()
            at = at * z / (1 + torch.exp(-z))
        live = (t < lens)[:, None]
        y[:, t] = torch.where(live, at, torch.zeros_like(at))
        h = torch.where(live[:, :, None], new, h)
    return dict(y=y, h=h)


def _exact_step(s):
    c = s["case"]
    b, H, P, N, G = c["rows"], c["heads"], c["headdim"], c["dstate"], c["groups"]
    y, hs = [], []
    start = range(b) if s["src"] is None else s["src"].tolist()
    group = torch.arange(H, device="cuda") * G // H if c["mode"] == "scalar" else torch.zeros(H, dtype=torch.long, device="cuda")
    for i, row in enumerate(start):
        dt, x = s["dt"][i].double(), s["x"][i].double().view(H, P)
        if c["softplus"]:
            dt = torch.logaddexp(dt + s["dt_bias"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
        decay = torch.exp(dt.view(H, 1) * s["A"].double().view(H, -1)).view(H, 1, -1)
        h = decay * s["h_in"][row].double() + dt[:, None, None] * x[:, :, None] * s["B"][i].double()[group][:, None]
        v = (torch.matmul(h, s["C"][i].double()[group][:, :, None])[..., 0] + s["D"].double()[:, None] * x).view(-1)
        if c["gate"]:
            z = s["z"][i].double()
            v = v * z / (1 + torch.exp(-z))
        y.append(v)
        hs.append(h)
    return dict(y=torch.stack(y), h=torch.stack(hs))


def _exact_beam(s):
    c = s["case"]
    b, W, K, V = c["batch"], c["beams_in"], c["beams_out"], c["vocab"]
    got = []
    for i in range(b):
        rows = s["logits"][i * W:(i + 1) * W].double()
        cand = s["scores"][i * W:(i + 1) * W].double()[:, None] + rows - torch.logsumexp(rows, -1, keepdim=True)
        if c["done"]:
            done = s["done"][i * W:(i + 1) * W] != 0
            cand[done] = -math.inf
            cand[done, EOS] = s["scores"][i * W:(i + 1) * W].double()[done]
        got.append(torch.sort(cand.view(-1), descending=True).values[:K])
    scores = torch.cat(got)
    return dict(parent=None, token=None, scores=scores, **(dict(done=None) if c["done"] else {}))


def exact(case, seed):
    c = case
    if c["kind"] == "scan" and c["length"] * (1e-4 + 1e-11 * c["batch"] * c["channels"] * c["dstate"]) > 15:
        return None                                          # over about 20 seconds
    s = prepare(case, seed)
    return dict(conv=_exact_conv, scan=_exact_scan, step=_exact_step, beam=_exact_beam)[c["kind"]](s)
