"""Beam search over a small Mamba-1 style language model (random weights): the prompt by whole-prompt calls, then a token a step.

Every layer of the model keeps one state a row: h (fp32) and the newest three conv inputs.  A prompt goes through
ssm_causal_conv and ssm_selective_scan, a new token through ssm_causal_conv and ssm_selective_step; ssmv_beam_select names for every
new beam the row that it descends from, and the next step's calls read that row's state.  Nothing is copied to reorder the beams.
With --repetition, ssmv_logit_rules makes the tokens that a beam's prompt and its own text hold less likely ahead of every choice.

    python examples/beam_decode.py [--layers 4] [--width 1024] [--beams 4] [--prompt 256] [--tokens 32] [--dtype bf16] [--repetition 1.2]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2408_15237_amd as ssmv  # noqa: E402

IO = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def make_weights(layers=2, width=128, inner=256, dstate=16, dt_rank=8, vocab=512, io="bf16", seed=0):
    """Weights of the model as CPU tensors that `io` represents exactly."""
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: (torch.randn(*s, generator=g) / s[-1] ** 0.5).to(IO[io])
    out = dict(io=io, width=width, inner=inner, dstate=dstate, dt_rank=dt_rank, vocab=vocab, embed=torch.randn(vocab, width, generator=g).to(IO[io]),
               norm=torch.ones(width), head=(4 * rand(vocab, width).float()).to(IO[io]), layers=[])
    for _ in range(layers):
        out["layers"].append(dict(norm=torch.ones(width), in_proj=rand(2 * inner, width), conv_w=(torch.randn(inner, 4, generator=g) / 2).to(IO[io]),
                                  conv_b=(torch.randn(inner, generator=g) * 0.1).to(IO[io]), x_proj=rand(dt_rank + 2 * dstate, inner),
                                  dt_proj=rand(inner, dt_rank), dt_bias=torch.rand(inner, generator=g) - 3.5,
                                  A=-torch.arange(1, dstate + 1, dtype=torch.float32).repeat(inner, 1), D=torch.ones(inner), out_proj=rand(width, inner)))
    return out


class Model:
    """The weights on the GPU, and the states of the rows that are being decoded."""

    def __init__(self, weights):
        move = lambda d: {k: v.cuda() if torch.is_tensor(v) else v for k, v in d.items() if k != "layers"}
        self.w, self.layers = move(weights), [move(x) for x in weights["layers"]]
        self.io, self.dtype = weights["io"], IO[weights["io"]]
        self.reset()

    def reset(self):
        """Empty states: what comes next is a prompt."""
        self.h, self.conv = [None] * len(self.layers), [None] * len(self.layers)

    def _norm(self, x, weight):
        flat, out = x.reshape(-1, x.shape[-1]), torch.empty_like(x)
        ssmv.ssmv_gated_rmsnorm(flat, None, weight, flat.shape[0], flat.shape[1], flat.shape[1], EPS, self.io, out)
        return out

    def _layer(self, i, u, src_row, seq_len):
        """One layer over u [rows][n][width]: its output, with the layer's states moved on (n > 1: a prompt, from empty states)."""
        w, io = self.layers[i], self.io
        C, N, R, rows, n = self.w["inner"], self.w["dstate"], self.w["dt_rank"], u.shape[0], u.shape[1]
        xz = u @ w["in_proj"].T                                               # x and z side by side
        xc, conv = torch.empty(rows, n, C, dtype=self.dtype, device="cuda"), torch.empty(rows, 3, C, dtype=self.dtype, device="cuda")
        ssmv.ssm_causal_conv(x=xz, wgt=w["conv_w"], bias=w["conv_b"], conv_in=self.conv[i], conv_out=conv, src_row=src_row, seq_len=seq_len, out=xc,
                             batch=rows, channels=C, L=n, io=io, act="silu", x_stride=2 * C)
        proj = xc @ w["x_proj"].T                                             # the low-rank step, B and C side by side
        dt = proj[..., :R] @ w["dt_proj"].T
        B, Cm, z = proj[..., R:R + N], proj[..., R + N:], xz[..., C:]
        y, h, wide = torch.empty_like(xc), torch.empty(rows, C, N, device="cuda"), R + 2 * N
        if n == 1:
            ssmv.ssm_selective_step(x=xc, dt=dt, A=w["A"], Bm=B, Cm=Cm, D=w["D"], y_out=y, h_in=self.h[i], h_out=h, rows=rows, nheads=C, headdim=1,
                                    dstate=N, io=io, a_mode="diag", dt_bias=w["dt_bias"], dt_softplus=True, z=z, src_row=src_row, b_stride=wide,
                                    c_stride=wide, z_stride=2 * C)
        else:
            need = ssmv.ssm_selective_scan_workspace(rows, C, N, n)
            ssmv.ssm_selective_scan(x=xc, dt=dt, A=w["A"], Bm=B, Cm=Cm, D=w["D"], y_out=y, h_out=h, batch=rows, channels=C, dstate=N, L=n, io=io,
                                    dt_bias=w["dt_bias"], dt_softplus=True, z=z, seq_len=seq_len, b_stride=wide, c_stride=wide, z_stride=2 * C,
                                    workspace=torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
        self.h[i], self.conv[i] = h, conv
        return y @ w["out_proj"].T

    def forward(self, tokens, src_row=None, seq_len=None):
        """Logits after the last token of every row; tokens [rows][n]."""
        x = self.w["embed"][tokens.long()]
        for i, w in enumerate(self.layers):
            x = x + self._layer(i, self._norm(x, w["norm"]), src_row, seq_len)
        last = x[:, -1] if seq_len is None else x[torch.arange(x.shape[0], device="cuda"), seq_len.long() - 1]
        return self._norm(last.contiguous(), self.w["norm"]) @ self.w["head"].T


class Histories:
    """What every beam has read and said, and a penalty on its tokens: logits of a token that occurs are divided by it where they are positive, else multiplied."""

    def __init__(self, prompts, lengths, steps, penalty):
        self.penalty = penalty
        self.room = prompts.shape[1] + steps
        self.tokens, self.length = torch.nn.functional.pad(prompts, (0, steps)).contiguous(), lengths.int()

    def apply(self, model, logits, parent, token):
        rows, i32 = logits.shape[0], dict(dtype=torch.int32, device="cuda")
        tokens, length = torch.empty(rows, self.room, **i32), torch.empty(rows, **i32)
        ssmv.ssmv_logit_rules(logits=logits, out=logits, rows=rows, vocab=model.w["vocab"], io=model.io, hist=self.tokens, hist_len=self.length, src_row=parent, token=token,
                              repetition=torch.full((rows,), self.penalty, device="cuda"), hist_out=tokens, hist_len_out=length)
        self.tokens, self.length = tokens, length


def beam_search(model, prompts, lengths, beams, steps, eos, repetition=None):
    """The `beams` best continuations of every prompt: (tokens [sequences][beams][steps], scores [sequences][beams]), best first.
    prompts [sequences][n] int32 and lengths [sequences] int32 on the GPU.  repetition: a penalty on tokens that occur already, or None."""
    b, vocab = prompts.shape[0], model.w["vocab"]
    i32 = dict(dtype=torch.int32, device="cuda")
    model.reset()
    logits = model.forward(prompts, seq_len=lengths)
    scores, done, rows_in, history = torch.zeros(b, device="cuda"), None, 1, []
    said = None if repetition is None else Histories(prompts, lengths, steps, repetition)
    for _ in range(steps):
        if said is not None:
            said.apply(model, logits, *(history[-1] if history else (None, None)))
        n = b * beams
        parent, token, best, ended = torch.empty(n, **i32), torch.empty(n, **i32), torch.empty(n, device="cuda"), torch.empty(n, **i32)
        work = torch.empty(ssmv.ssmv_beam_workspace(b, rows_in, beams, vocab), dtype=torch.uint8, device="cuda")
        ssmv.ssmv_beam_select(logits=logits, scores=scores, parent=parent, token=token, scores_out=best, batch=b, beams_in=rows_in, beams_out=beams,
                              vocab=vocab, io=model.io, done=done, done_out=ended, eos=eos, workspace=work)
        history.append((parent, token))
        scores, done, rows_in = best, ended, beams
        if len(history) < steps:
            logits = model.forward(token[:, None], src_row=parent)
    # the tokens of the beams that are left, from the last choice back to the first
    row, out = torch.arange(b * beams, device="cuda"), []
    for parent, token in reversed(history):
        out.append(token[row])
        row = parent[row].long()
    return torch.stack(out[::-1], dim=1).view(b, beams, steps), scores.view(b, beams)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("layers", 4), ("width", 1024), ("vocab", 32000), ("sequences", 2), ("beams", 4), ("prompt", 256), ("tokens", 32), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--dtype", choices=sorted(IO), default="bf16")
    ap.add_argument("--repetition", type=float, default=None)
    a = ap.parse_args()
    model = Model(make_weights(a.layers, a.width, 2 * a.width, 16, max(8, a.width // 16 // 8 * 8), a.vocab, a.dtype, a.seed))
    g = torch.Generator().manual_seed(a.seed + 1)
    prompts = torch.randint(3, a.vocab, (a.sequences, a.prompt), generator=g, dtype=torch.int32).cuda()
    lengths = torch.randint(max(1, a.prompt // 2), a.prompt + 1, (a.sequences,), generator=g, dtype=torch.int32).cuda()
    beam_search(model, prompts, lengths, a.beams, 2, eos=2, repetition=a.repetition)
    torch.cuda.synchronize()
    began = time.perf_counter()
    tokens, scores = beam_search(model, prompts, lengths, a.beams, a.tokens, eos=2, repetition=a.repetition)
    torch.cuda.synchronize()
    took = time.perf_counter() - began
    for s in range(a.sequences):
        print("prompt %d (%d tokens): best of %d beams, log-probability %.3f: %s" % (s, int(lengths[s]), a.beams, float(scores[s, 0]), tokens[s, 0].tolist()))
    print("%d layers, %d sequences x %d beams: prompt and %d tokens in %.1f ms" % (a.layers, a.sequences, a.beams, a.tokens, took * 1e3))


if __name__ == "__main__":
    main()
