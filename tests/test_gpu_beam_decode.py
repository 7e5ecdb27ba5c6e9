"""examples/beam_decode.py on the GPU: the beams that it finds against the same search over the same model in 64 bits on the CPU."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import beam_decode  # noqa: E402

pytestmark = pytest.mark.gpu


class Reference:
    """The model in 64 bits; a row's state is a list of (h, three conv inputs) per layer."""

    def __init__(self, w):
        dbl = lambda d: {k: v.double() if torch.is_tensor(v) else v for k, v in d.items() if k != "layers"}
        self.w, self.layers = dbl(w), [dbl(x) for x in w["layers"]]

    def empty(self):
        return [(torch.zeros(self.w["inner"], self.w["dstate"], dtype=torch.float64), torch.zeros(3, self.w["inner"], dtype=torch.float64)) for _ in self.layers]

    @staticmethod
    def norm(x, weight):
        return x * torch.rsqrt((x * x).mean() + beam_decode.EPS) * weight

    def token(self, state, token):
        """Log-probabilities after one more token, and the new state."""
        x, out = self.w["embed"][token], []
        C, N, R = self.w["inner"], self.w["dstate"], self.w["dt_rank"]
        for w, (h, conv) in zip(self.layers, state):
            xz = w["in_proj"] @ self.norm(x, w["norm"])
            raw = torch.cat([conv, xz[None, :C]])
            v = (raw.T * w["conv_w"]).sum(1) + w["conv_b"]
            xc = v * torch.sigmoid(v)
            proj = w["x_proj"] @ xc
            dt = torch.logaddexp(w["dt_proj"] @ proj[:R] + w["dt_bias"], torch.zeros((), dtype=torch.float64))
            h = torch.exp(dt[:, None] * w["A"]) * h + (dt * xc)[:, None] * proj[None, R:R + N]
            z = xz[C:]
            x = x + w["out_proj"] @ ((h @ proj[R + N:] + w["D"] * xc) * z * torch.sigmoid(z))
            out.append((h, raw[1:]))
        return torch.log_softmax(self.w["head"] @ self.norm(x, self.w["norm"]), 0), out


def search(ref, prompt, beams, steps, eos):
    state = ref.empty()
    for t in prompt:
        logp, state = ref.token(state, int(t))
    live = [(0.0, [], state, logp)]
    gaps = []
    for _ in range(steps):
        cand = []
        for r, (score, toks, state, logp) in enumerate(live):
            if toks and toks[-1] == eos:
                cand.append((score, r, eos))
            else:
                cand += [(score + float(logp[v]), r, v) for v in torch.topk(logp, beams + 1).indices.tolist()]
        cand.sort(key=lambda c: -c[0])
        gaps += [a[0] - b[0] for a, b in zip(cand[:beams], cand[1:beams + 1])]
        new = []
        for score, r, v in cand[:beams]:
            _, toks, state, logp = live[r]
            if not (toks and toks[-1] == eos):
                logp, state = ref.token(state, v)
            new.append((score, toks + [v], state, logp))
        live = new
    return live, min(gaps)


@pytest.mark.parametrize("beams", [1, 4])
def test_search_finds_the_same_beams(beams):
    w = beam_decode.make_weights(layers=2, width=64, inner=96, dstate=16, dt_rank=6, vocab=200, io="f32", seed=3)
    w["head"][2] *= 1.5                                           # an end token that wins now and then
    g = torch.Generator().manual_seed(5)
    lengths = torch.tensor([11, 1, 40], dtype=torch.int32)
    prompts = torch.randint(3, 200, (3, 40), generator=g, dtype=torch.int32)
    tokens, scores = beam_decode.beam_search(beam_decode.Model(w), prompts.cuda(), lengths.cuda(), beams, 9, eos=2)
    ref, ended = Reference(w), 0
    for s in range(3):
        want, gap = search(ref, prompts[s, :lengths[s]].tolist(), beams, 9, 2)
        assert gap > 1e-3, "two candidates too near for a comparison in 32 bits"
        assert tokens[s].tolist() == [x[1] for x in want]
        assert torch.allclose(scores[s].cpu().double(), torch.tensor([x[0] for x in want], dtype=torch.float64), rtol=0, atol=2e-4)
        ended += sum(2 in x[1] for x in want)
    if beams > 1:
        assert ended > 0


def test_bf16_runs():
    model = beam_decode.Model(beam_decode.make_weights(io="bf16"))
    prompts = torch.randint(3, 512, (2, 70), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    tokens, scores = beam_decode.beam_search(model, prompts, torch.tensor([70, 33], dtype=torch.int32, device="cuda"), 3, 6, eos=2)
    assert tokens.shape == (2, 3, 6) and bool(torch.isfinite(scores).all()) and bool((scores[:, :-1] >= scores[:, 1:]).all())
    assert int(tokens.min()) >= 0 and int(tokens.max()) < 512


@pytest.mark.parametrize("n", [1, 40])
def test_a_second_search_starts_from_nothing(n):
    """One model, two searches: the second one's prompts do not go on from the first one's states."""
    w = beam_decode.make_weights(layers=2, width=64, inner=96, dstate=16, dt_rank=6, vocab=200, io="f32", seed=3)
    g = torch.Generator().manual_seed(6)
    first, second = (torch.randint(3, 200, (3, m), generator=g, dtype=torch.int32).cuda() for m in (40, n))
    lengths = torch.tensor([n, 1, (n + 1) // 2], dtype=torch.int32).cuda()
    used = beam_decode.Model(w)
    beam_decode.beam_search(used, first, torch.tensor([40, 3, 12], dtype=torch.int32).cuda(), 4, 5, eos=2)
    again = beam_decode.beam_search(used, second, lengths, 4, 5, eos=2)
    fresh = beam_decode.beam_search(beam_decode.Model(w), second, lengths, 4, 5, eos=2)
    assert torch.equal(again[0], fresh[0])
    assert torch.allclose(again[1], fresh[1], rtol=0, atol=2e-4)


def test_bf16_scores_are_those_of_the_tokens():
    """The scores of a bf16 search are what the model in 64 bits gives the tokens that it found.  Some ten roundings to bf16 a layer, 2^-9 each in the mean, make
    about 1 % of a hidden state, 0.04 of a logit (they are about 4) and 0.2 of the farthest; the logits' own rounding 0.06: 0.25 a token."""
    w = beam_decode.make_weights(io="bf16", seed=9)
    lengths, steps = [70, 1, 33], 6
    prompts = torch.randint(3, 512, (3, 70), generator=torch.Generator().manual_seed(4), dtype=torch.int32)
    tokens, scores = beam_decode.beam_search(beam_decode.Model(w), prompts.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), 3, steps, eos=2)
    ref = Reference(w)
    for s in range(3):
        start = ref.empty()
        for t in prompts[s, :lengths[s]].tolist():
            first, start = ref.token(start, t)
        assert len(set(map(tuple, tokens[s].tolist()))) == 3
        for beam in range(3):
            logp, state, total = first, start, 0.0
            for t in tokens[s, beam].tolist():
                total += float(logp[t])
                if t == 2:
                    break
                logp, state = ref.token(state, t)
            assert abs(total - float(scores[s, beam])) <= 0.25 * steps, (s, beam, total, float(scores[s, beam]))
