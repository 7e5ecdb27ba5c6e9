"""ssmv_beam_select on the GPU against all candidates sorted in 64 bits."""
import math

import pytest
import torch

import paper_2408_15237_amd as ssmv
from _decode import IO, beam_reference, cuda, gen, strided

pytestmark = pytest.mark.gpu

# a row's sum in 32 bits: exponents rounded (log2 e times up to 100 apart, weighted by the terms themselves: under 4 * 2^-24 of the sum where
# the terms count), exp2 2^-23, adding under 32 + 14 terms 2^-24 each
LSE = 52 * 2.0 ** -24


def _select(logits, scores, batch, beams_out, io, done=None, eos=-1):
    rows, V = logits.shape
    W = rows // batch
    n = batch * beams_out
    parent, token = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    out, done_out = torch.full((n,), 7.0, device="cuda"), torch.full((n,), -7, dtype=torch.int32, device="cuda")
    ws = torch.full((ssmv.ssmv_beam_workspace(batch, W, beams_out, V),), 0xFF, dtype=torch.uint8, device="cuda")
    d = cuda(logits)
    ssmv.ssmv_beam_select(logits=d, scores=cuda(scores), parent=parent, token=token, scores_out=out, batch=batch, beams_in=W, beams_out=beams_out, vocab=V, io=io,
                          row_stride=d.stride(0) if rows > 1 else 0, done=cuda(done), done_out=done_out, eos=eos, workspace=ws)
    torch.cuda.synchronize()
    return [t.cpu().view(batch, beams_out) for t in (parent, token, out, done_out)]


def _check(logits, scores, batch, beams_out, io, done=None, eos=-1):
    parent, token, out, done_out = _select(logits, scores, batch, beams_out, io, done, eos)
    ref = beam_reference(logits, scores, beams_out, batch, done, eos)
    for s in range(batch):
        cand = ref[s]
        where = {}
        for c in cand:
            where.setdefault((c[1], c[2]), []).append(c[0])
        for i in range(beams_out):
            want = cand[i]
            tol = LSE + 2.0 ** -24 * abs(want[0]) if math.isfinite(want[0]) else 0.0
            got = (int(parent[s, i]), int(token[s, i]))
            score = float(out[s, i])
            assert score == want[0] or abs(score - want[0]) <= tol, (s, i, score, want)
            # another candidate may stand here only if the reference has it as near as a rounding of the rows' sums
            if got != want[1:]:
                assert got in where, (s, i, got, want)
                assert got[0] != want[1] and any(abs(v - want[0]) <= 2 * LSE for v in where[got]), (s, i, got, want, where[got])
            assert int(done_out[s, i]) == int((done is not None and bool(done[got[0]])) or got[1] == eos)
        pairs = [(int(parent[s, i]), int(token[s, i])) for i in range(beams_out) if math.isfinite(float(out[s, i]))]
        assert len(set(pairs)) == len(pairs)


def _inputs(batch, W, V, io, seed, masked=0.0):
    g = gen(seed)
    logits = (3 * torch.randn(batch * W, V, generator=g)).to(IO[io])
    if masked:
        logits[torch.rand(logits.shape, generator=g) < masked] = -math.inf
    return logits, -(20 + 2 * torch.randn(batch * W, generator=g).abs())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 255, 256, 257, 2048, 2049, 8191, 8192, 8193, 32000, 100003])
def test_vocabularies(io, V):
    for W, K in ((1, min(4, V)), (4, 4)):
        logits, scores = _inputs(2, W, V, io, V)
        _check(logits, scores, 2, min(K, W * V), io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("W,K", [(1, 1), (1, 64), (3, 6), (5, 2), (8, 16), (64, 64), (17, 33)])
def test_beam_counts(io, W, K):
    logits, scores = _inputs(3, W, 9001, io, W * 100 + K)
    _check(logits, scores, 3, K, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_masked_tokens_and_rows(io):
    logits, scores = _inputs(3, 4, 20000, io, 1, masked=0.9)
    logits[5] = -math.inf                                         # a row that allows nothing
    logits[8:12] = -math.inf                                      # a sequence that allows nothing
    logits[9, 777] = 0.0                                          # but for one token
    _check(logits, scores, 3, 4, io)
    scores[1] = -math.inf                                         # a beam that is none
    scores[2] = float("nan")
    logits[0, 17], logits[0, 19000] = math.inf, math.inf
    logits[6, 3] = float("nan")
    logits[7, :] = torch.finfo(IO[io]).min                        # a mask of the type's lowest value, everywhere
    _check(logits, scores, 3, 4, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_ties_go_to_the_lower_row_then_token(io):
    V, W, K = 10007, 4, 10
    logits = torch.zeros(2 * W, V, dtype=IO[io])
    scores = torch.full((2 * W,), -3.0)
    parent, token, _, _ = _select(logits, scores, 2, K, io)
    for s in range(2):
        assert parent[s].tolist() == [s * W] * K and token[s].tolist() == list(range(K))
    one = (torch.randint(-40, 40, (V,), generator=gen(2)) / 4).to(IO[io])        # every value many times over; rows alike
    logits = one.repeat(2 * W, 1)
    parent, token, _, _ = _select(logits, scores, 2, K, io)
    order = torch.sort(one.float(), descending=True, stable=True).indices
    best = one.float().max()
    for s in range(2):
        want = [(s * W + r, int(v)) for r in range(W) for v in order[:K] if float(one[v]) == float(best)][:K]
        assert list(zip(parent[s].tolist(), token[s].tolist()))[:len(want)] == want
    z = torch.zeros(1, V, dtype=IO[io])
    z[0, ::2] = -0.0                                              # minus zero is zero
    _, token, _, _ = _select(z, torch.zeros(1), 1, 6, io)
    assert token[0].tolist() == list(range(6))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_finished_beams(io):
    logits, scores = _inputs(4, 4, 5000, io, 8)
    done = torch.tensor([0, 1, 0, 0, 1, 1, 1, 1, 0, 0, 0, 0, 0, 0, 5, -1], dtype=torch.int32)
    scores[1] = -1.0                                              # a finished beam that stays the best
    logits[1], logits[4] = float("nan"), math.inf                 # its logits are not read
    logits[9, 42] = 60.0                                          # and one that finishes now
    _check(logits, scores, 4, 4, io, done, eos=42)
    _check(logits, scores, 4, 8, io, done, eos=0)
    _check(logits[4:5], scores[4:5], 1, 3, io, done[4:5], eos=7)  # nothing but a finished beam


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("wide", [(0, 8), (8, 8), (3, 2), (1, 0)])
def test_strides(io, wide):
    logits, scores = _inputs(2, 3, 8205, io, 5)
    _check(strided(logits, *wide), scores, 2, 5, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_sorted_logits(io):
    """All of the best in the elements of one thread, or spread over all of them."""
    for V in (4096, 33000):
        up = torch.linspace(-60, 60, V).to(IO[io]).repeat(2, 1)
        _check(up, torch.tensor([-1.0, -1.25]), 1, 64, io)
        _check(up.flip(1).contiguous(), torch.tensor([-1.0, -1.25]), 1, 64, io)


def test_the_same_call_gives_the_same_bits_also_in_a_graph():
    batch, W, K, V = 3, 4, 4, 30011
    logits, scores = _inputs(batch, W, V, "bf16", 77)
    first = _select(logits, scores, batch, K, "bf16")
    for a, b in zip(first, _select(logits, scores, batch, K, "bf16")):
        assert torch.equal(a, b)
    d, sc = logits.cuda(), scores.cuda()
    parent, token = (torch.zeros(batch * K, dtype=torch.int32, device="cuda") for _ in range(2))
    out = torch.zeros(batch * K, device="cuda")
    ws = torch.zeros(ssmv.ssmv_beam_workspace(batch, W, K, V), dtype=torch.uint8, device="cuda")
    kw = dict(logits=d, scores=sc, parent=parent, token=token, scores_out=out, batch=batch, beams_in=W, beams_out=K, vocab=V, io="bf16", workspace=ws)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        ssmv.ssmv_beam_select(**kw)
        graph.capture_end()
    for _ in range(3):
        parent.zero_(), token.zero_(), out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(parent.cpu().view(batch, K), first[0]) and torch.equal(token.cpu().view(batch, K), first[1]) and torch.equal(out.cpu().view(batch, K), first[2])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3, 10, 63, 500, 1318, 2040, 6313, 8571])
@pytest.mark.parametrize("W,K", [(16, 9), (32, 64), (9, 33), (1, 9), (2, 3)])
def test_ends_of_rows_and_many_candidates(io, V, W, K):
    """Vocabularies that leave most lanes without logits; fewer tokens than beams; hundreds of candidates of a sequence, equal ones among them."""
    K = min(K, W * V)
    logits, scores = _inputs(3, W, V, io, V + W, masked=0.1)
    logits[W:2 * W] = logits[W]                                   # a sequence of equal rows,
    scores[W:2 * W] = scores[W]                                   # all of whose candidates tie
    scores[2 * W + W // 2] = -math.inf
    logits[2 * W, V // 2:] = -math.inf
    _check(logits, scores, 3, K, io)
    done = torch.zeros(3 * W, dtype=torch.int32)
    done[::3] = 1
    _check(logits, scores, 3, K, io, done, eos=V - 1)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("V", [500, 33001])
@pytest.mark.parametrize("big", [3e4, 3e6, 1e9, 1e10, 1e12, 1e20, 9e29, 2e30, 1e38])
def test_rows_at_a_large_finite_value(io, V, big):
    """A mask that is a large finite number, in a whole row too, and logits as large: the exponentials' common reference must not cost the sum."""
    logits, scores = _inputs(3, 2, V, io, 12)
    logits[0:2] = -big                                            # a sequence that masks everything
    logits[1, V - 3] = -big * 0.5
    logits[2, ::2] = -big                                         # a row half masked beside one that is masked whole
    logits[3] = -big
    logits[4, ::7] = big                                          # and logits that are as large
    logits[5, 1::9] = big
    logits[5, 4] = big * 1.5
    _check(logits, scores, 3, 5, io)
