"""ssmv_logit_rules on the GPU against the rules in 64 bits, row by row."""
import math

import pytest
import torch

import paper_2408_15237_amd as ssmv
from _layers import IO, check_rules, cuda, gen, randn, rules_reference, strided

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def _mask(g, rows, V, share):
    bits = torch.rand(rows, (V + 31) // 32, 32, generator=g) < share
    words = (bits.long() << torch.arange(32)).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).int()


def _ints(g, hi, *s, lo=0):
    return torch.randint(lo, hi, s, generator=g, dtype=torch.int32)


def _run(rows, V, io, seed=0, room=40, rows_in=None, hist=True, token=True, prompt=True, rep=True, freq=True, pres=True, bias_n=5, grammar=4, share=0.5, src=None, lens=None,
         wide=None, in_place=False, keep=True, hist_in_place=False, edit=None):
    g = gen(seed)
    t = dict(logits=(3 * randn(g, rows, V)).to(IO[io]))
    if hist:
        n = rows_in or rows
        t["hist"] = (V * torch.rand(n, room, generator=g) ** 2).int()
        t["hist_len"] = _ints(g, room, n) if lens is None else torch.tensor(lens, dtype=torch.int32)
        t["src"] = None if src is None else torch.tensor(src, dtype=torch.int32)
        t["token"] = _ints(g, V, rows) if token else None
        t["prompt"] = _ints(g, room, rows) if prompt else None
        t["rep"] = 1 + torch.rand(rows, generator=g) if rep else None
        t["freq"], t["pres"] = torch.rand(rows, generator=g) if freq else None, torch.rand(rows, generator=g) if pres else None
    if bias_n:
        t["bias_token"], t["bias"] = _ints(g, V, rows, bias_n), randn(g, rows, bias_n)
    if grammar:
        t["mask"], t["mask_row"] = _mask(g, grammar, V, share), _ints(g, grammar + 1, rows, lo=-1)
    if edit:
        edit(t)
    t = {k: v for k, v in t.items() if v is not None}
    want, err, said = rules_reference(**t)
    d = {k: cuda(strided(v, *wide) if wide and k == "logits" else v) for k, v in t.items()}
    out = d["logits"] if in_place else strided(torch.full((rows, V), 7.0, dtype=IO[io], device="cuda"), *(wide or (0, 0)), fill=5.0)
    o, args = d.get, {}
    if hist and keep:
        args = dict(hist_out=d["hist"] if hist_in_place else torch.full((rows, room), -9, dtype=torch.int32, device="cuda"),
                    hist_len_out=torch.full((rows,), -9, dtype=torch.int32, device="cuda"))
    ssmv.ssmv_logit_rules(logits=d["logits"], out=out, rows=rows, vocab=V, io=io, row_stride=d["logits"].stride(0), out_stride=out.stride(0), hist=o("hist"),
                          hist_len=o("hist_len"), src_row=o("src"), token=o("token"), prompt_len=o("prompt"), repetition=o("rep"), frequency=o("freq"), presence=o("pres"),
                          bias_token=o("bias_token"), bias=o("bias"), mask=o("mask"), mask_row=o("mask_row"), **args)
    torch.cuda.synchronize()
    check_rules(out, want, err, io, "logits")
    if args:
        left = t["hist"] if hist_in_place else torch.full((rows, room), -9, dtype=torch.int32)
        for b in range(rows):
            n = min(len(said[b]), room)
            assert args["hist_out"][b, :n].tolist() == said[b][:n]
            assert int(args["hist_len_out"][b]) == n
            assert torch.equal(args["hist_out"][b, n:].cpu(), left[b, n:])
    if wide:
        parent = out._base.cpu()
        edge = torch.cat([parent[:, :wide[0]], parent[:, wide[0] + V:]], 1)
        assert bool((torch.isnan(edge) if in_place else edge == 5.0).all())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 33, 100, 2047, 2049, 4100])
def test_vocabularies(io, V):
    _run(3, V, io, seed=V)
    _run(3, V, io, seed=V, in_place=True)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_large_vocabulary_and_large_pieces(io):
    _run(2, 50021, io, seed=1, room=3000, bias_n=600)
    _run(90, 50021, io, seed=2, room=20)
    _run(90, 50021, io, seed=3, room=20, in_place=True, share=0.001)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("parts", [dict(hist=False), dict(bias_n=0), dict(grammar=0), dict(hist=False, bias_n=0), dict(hist=False, grammar=0), dict(bias_n=0, grammar=0),
                                   dict(hist=False, bias_n=0, grammar=0), dict(rep=False), dict(freq=False), dict(pres=False, freq=False), dict(prompt=False), dict(token=False),
                                   dict(keep=False), dict(token=False, keep=False, rep=False)])
def test_parts(io, parts):
    for in_place in (False, True):
        _run(4, 300, io, seed=5, in_place=in_place, **parts)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("wide", [(0, 8), (3, 2), (1, 0)])
def test_strides(io, wide):
    for in_place in (False, True):
        _run(4, 333, io, wide=wide, in_place=in_place)


def test_histories_of_parents():
    _run(6, 200, "f32", src=[2, 2, 0, -1, 3, 77], rows_in=4)
    _run(6, 200, "bf16", src=[2, 2, 0, -1, 3, 77], rows_in=4, token=False)


def test_history_lengths():
    """Empty, longer than their room (all of it counts, a new token is counted and not kept), negative; in place."""
    for room in (1, 40):
        _run(5, 100, "f32", room=room, lens=[0, 1, room, room + 9, -3])
        _run(5, 100, "f32", room=room, lens=[0, 1, room, room + 9, -3], hist_in_place=True)
        _run(5, 100, "f32", room=room, lens=[0, 1, room, room + 9, -3], token=False, hist_in_place=True)


def test_tokens_that_are_none_and_tokens_said_often():
    def edit(t):
        t["hist"][0, :] = 7
        t["hist"][1, ::2] = -1
        t["hist"][2, ::2] = 100
        t["hist"][3, 0], t["hist"][3, 1] = 2 ** 31 - 1, -2 ** 31
        t["token"][1], t["token"][2] = -5, 2 ** 30
        t["bias_token"][0, :3] = torch.tensor([-1, 100, 2 ** 31 - 1])
    _run(4, 100, "f32", lens=[40, 40, 40, 40], edit=edit)


def test_a_token_that_is_often_in_the_list():
    """Its values are added in the order of the list: large ones that take each other away show another order (2^24 + 1 is no fp32 number)."""
    def edit(t):
        t["bias_token"][:] = 5
        t["bias_token"][1, 2] = 6
        t["bias"][:] = 0.25
    _run(3, 64, "f32", bias_n=4000, edit=edit, grammar=0)
    n = 3
    logits, out = torch.zeros(1, n, device="cuda"), torch.zeros(1, n, device="cuda")
    ssmv.ssmv_logit_rules(logits=logits, out=out, rows=1, vocab=n, io="f32", bias_token=torch.tensor([[1, 1, 1, 2]], dtype=torch.int32, device="cuda"),
                          bias=torch.tensor([[2.0 ** 24, 1.0, -2.0 ** 24, 3.0]], device="cuda"))
    assert out.tolist() == [[0.0, 0.0, 3.0]]


def test_infinities_and_numbers_that_are_none():
    def edit(t):
        t["logits"][0, :4] = torch.tensor([INF, -INF, NAN, 0.0])
        t["hist"][0, :4] = torch.arange(4, dtype=torch.int32)
        t["bias"][1, 0], t["bias"][1, 1] = -INF, INF
        t["bias_token"][1, :2] = torch.tensor([3, 4], dtype=torch.int32)
        t["logits"][2, :] = -1e30 if t["logits"].dtype == torch.float32 else -1e30
        t["mask_row"][:] = torch.tensor([-1, 9, 1, 2], dtype=torch.int32)
        t["mask"][1] = 0
        t["logits"][3, :8] = NAN
        t["mask"][2] = 0x55555555
    for io in ("bf16", "f32"):
        for in_place in (False, True):
            _run(4, 77, io, lens=[4, 4, 4, 4], edit=edit, in_place=in_place)


def test_rows_without_a_mask_row_index():
    g = gen(1)
    logits, mask = randn(g, 3, 70), _mask(g, 3, 70, 0.5)
    want, err, _ = rules_reference(logits, mask=mask)
    out = torch.empty(3, 70, device="cuda")
    wide = torch.full((3, 5), -1, dtype=torch.int32)
    wide[:, :3] = mask
    ssmv.ssmv_logit_rules(logits=logits.cuda(), out=out, rows=3, vocab=70, io="f32", mask=wide.cuda(), mask_stride=5)
    check_rules(out, want, err, "f32", "logits")


def test_in_place_leaves_what_nothing_changes():
    """Logits that no rule names keep their bits: a NaN's payload, a bf16 that no rounding would give back."""
    logits = torch.full((2, 5000), 0x7FC5, dtype=torch.int16).view(torch.bfloat16).cuda()
    ssmv.ssmv_logit_rules(logits=logits, out=logits, rows=2, vocab=5000, io="bf16", bias_token=torch.tensor([[17], [4999]], dtype=torch.int32, device="cuda"),
                          bias=torch.ones(2, 1, device="cuda"))
    keep = torch.ones(2, 5000, dtype=torch.bool)
    keep[0, 16:24], keep[1, 4992:] = False, False                   # vectors of eight that a rule touches
    assert bool((logits.view(torch.int16).cpu()[keep] == 0x7FC5).all())


def test_captured_and_on_another_stream():
    rows, V, room = 5, 3000, 50
    g = gen(2)
    d = dict(logits=randn(g, rows, V).cuda(), out=torch.zeros(rows, V, device="cuda"), hist=_ints(g, V, rows, room).cuda(), hist_len=_ints(g, room, rows).cuda(),
             src_row=_ints(g, rows, rows).cuda(), token=_ints(g, V, rows).cuda(), repetition=1 + torch.rand(rows, generator=g).cuda(), hist_out=torch.zeros(rows, room, dtype=torch.int32, device="cuda"),
             hist_len_out=torch.zeros(rows, dtype=torch.int32, device="cuda"), bias_token=_ints(g, V, rows, 9).cuda(), bias=randn(g, rows, 9).cuda(),
             mask=_mask(g, 3, V, 0.7).cuda(), mask_row=_ints(g, 3, rows).cuda())
    names = ("out", "hist_out", "hist_len_out")
    call = lambda: ssmv.ssmv_logit_rules(**d, rows=rows, vocab=V, io="f32")
    call()
    torch.cuda.synchronize()
    eager = {k: d[k].clone() for k in names}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert all(torch.equal(d[k], eager[k]) for k in names)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(3):
        d["logits"].mul_(-1.5)
        d["token"].copy_((d["token"] * 7 + turn) % V)
        for k in names:
            d[k].zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: d[k].clone() for k in names}
        for k in names:
            d[k].zero_()
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(d[k], got[k]) for k in names), turn


def test_a_search_keeps_its_histories():
    """Ten choices of ssmv_beam_select, each behind the rules: the histories are what following the parents back gives, and no beam says a token twice where the penalty forbids it."""
    g = gen(4)
    b, W, V, steps = 2, 3, 40, 10
    rows = b * W
    i32 = dict(dtype=torch.int32, device="cuda")
    hist, hist_len = torch.zeros(rows, steps, **i32), torch.zeros(rows, **i32)
    scores = torch.tensor([0.0, -INF, -INF] * b, device="cuda")
    parent = token = None
    trail, freq = [], torch.full((rows,), 1000.0, device="cuda")
    work = torch.empty(ssmv.ssmv_beam_workspace(b, W, W, V), dtype=torch.uint8, device="cuda")
    for step in range(steps):
        logits = randn(g, rows, V).cuda()
        hist2, len2 = torch.zeros(rows, steps, **i32), torch.zeros(rows, **i32)
        ssmv.ssmv_logit_rules(logits=logits, out=logits, rows=rows, vocab=V, io="f32", hist=hist, hist_len=hist_len, src_row=parent, token=token, frequency=freq, hist_out=hist2,
                              hist_len_out=len2)
        hist, hist_len = hist2, len2
        best = torch.empty(rows, device="cuda")
        parent, token = torch.empty(rows, **i32), torch.empty(rows, **i32)
        ssmv.ssmv_beam_select(logits=logits, scores=scores, parent=parent, token=token, scores_out=best, batch=b, beams_in=W, beams_out=W, vocab=V, io="f32", workspace=work)
        trail.append((parent.cpu(), token.cpu()))
        scores = best
    for r in range(rows):
        row, said = r, []
        for p, t in reversed(trail):
            said.insert(0, int(t[row]))
            row = int(p[row])
        assert len(set(said)) == steps, said
        row = int(trail[-1][0][r])
        assert hist[row, :steps - 1].tolist() == said[:-1] and int(hist_len[row]) == steps - 1
