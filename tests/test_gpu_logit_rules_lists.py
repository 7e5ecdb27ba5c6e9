"""ssmv_logit_rules with lists of biases in which tokens are listed again and again: the sums, bit by bit, and what they cost."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _layers import gen

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,pick,n", [(1, "all", 4095), (4100, "pairs", 4095), (64, "random", 4095), (64, "random", 63), (9000, "random", 1000), (9000, "random", 65), (300, "one", 300), (5000, "outside", 700),
                                      (128011, "first", 257)])
@pytest.mark.parametrize("history", [False, True])
def test_sums_in_the_order_of_the_list(V, pick, n, history):
    """fp32 sums from a token's first place on, one rounding after the other, added to the logit: values of every size, so that another order shows."""
    g, rows = gen(V + n), 3
    token = dict(all=torch.zeros(rows, n), pairs=torch.arange(n).repeat(rows, 1) // 2 * 2, random=torch.randint(0, V, (rows, n), generator=g), one=torch.arange(n).repeat(rows, 1),
                 outside=torch.randint(-50, V + 50, (rows, n), generator=g), first=torch.arange(n).repeat(rows, 1) * 400)[pick].int()
    if pick == "one":
        token[0, -1], token[1, 1], token[2, 150] = 0, 0, 149
    if pick == "first":                                             # a list filled up with the first token, and one that has it once
        token[:, 100:], token[2, 100:] = 0, -1
    bias = torch.randn(rows, n, generator=g) * 2.0 ** torch.randint(-20, 20, (rows, n), generator=g)
    logits = torch.randn(rows, V, generator=g)
    want, order = logits.clone(), [dict() for _ in range(rows)]
    for b in range(rows):
        for v, w in zip(token[b].tolist(), bias[b]):
            if 0 <= v < V:
                order[b][v] = order[b][v] + w if v in order[b] else w.clone()
        for v, w in order[b].items():
            want[b, v] += w
    kw = {}
    if history:                                                     # counts next to the places of the list; penalties that change nothing
        kw = dict(hist=torch.randint(0, V, (rows, 500), generator=g, dtype=torch.int32).cuda(), hist_len=torch.full((rows,), 500, dtype=torch.int32, device="cuda"),
                  repetition=torch.ones(rows, device="cuda"), frequency=torch.zeros(rows, device="cuda"))
    for in_place in (False, True):
        d = logits.cuda()
        out = d if in_place else torch.empty_like(d)
        ssmv.ssmv_logit_rules(logits=d, out=out, rows=rows, vocab=V, io="f32", bias_token=token.cuda(), bias=bias.cuda(), **kw)
        assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("again", ["one", "filled"])
@pytest.mark.parametrize("n,times", [(100, 10), (4095, 60)])
def test_a_token_listed_again_costs_little(n, times, again):
    """One token twice, or half of the list filled up with one.  A place that is listed again takes its wave some 130 cycles, one after the other: 50 of them 3 us and 2048 of them 110 us, behind calls of 5 and
    7 us, which is twice and 16 times as long; so often again is left for a busy machine.  Where every listed token looks for itself in the rest of the list it is 13 and 480 times."""
    rows, V = 64, 8192
    logits = torch.randn(rows, V, device="cuda")
    out, bias, once = torch.empty_like(logits), torch.randn(rows, n, device="cuda"), torch.arange(n, dtype=torch.int32).repeat(rows, 1)
    twice = once.clone()
    twice[:, (n // 2 if again == "filled" else n - 1):] = 0

    def took(token):
        token, best = token.cuda(), float("inf")
        for _ in range(4):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(5):
                ssmv.ssmv_logit_rules(logits=logits, out=out, rows=rows, vocab=V, io="f32", bias_token=token, bias=bias)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    assert took(twice) < times * took(once)
