"""The layer operators on tensors of more than 2^31 elements (more than 2^32 bytes): what lies at their far ends against the formulas in 64 bits."""
import pytest
import torch

import paper_2408_15237_amd as ssmv
from _layers import EPS, Num, check, check_rules, gated_backward, gated_forward, norm_backward, norm_forward, rules_reference

pytestmark = pytest.mark.gpu
BF = dict(dtype=torch.bfloat16, device="cuda")


@pytest.fixture(autouse=True)
def _memory():
    torch.cuda.empty_cache()
    torch.manual_seed(5)
    yield
    torch.cuda.empty_cache()


def test_norm_rows():
    rows, C = 270001, 8192
    x, res, dn = torch.randn(rows, C, **BF), torch.randn(rows, C, **BF), torch.randn(rows, C, **BF)
    post, pre = 1 + torch.randn(C, device="cuda") / 8, 1 + torch.randn(C, device="cuda") / 8
    r, n, dx, dres = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    ssmv.ssmv_block_norm(x=x, res=res, post_wgt=post, pre_wgt=pre, r_out=r, n_out=n, rows=rows, channels=C, io="bf16", eps=EPS)
    ssmv.ssmv_block_norm_backward(x=x, res=res, post_wgt=post, pre_wgt=pre, dn=dn, dx=dx, dres=dres, rows=rows, channels=C, io="bf16", eps=EPS)
    for at in (slice(0, 2), slice(262143, 262146), slice(rows - 2, rows)):
        part = [t[at].cpu() for t in (x, res, dn)]
        _, _, _, wr, _, wn = norm_forward(part[0], None, part[1], post.cpu(), None, pre.cpu(), 1.0)
        check(r[at], wr, "bf16", "r")
        check(n[at], wn, "bf16", "n")
        want = norm_backward(part[0], None, part[1], post.cpu(), None, pre.cpu(), 1.0, None, part[2])
        check(dx[at], want["dx"], "bf16", "dx")
        check(dres[at], want["dres"], "bf16", "dres")


def _mix(x, f, dy, h=None):
    b, n, C = x.shape
    y, states, dx, df = torch.empty_like(x), torch.empty(b, (n + 63) // 64, C, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    out = torch.empty(b, C, device="cuda")
    work = [torch.empty(max(16, size(b, C, n)), dtype=torch.uint8, device="cuda") for size in (ssmv.ssm_gated_recurrence_workspace, ssmv.ssm_gated_recurrence_backward_workspace)]
    ssmv.ssm_gated_recurrence(x=x, f=f, y_out=y, states=states, h_out=out, batch=b, channels=C, L=n, io="bf16", form="mix", workspace=work[0])
    ssmv.ssm_gated_recurrence_backward(x=x, f=f, dy=dy, states=states, dx=dx, df=df, batch=b, channels=C, L=n, io="bf16", form="mix", workspace=work[1])
    return y, out, dx, df


def test_recurrence_over_many_sequences():
    b, n, C = 131, 2051, 8200
    x, f, dy = (torch.randn(b, n, C, **BF) for _ in range(3))
    y, out, dx, df = _mix(x, f, dy)
    for i, c in ((0, 0), (b - 1, C - 6)):                          # a channel does not depend on others
        px, pf, pd = (t[i:i + 1, :, c:c + 6].cpu() for t in (x, f, dy))
        wy, _, wh, _ = gated_forward(px, pf)
        check(y[i:i + 1, :, c:c + 6], wy, "bf16", "y")
        check(out[i:i + 1, c:c + 6], wh, "f32", "h")
        want = gated_backward(px, pf, pd)
        check(dx[i:i + 1, :, c:c + 6], want["dx"], "bf16", "dx")
        check(df[i:i + 1, :, c:c + 6], want["df"], "bf16", "df")


def test_recurrence_over_a_long_sequence():
    """Decays are sigmoids of N(0,1): 600 tokens leave less than 1e-100 of a state, so that windows at the ends stand for the whole."""
    n, C, w = 2200003, 1000, 700
    x, f, dy = (torch.randn(1, n, C, **BF) for _ in range(3))
    y, out, dx, df = _mix(x, f, dy)
    cut = lambda q, at: Num(q.v[:, at], q.e[:, at])
    for at, keep in ((slice(0, w), slice(0, 50)), (slice(n - w, n), slice(w - 50, w))):
        px, pf, pd = (t[:, at, -9:].cpu() for t in (x, f, dy))
        wy, _, wh, _ = gated_forward(px, pf)
        want = gated_backward(px, pf, pd)
        check(y[:, at, -9:][:, keep], cut(wy, keep), "bf16", "y")
        check(dx[:, at, -9:][:, keep], cut(want["dx"], keep), "bf16", "dx")
        check(df[:, at, -9:][:, keep], cut(want["df"], keep), "bf16", "df")
    check(out[:, -9:], wh, "f32", "h")


@pytest.mark.parametrize("in_place", [False, True])
def test_rules_rows(in_place):
    rows, V, room = 17001, 128011, 40
    logits = torch.randn(rows, V, **BF)
    hist = torch.randint(0, V, (rows, room), dtype=torch.int32, device="cuda")
    hist_len = torch.randint(0, room, (rows,), dtype=torch.int32, device="cuda")
    mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (3, (V + 31) // 32), dtype=torch.int32, device="cuda")
    mask_row = torch.randint(-1, 3, (rows,), dtype=torch.int32, device="cuda")
    rep, freq = 1 + torch.rand(rows, device="cuda"), torch.rand(rows, device="cuda")
    far = [0, 16776, 16777, 16778, rows - 1]                        # around 2^31 elements, and the last one
    was = logits[far].cpu()
    out = logits if in_place else torch.empty_like(logits)
    ssmv.ssmv_logit_rules(logits=logits, out=out, rows=rows, vocab=V, io="bf16", hist=hist, hist_len=hist_len, repetition=rep, frequency=freq, mask=mask, mask_row=mask_row)
    want, err, _ = rules_reference(was, hist[far].cpu(), hist_len[far].cpu(), rep=rep[far].cpu(), freq=freq[far].cpu(), mask=mask.cpu(), mask_row=mask_row[far].cpu())
    check_rules(out[far], want, err, "bf16", "logits")
