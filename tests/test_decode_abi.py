"""The state-to-state calls without a GPU: argument structs as the header declares them, workspaces, and refusals on the host before any
HIP call."""
import ctypes
import os
import re

import pytest

import paper_2408_15237_amd as ssmv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x20000              # plausible, aligned, never touched


def _code(fn, *a, **kw):
    with pytest.raises(ssmv.SsmvError) as ei:
        fn(*a, **kw)
    return ei.value.code


@pytest.mark.parametrize("name", ["ssmv_conv_args", "ssmv_scan_args", "ssmv_token_args", "ssmv_beam_args"])
def test_argument_structs_match_the_header(name):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ssmv.h")).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    want = []
    for decl in body.split(";"):
        decl = decl.strip()
        if not decl:
            continue
        if "*" in decl:
            kind, names = ctypes.c_void_p, re.findall(r"\*\s*(\w+)", decl)
        else:
            kind = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32}[decl.split()[0]]
            names = [n.strip() for n in decl.split(None, 1)[1].split(",")]
        want += [(n, kind) for n in names]
    assert list(getattr(ssmv, name)._fields_) == want


def test_beam_limit_matches_the_header():
    m = re.search(r"#define\s+SSMV_BEAMS_MAX\s+(\d+)", open(os.path.join(ROOT, "include", "ssmv.h")).read())
    assert int(m.group(1)) == ssmv.SSMV_BEAMS_MAX


CONV = dict(x=P, wgt=P, out=P + 64, batch=2, channels=16, L=5, io="bf16", stream=0)
SCAN = dict(x=P, dt=P, A=P, Bm=P, Cm=P, D=P, y_out=P + 64, batch=2, channels=16, dstate=16, L=5, io="bf16", workspace=P, stream=0)
STEP = dict(x=P, dt=P, A=P, Bm=P, Cm=P, D=P, y_out=P + 64, h_in=P, h_out=P, rows=2, nheads=4, headdim=8, dstate=16, io="bf16", stream=0)
BEAM = dict(logits=P, scores=P, parent=P + 64, token=P + 64, scores_out=P + 128, batch=2, beams_in=3, beams_out=4, vocab=100, io="bf16", workspace=P, stream=0)


@pytest.mark.parametrize("bad,code", [
    (dict(x=None), ssmv.SSMV_EINVAL), (dict(wgt=None), ssmv.SSMV_EINVAL), (dict(out=None), ssmv.SSMV_EINVAL), (dict(x=P + 1), ssmv.SSMV_EALIGN),
    (dict(bias=P + 1), ssmv.SSMV_EALIGN), (dict(conv_in=P + 1), ssmv.SSMV_EALIGN), (dict(conv_out=P + 1), ssmv.SSMV_EALIGN), (dict(seq_len=P + 2), ssmv.SSMV_EALIGN),
    (dict(src_row=P + 2), ssmv.SSMV_EALIGN), (dict(out=P), ssmv.SSMV_EINVAL), (dict(conv_in=P, conv_out=P, src_row=P), ssmv.SSMV_EINVAL),
    (dict(batch=0), ssmv.SSMV_EINVAL), (dict(channels=0), ssmv.SSMV_EINVAL), (dict(L=0), ssmv.SSMV_EINVAL), (dict(io=7), ssmv.SSMV_EINVAL), (dict(act=7), ssmv.SSMV_EINVAL),
    (dict(x_stride=15), ssmv.SSMV_EINVAL), (dict(out_stride=-16), ssmv.SSMV_EINVAL), (dict(x_stride=1 << 41), ssmv.SSMV_EINVAL), (dict(rows_in=1), ssmv.SSMV_EINVAL),
    (dict(rows_in=-1, src_row=P), ssmv.SSMV_EINVAL), (dict(batch=70000), ssmv.SSMV_EUNSUPPORTED), (dict(L=1 << 30, channels=1 << 20), ssmv.SSMV_EUNSUPPORTED),
    (dict(batch=60000, L=100000, channels=100), ssmv.SSMV_EUNSUPPORTED),
])
def test_conv_refusals(bad, code):
    assert _code(ssmv.ssm_causal_conv, **{**CONV, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict([(k, None)]), ssmv.SSMV_EINVAL) for k in ("x", "dt", "A", "Bm", "Cm", "D", "y_out")] + [
    (dict(x=P + 1), ssmv.SSMV_EALIGN), (dict(A=P + 4), ssmv.SSMV_EALIGN), (dict(Bm=P + 2), ssmv.SSMV_EALIGN), (dict(Cm=P + 2), ssmv.SSMV_EALIGN),
    (dict(h_in=P + 4), ssmv.SSMV_EALIGN), (dict(h_out=P + 8), ssmv.SSMV_EALIGN), (dict(dt_bias=P + 2), ssmv.SSMV_EALIGN), (dict(z=P + 1), ssmv.SSMV_EALIGN),
    (dict(seq_len=P + 2), ssmv.SSMV_EALIGN), (dict(b_stride=17), ssmv.SSMV_EALIGN), (dict(c_stride=19), ssmv.SSMV_EALIGN), (dict(b_stride=8), ssmv.SSMV_EINVAL),
    (dict(y_stride=4), ssmv.SSMV_EINVAL), (dict(dstate=8), ssmv.SSMV_EUNSUPPORTED), (dict(dstate=128), ssmv.SSMV_EUNSUPPORTED), (dict(L=0), ssmv.SSMV_EINVAL),
    (dict(batch=70000), ssmv.SSMV_EUNSUPPORTED), (dict(channels=1 << 25), ssmv.SSMV_EUNSUPPORTED), (dict(dt_softplus=2), ssmv.SSMV_EINVAL), (dict(io=3), ssmv.SSMV_EINVAL),
    (dict(h_in=P, h_out=P, src_row=P), ssmv.SSMV_EINVAL), (dict(rows_in=1, h_in=P), ssmv.SSMV_EINVAL), (dict(batch=60000, L=100000, channels=100), ssmv.SSMV_EUNSUPPORTED),
])
def test_scan_refusals(bad, code):
    assert _code(ssmv.ssm_selective_scan, **{**SCAN, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict([(k, None)]), ssmv.SSMV_EINVAL) for k in ("x", "dt", "A", "Bm", "Cm", "D", "y_out", "h_out")] + [
    (dict(x=P + 1), ssmv.SSMV_EALIGN), (dict(A=P + 2), ssmv.SSMV_EALIGN), (dict(h_out=P + 4), ssmv.SSMV_EALIGN), (dict(h_in=P + 4), ssmv.SSMV_EALIGN),
    (dict(b_stride=17), ssmv.SSMV_EALIGN), (dict(rows=0), ssmv.SSMV_EINVAL), (dict(rows=70000), ssmv.SSMV_EUNSUPPORTED), (dict(ngroups=3), ssmv.SSMV_EINVAL),
    (dict(dstate=17), ssmv.SSMV_EUNSUPPORTED), (dict(a_mode="diag"), ssmv.SSMV_EINVAL), (dict(a_mode=5), ssmv.SSMV_EINVAL),
    (dict(a_mode="diag", headdim=1, dstate=128), ssmv.SSMV_EUNSUPPORTED), (dict(a_mode="diag", headdim=1, A=P + 4), ssmv.SSMV_EALIGN),
    (dict(src_row=P), ssmv.SSMV_EINVAL), (dict(x_stride=31), ssmv.SSMV_EINVAL), (dict(nheads=1 << 20, headdim=128), ssmv.SSMV_EUNSUPPORTED), (dict(dt_softplus=-1), ssmv.SSMV_EINVAL),
])
def test_step_refusals(bad, code):
    assert _code(ssmv.ssm_selective_step, **{**STEP, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict([(k, None)]), ssmv.SSMV_EINVAL) for k in ("logits", "scores", "parent", "token", "scores_out", "workspace")] + [
    (dict(logits=P + 1), ssmv.SSMV_EALIGN), (dict(scores=P + 2), ssmv.SSMV_EALIGN), (dict(done=P + 2, eos=1), ssmv.SSMV_EALIGN), (dict(done=P), ssmv.SSMV_EINVAL),
    (dict(workspace=P + 8), ssmv.SSMV_EALIGN), (dict(eos=100), ssmv.SSMV_EINVAL), (dict(eos=-2), ssmv.SSMV_EINVAL), (dict(beams_in=65), ssmv.SSMV_EUNSUPPORTED),
    (dict(beams_out=65), ssmv.SSMV_EUNSUPPORTED), (dict(beams_out=0), ssmv.SSMV_EINVAL), (dict(vocab=1, beams_out=4), ssmv.SSMV_EINVAL), (dict(vocab=0), ssmv.SSMV_EINVAL),
    (dict(vocab=1 << 25), ssmv.SSMV_EUNSUPPORTED), (dict(batch=0), ssmv.SSMV_EINVAL), (dict(batch=30000), ssmv.SSMV_EUNSUPPORTED), (dict(row_stride=99), ssmv.SSMV_EINVAL),
    (dict(scores_out=P), ssmv.SSMV_EINVAL), (dict(done=P, done_out=P, eos=1), ssmv.SSMV_EINVAL), (dict(io=2), ssmv.SSMV_EINVAL),
])
def test_beam_refusals(bad, code):
    assert _code(ssmv.ssmv_beam_select, **{**BEAM, **bad}) == code


def test_history_refusals():
    d = ssmv.make_dims(2, 4, 16, 16, kmax=4, io="f32")
    assert _code(ssmv.ssmv_conv_history, d, ssmv.ssmv_cache(), P, stream=0) == ssmv.SSMV_EINVAL


def test_workspaces():
    assert _code(ssmv.ssm_selective_scan_workspace, 1, 64, 8, 10) == ssmv.SSMV_EUNSUPPORTED
    assert _code(ssmv.ssm_selective_scan_workspace, 0, 64, 16, 10) == ssmv.SSMV_EINVAL
    assert ssmv.ssm_selective_scan_workspace(64, 8192, 16, 2048) == 0                  # a batch that fills the chip is not cut
    assert ssmv.ssm_selective_scan_workspace(1, 8192, 16, 32) == 0                     # nor is a prompt of one tile
    assert _code(ssmv.ssmv_beam_workspace, 1, 65, 4, 100) == ssmv.SSMV_EUNSUPPORTED
    small, large = ssmv.ssmv_beam_workspace(1, 1, 1, 1), ssmv.ssmv_beam_workspace(16, 8, 8, 128011)
    assert 0 < small <= 256 and small < large < 1 << 22
    assert small % 16 == 0 and large % 16 == 0


@pytest.mark.parametrize("name", ["ssmv_conv_args", "ssmv_scan_args", "ssmv_token_args", "ssmv_beam_args"])
def test_packed_structs_are_the_structs(name):
    cls = getattr(ssmv, name)
    values = list(range(1, len(cls._fields_) + 1))
    packed = cls.pack(*values)
    assert len(packed) == ctypes.sizeof(cls)
    assert [getattr(cls.from_buffer_copy(packed), n) for n, _ in cls._fields_] == values


@pytest.mark.parametrize("fn,args", [("ssm_selective_scan", SCAN), ("ssm_selective_step", STEP)])
def test_a_bias_without_softplus_is_refused(fn, args):
    """The step without softplus is taken as given; a bias that would not be added is an error, not a silence."""
    with pytest.raises(ssmv.SsmvError, match="dt_bias") as ei:
        getattr(ssmv, fn)(**{**args, "dt_bias": P, "dt_softplus": False, "h_in": P, "h_out": P, "src_row": P})   # (which would end the call later)
    assert ei.value.code == ssmv.SSMV_EINVAL
