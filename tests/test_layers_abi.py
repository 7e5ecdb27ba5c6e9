"""The layer operators without a GPU: argument structs as the header declares them, workspaces, and refusals on the host before any HIP call."""
import ctypes
import os
import re

import pytest

import paper_2408_15237_amd as ssmv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x20000              # plausible, aligned, never touched
STRUCTS = ["ssmv_block_norm_args", "ssmv_block_norm_grad_args", "ssmv_gated_args", "ssmv_gated_grad_args", "ssmv_rules_args"]
EINVAL, EALIGN, EUNSUPPORTED = ssmv.SSMV_EINVAL, ssmv.SSMV_EALIGN, ssmv.SSMV_EUNSUPPORTED


def _header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ssmv_layers.h")).read(), flags=re.S)


def _code(fn, **kw):
    with pytest.raises(ssmv.SsmvError) as ei:
        fn(**kw)
    return ei.value.code


def test_library_exports_every_declared_symbol():
    names = re.findall(r"^int\s+(\w+)\s*\(", _header(), flags=re.M)
    lib = ssmv.load_library()
    assert sorted(names) == sorted(ssmv.LAYER_EXPORTS) and len(names) == 8
    assert all(hasattr(lib, n) and hasattr(ssmv, n) for n in names)


def test_constants_match_the_header():
    for name in ("SSMV_BLOCK_NORM_MAX", "SSMV_GATED_TILE", "SSMV_RULES_BIAS_MAX", "SSMV_RULES_HISTORY_MAX", "SSMV_LAYER_STRIDE_MAX"):
        value = re.search(r"#define\s+%s\s+(.*)" % name, _header()).group(1)
        assert eval(value) == getattr(ssmv, name)
    assert re.search(r"SSMV_GATED_LRU = 0, SSMV_GATED_MIX = 1", _header()) and (ssmv.SSMV_GATED_LRU, ssmv.SSMV_GATED_MIX) == (0, 1)


@pytest.mark.parametrize("name", STRUCTS)
def test_argument_structs_match_the_header(name):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), _header(), flags=re.S).group(1)
    want = []
    for decl in filter(None, (d.strip() for d in body.split(";"))):
        if "*" in decl:
            kind, names = ctypes.c_void_p, re.findall(r"\*\s*(\w+)", decl)
        else:
            kind = {"int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32, "float": ctypes.c_float}[decl.split()[0]]
            names = [n.strip() for n in decl.split(None, 1)[1].split(",")]
        want += [(n, kind) for n in names]
    assert list(getattr(ssmv, name)._fields_) == want


@pytest.mark.parametrize("name", STRUCTS)
def test_packed_structs_are_the_structs(name):
    cls = getattr(ssmv, name)
    values = list(range(1, len(cls._fields_) + 1))
    packed = cls.pack(*values)
    assert len(packed) == ctypes.sizeof(cls)
    assert [getattr(cls.from_buffer_copy(packed), n) for n, _ in cls._fields_] == values


NORM = dict(x=P, z=P, res=P, post_wgt=P, ch_scale=P, pre_wgt=P, r_out=P + 4096, n_out=P + 8192, rows=2, channels=16, io="bf16", stream=0)
GRAD = dict(x=P, z=P, res=P, post_wgt=P, ch_scale=P, pre_wgt=P, dr=P + 64, dn=P + 128, dx=P + 4096, dz=P + 8192, dres=P + 12288, dpost_wgt=P, dch_scale=P, dpre_wgt=P, rows=2,
            channels=16, io="bf16", workspace=P, stream=0)
REC = dict(x=P, f=P, i=P, z=P, A=P, f_bias=P, i_bias=P, y_out=P + 64, h_in=P, h_out=P, states=P + 4096, batch=2, channels=16, L=5, io="bf16", stream=0)
BACK = dict(x=P, f=P, i=P, z=P, A=P, f_bias=P, i_bias=P, states=P, dy=P + 64, dh_out=P + 64, dx=P + 128, df=P + 256, di=P + 512, dz=P + 1024, dA=P, df_bias=P, di_bias=P, dh_in=P + 2048,
            batch=2, channels=16, L=5, io="bf16", workspace=P, stream=0)
RULES = dict(logits=P, out=P + 64, rows=2, vocab=100, io="bf16", hist=P, hist_len=P, hist_stride=10, token=P, prompt_len=P, repetition=P, frequency=P, presence=P, hist_out=P + 64,
             hist_len_out=P + 64, bias_token=P, bias=P, bias_n=3, mask=P, mask_row=P, mask_rows=2, stream=0)


@pytest.mark.parametrize("bad,code", [(dict([(k, P + 1)]), EALIGN) for k in ("x", "z", "res", "post_wgt", "ch_scale", "pre_wgt", "r_out", "n_out")] + [
    (dict(x=None, res=None), EINVAL), (dict(x=None), EINVAL), (dict(x=None, z=None, post_wgt=None, ch_scale=None), EINVAL), (dict(r_out=None, n_out=None), EINVAL),
    (dict(rows=0), EINVAL), (dict(channels=0), EINVAL), (dict(channels=16385), EUNSUPPORTED), (dict(rows=1 << 27, channels=8), EUNSUPPORTED),
    (dict(rows=1 << 23, channels=8192), EUNSUPPORTED), (dict(io=7), EINVAL), (dict(res_io=7), EINVAL), (dict(io="f32", res_io="bf16"), EINVAL),
    (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(x_stride=15), EINVAL), (dict(z_stride=-16), EINVAL), (dict(res_stride=1 << 25), EUNSUPPORTED),
    (dict(r_stride=8), EINVAL), (dict(n_stride=8), EINVAL), (dict(r_out=P, res_stride=32), EINVAL), (dict(n_out=P), EINVAL), (dict(r_out=P, res=P + 64), EINVAL),
    (dict(n_out=P + 4096), EINVAL), (dict(res_io="f32", res=P + 2), EALIGN),
])
def test_norm_refusals(bad, code):
    assert _code(ssmv.ssmv_block_norm, **{**NORM, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict([(k, P + 1)]), EALIGN) for k in ("x", "z", "res", "post_wgt", "dr", "dn", "dx", "dz", "dres", "dpost_wgt", "dch_scale", "dpre_wgt")] + [
    (dict(dr=None, dn=None), EINVAL), (dict(z=None), EINVAL), (dict(res=None), EINVAL), (dict(post_wgt=None), EINVAL), (dict(ch_scale=None), EINVAL), (dict(pre_wgt=None), EINVAL),
    (dict(x=None, z=None, post_wgt=None, ch_scale=None, dz=None, dpost_wgt=None, dch_scale=None), EINVAL), (dict(workspace=None), EINVAL), (dict(workspace=P + 8), EALIGN),
    (dict(dx=P), EINVAL), (dict(dz=P + 128), EINVAL), (dict(dres=P + 128), EINVAL), (dict(dx=P + 64), EINVAL), (dict(dx=P + 12288), EINVAL), (dict(dres=P + 64, dres_stride=32), EINVAL),
    (dict(dx=P + 128, dx_stride=32), EINVAL), (dict(dn_stride=4), EINVAL), (dict(rows=-1), EINVAL), (dict(channels=20000), EUNSUPPORTED),
    (dict(rows=1 << 27), EUNSUPPORTED),
])
def test_norm_gradient_refusals(bad, code):
    assert _code(ssmv.ssmv_block_norm_backward, **{**GRAD, **bad}) == code


GATED = [(dict([(k, P + 1)]), EALIGN) for k in ("x", "f", "i", "z", "A", "f_bias", "i_bias", "states")] + [(dict([(k, None)]), EINVAL) for k in ("x", "f", "A")] + [
    (dict(form="mix"), EINVAL), (dict(form=3), EINVAL), (dict(i=None), EINVAL), (dict(io=7), EINVAL), (dict(batch=0), EINVAL), (dict(channels=0), EINVAL), (dict(L=0), EINVAL),
    (dict(batch=70000), EUNSUPPORTED), (dict(channels=1 << 23), EUNSUPPORTED), (dict(seq_len=P + 2), EALIGN), (dict(x_stride=15), EINVAL), (dict(f_stride=15), EINVAL),
    (dict(i_stride=-1), EINVAL), (dict(z_stride=1 << 25), EUNSUPPORTED)]


@pytest.mark.parametrize("bad,code", GATED + [
    (dict(y_out=None), EINVAL), (dict(y_out=P), EINVAL), (dict(y_out=P + 1), EALIGN), (dict(h_in=P + 2), EALIGN), (dict(h_out=P + 2), EALIGN), (dict(src_row=P), EINVAL),
    (dict(src_row=P + 2), EALIGN), (dict(rows_in=1), EINVAL), (dict(rows_in=-1, src_row=P), EINVAL), (dict(states=P), EINVAL), (dict(y_stride=3), EINVAL),
    (dict(L=100000), EINVAL), (dict(L=100000, workspace=P + 4), EALIGN)])
def test_recurrence_refusals(bad, code):
    assert _code(ssmv.ssm_gated_recurrence, **{**REC, **bad}) == code


@pytest.mark.parametrize("bad,code", GATED + [
    (dict(states=None), EINVAL), (dict(dy=None), EINVAL), (dict(z=None), EINVAL), (dict(f_bias=None), EINVAL), (dict(i_bias=None), EINVAL), (dict(workspace=None), EINVAL),
    (dict(workspace=P + 8), EALIGN), (dict(dx=P), EINVAL), (dict(dx=P + 64), EINVAL), (dict(df=P + 128), EINVAL), (dict(dz=P + 512), EINVAL), (dict(dh_in=P + 64), EINVAL),
    (dict(dh_in=P), EINVAL), (dict(dx_stride=3), EINVAL), (dict(dy_stride=3), EINVAL), (dict(dz_stride=1 << 25), EUNSUPPORTED), (dict(dA=P + 2), EALIGN), (dict(dh_in=P + 2), EALIGN),
    (dict(dA=None, df_bias=None, di_bias=None, L=100000, workspace=None), EINVAL)])
def test_recurrence_gradient_refusals(bad, code):
    assert _code(ssmv.ssm_gated_recurrence_backward, **{**BACK, **bad}) == code


@pytest.mark.parametrize("bad,code", [(dict([(k, P + 1)]), EALIGN) for k in (
    "logits", "out", "hist", "hist_len", "token", "prompt_len", "repetition", "frequency", "presence", "hist_out", "hist_len_out", "bias_token", "bias", "mask", "mask_row")] + [
    (dict(logits=None), EINVAL), (dict(out=None), EINVAL), (dict(rows=0), EINVAL), (dict(vocab=0), EINVAL), (dict(rows=70000), EUNSUPPORTED), (dict(vocab=1 << 25), EUNSUPPORTED),
    (dict(io=3), EINVAL), (dict(row_stride=99), EINVAL), (dict(out_stride=1 << 25), EUNSUPPORTED), (dict(out=P, out_stride=128), EINVAL), (dict(hist=None), EINVAL),
    (dict(hist_len=None), EINVAL), (dict(hist_stride=0), EINVAL), (dict(hist_stride=1 << 19), EUNSUPPORTED), (dict(src_row=P + 2), EALIGN), (dict(rows_in=1), EINVAL),
    (dict(hist_out=None), EINVAL), (dict(hist_len_out=None), EINVAL), (dict(hist_len_out=P), EINVAL), (dict(hist_out=P, src_row=P), EINVAL), (dict(bias=None), EINVAL),
    (dict(bias_token=None), EINVAL), (dict(bias_n=0), EINVAL), (dict(bias_n=4096), EUNSUPPORTED), (dict(mask=None), EINVAL), (dict(mask_rows=0), EINVAL),
    (dict(mask_stride=3), EINVAL), (dict(mask_row=None, mask_rows=1), EINVAL)])
def test_rules_refusals(bad, code):
    assert _code(ssmv.ssmv_logit_rules, **{**RULES, **bad}) == code


def test_penalties_without_a_history_are_refused():
    bare = dict(logits=P, out=P, rows=2, vocab=100, io="f32", stream=0)
    for k in ("hist_len", "src_row", "token", "prompt_len", "repetition", "frequency", "presence", "hist_out"):
        assert _code(ssmv.ssmv_logit_rules, **{**bare, k: P}) == EINVAL


def test_workspaces():
    def size(fn, *a):
        return getattr(ssmv, fn)(*a)
    assert size("ssm_gated_recurrence_workspace", 64, 8192, 2048) == 0 and size("ssm_gated_recurrence_workspace", 1, 16, 100) == 0
    assert 0 < size("ssm_gated_recurrence_workspace", 1, 16, 1 << 20) < 1 << 14
    assert size("ssm_gated_recurrence_backward_workspace", 3, 16, 1 << 20) % 16 == 0
    assert size("ssm_gated_recurrence_backward_workspace", 3, 16, 1) >= 3 * 3 * 16 * 4
    assert size("ssmv_block_norm_backward_workspace", 1, 1) >= 3 * 4 and size("ssmv_block_norm_backward_workspace", 1 << 20, 5120) <= 1 << 26
    for fn, bad in (("ssm_gated_recurrence_workspace", (0, 1, 1)), ("ssm_gated_recurrence_backward_workspace", (1, 1, 0)), ("ssmv_block_norm_backward_workspace", (1, 0))):
        with pytest.raises(ssmv.SsmvError) as ei:
            size(fn, *bad)
        assert ei.value.code == EINVAL
