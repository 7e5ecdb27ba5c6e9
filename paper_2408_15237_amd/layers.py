"""ctypes binding of the layer operators of libssmv (declared in include/ssmv_layers.h).

Argument marshalling only, as in `binding`: what stands around and in place of a selective layer in training and decoding - the norms before
and after a block, the gated linear recurrence, both with their gradients, and the rules on logits ahead of ssmv_beam_select.
"""
from __future__ import annotations

import ctypes

from .binding import IO_CODES, SsmvError, SSMV_EHIP, _args_struct, _ck, _ptrs, _rows, _stream, load_library

SSMV_GATED_LRU, SSMV_GATED_MIX = 0, 1
FORM_CODES = {"lru": SSMV_GATED_LRU, "mix": SSMV_GATED_MIX}
SSMV_LAYER_STRIDE_MAX = 1 << 24
SSMV_BLOCK_NORM_MAX = 16384
SSMV_GATED_TILE = 64
SSMV_RULES_HISTORY_MAX = (1 << 19) - 2
SSMV_RULES_BIAS_MAX = 4095

LAYER_EXPORTS = ["ssmv_block_norm", "ssmv_block_norm_backward", "ssmv_block_norm_backward_workspace", "ssm_gated_recurrence", "ssm_gated_recurrence_workspace",
                 "ssm_gated_recurrence_backward", "ssm_gated_recurrence_backward_workspace", "ssmv_logit_rules"]

ssmv_block_norm_args = _args_struct("ssmv_block_norm_args", ("x", "z", "res", "post_wgt", "ch_scale", "pre_wgt", "r_out", "n_out"),
                                    ("x_stride", "z_stride", "res_stride", "r_stride", "n_stride"), ("rows", "channels", "io_dtype", "res_dtype"),
                                    ("eps", "res_scale"))
ssmv_block_norm_grad_args = _args_struct("ssmv_block_norm_grad_args", ("x", "z", "res", "post_wgt", "ch_scale", "pre_wgt", "dr", "dn", "dx", "dz", "dres", "dpost_wgt",
                                                                       "dch_scale", "dpre_wgt", "workspace"),
                                         ("x_stride", "z_stride", "res_stride", "dr_stride", "dn_stride", "dx_stride", "dz_stride", "dres_stride"),
                                         ("rows", "channels", "io_dtype", "res_dtype"), ("eps", "res_scale"))
ssmv_gated_args = _args_struct("ssmv_gated_args", ("x", "f", "i", "z", "A", "f_bias", "i_bias", "h_in", "src_row", "seq_len", "y_out", "h_out", "states", "workspace"),
                               ("x_stride", "f_stride", "i_stride", "z_stride", "y_stride"), ("batch", "rows_in", "channels", "L", "io_dtype", "form"))
ssmv_gated_grad_args = _args_struct("ssmv_gated_grad_args", ("x", "f", "i", "z", "A", "f_bias", "i_bias", "states", "seq_len", "dy", "dh_out", "dx", "df", "di", "dz",
                                                             "dA", "df_bias", "di_bias", "dh_in", "workspace"),
                                    ("x_stride", "f_stride", "i_stride", "z_stride", "dy_stride", "dx_stride", "df_stride", "di_stride", "dz_stride"),
                                    ("batch", "channels", "L", "io_dtype", "form"))
ssmv_rules_args = _args_struct("ssmv_rules_args", ("logits", "hist", "hist_len", "src_row", "token", "prompt_len", "repetition", "frequency", "presence", "bias_token",
                                                   "bias", "mask", "mask_row", "out", "hist_out", "hist_len_out"), ("row_stride", "out_stride", "mask_stride"),
                               ("rows", "rows_in", "vocab", "io_dtype", "hist_stride", "bias_n", "mask_rows"))

_lib = None


def _layers() -> ctypes.CDLL:
    """The library, with the signatures of these calls."""
    global _lib
    if _lib is None:
        lib = load_library()
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_size_t)
        for name in LAYER_EXPORTS:
            if not hasattr(lib, name):
                raise SsmvError(SSMV_EHIP, "the library has no %s: build it again" % name)
            fn = getattr(lib, name)
            fn.restype = ctypes.c_int
            fn.argtypes = [i32, i32, sz] if name == "ssmv_block_norm_backward_workspace" else [i32, i32, i32, sz] if name.endswith("_workspace") else [vp, vp]
        _lib = lib
    return _lib


def _size(name, *sizes) -> int:
    out = ctypes.c_size_t()
    _ck(getattr(_layers(), name)(*sizes, ctypes.byref(out)))
    return out.value


def ssmv_block_norm(*, rows: int, channels: int, io, x=None, z=None, res=None, post_wgt=None, ch_scale=None, pre_wgt=None, r_out=None, n_out=None, eps: float = 1e-5,
                    res_scale: float = 1.0, res_io=None, x_stride: int = 0, z_stride: int = 0, res_stride: int = 0, r_stride: int = 0, n_stride: int = 0,
                    stream=None) -> None:
    """res_io: the type of res and r_out, None: io's."""
    io = IO_CODES.get(io, io)
    a = ssmv_block_norm_args.pack(*_ptrs(x, z, res, post_wgt, ch_scale, pre_wgt, r_out, n_out), x_stride, z_stride, res_stride, r_stride, n_stride, rows, channels, io,
                                  io if res_io is None else IO_CODES.get(res_io, res_io), eps, res_scale)
    _ck((_lib or _layers()).ssmv_block_norm(a, _stream(stream)))


def ssmv_block_norm_backward_workspace(rows: int, channels: int) -> int:
    return _size("ssmv_block_norm_backward_workspace", rows, channels)


def ssmv_block_norm_backward(*, rows: int, channels: int, io, x=None, z=None, res=None, post_wgt=None, ch_scale=None, pre_wgt=None, dr=None, dn=None, dx=None, dz=None,
                             dres=None, dpost_wgt=None, dch_scale=None, dpre_wgt=None, eps: float = 1e-5, res_scale: float = 1.0, res_io=None, x_stride: int = 0,
                             z_stride: int = 0, res_stride: int = 0, dr_stride: int = 0, dn_stride: int = 0, dx_stride: int = 0, dz_stride: int = 0,
                             dres_stride: int = 0, workspace=None, stream=None) -> None:
    io = IO_CODES.get(io, io)
    a = ssmv_block_norm_grad_args.pack(*_ptrs(x, z, res, post_wgt, ch_scale, pre_wgt, dr, dn, dx, dz, dres, dpost_wgt, dch_scale, dpre_wgt, workspace), x_stride, z_stride,
                                       res_stride, dr_stride, dn_stride, dx_stride, dz_stride, dres_stride, rows, channels, io,
                                       io if res_io is None else IO_CODES.get(res_io, res_io), eps, res_scale)
    _ck((_lib or _layers()).ssmv_block_norm_backward(a, _stream(stream)))


def ssm_gated_recurrence_workspace(batch: int, channels: int, L: int) -> int:
    return _size("ssm_gated_recurrence_workspace", batch, channels, L)


def ssm_gated_recurrence(*, x, f, y_out, batch: int, channels: int, L: int, io, form="lru", A=None, i=None, z=None, f_bias=None, i_bias=None, h_in=None, h_out=None,
                         states=None, src_row=None, rows_in: int = 0, seq_len=None, x_stride: int = 0, f_stride: int = 0, i_stride: int = 0, z_stride: int = 0,
                         y_stride: int = 0, workspace=None, stream=None) -> None:
    a = ssmv_gated_args.pack(*_ptrs(x, f, i, z, A, f_bias, i_bias, h_in, src_row, seq_len, y_out, h_out, states, workspace), x_stride, f_stride, i_stride, z_stride,
                             y_stride, batch, _rows(h_in, rows_in, src_row), channels, L, IO_CODES.get(io, io), FORM_CODES.get(form, form))
    _ck((_lib or _layers()).ssm_gated_recurrence(a, _stream(stream)))


def ssm_gated_recurrence_backward_workspace(batch: int, channels: int, L: int) -> int:
    return _size("ssm_gated_recurrence_backward_workspace", batch, channels, L)


def ssm_gated_recurrence_backward(*, x, f, dy, states, batch: int, channels: int, L: int, io, form="lru", A=None, i=None, z=None, f_bias=None, i_bias=None, seq_len=None,
                                  dh_out=None, dx=None, df=None, di=None, dz=None, dA=None, df_bias=None, di_bias=None, dh_in=None, x_stride: int = 0, f_stride: int = 0,
                                  i_stride: int = 0, z_stride: int = 0, dy_stride: int = 0, dx_stride: int = 0, df_stride: int = 0, di_stride: int = 0, dz_stride: int = 0,
                                  workspace=None, stream=None) -> None:
    a = ssmv_gated_grad_args.pack(*_ptrs(x, f, i, z, A, f_bias, i_bias, states, seq_len, dy, dh_out, dx, df, di, dz, dA, df_bias, di_bias, dh_in, workspace), x_stride,
                                  f_stride, i_stride, z_stride, dy_stride, dx_stride, df_stride, di_stride, dz_stride, batch, channels, L, IO_CODES.get(io, io),
                                  FORM_CODES.get(form, form))
    _ck((_lib or _layers()).ssm_gated_recurrence_backward(a, _stream(stream)))


def _first(t, given: int, dim: int) -> int:
    """A size as given, else the tensor's."""
    return given or (0 if t is None or isinstance(t, int) else t.shape[dim])


def ssmv_logit_rules(*, logits, out, rows: int, vocab: int, io, row_stride: int = 0, out_stride: int = 0, hist=None, hist_len=None, src_row=None, rows_in: int = 0,
                     token=None, prompt_len=None, repetition=None, frequency=None, presence=None, hist_out=None, hist_len_out=None, hist_stride: int = 0, bias_token=None,
                     bias=None, bias_n: int = 0, mask=None, mask_row=None, mask_rows: int = 0, mask_stride: int = 0, stream=None) -> None:
    """rows_in, hist_stride, bias_n and mask_rows: 0 = as the tensors have them."""
    a = ssmv_rules_args.pack(*_ptrs(logits, hist, hist_len, src_row, token, prompt_len, repetition, frequency, presence, bias_token, bias, mask, mask_row, out, hist_out,
                                    hist_len_out), row_stride, out_stride, mask_stride, rows, _rows(hist, rows_in, src_row), vocab, IO_CODES.get(io, io),
                             _first(hist, hist_stride, -1), _first(bias_token, bias_n, -1), _first(mask, mask_rows, 0))
    _ck((_lib or _layers()).ssmv_logit_rules(a, _stream(stream)))
