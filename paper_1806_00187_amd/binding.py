"""ctypes binding of libnmt.so: one Python function per C entry point, same names, argument
marshalling only.  Device buffers are torch tensors (their data_ptr() is passed through); the HIP
stream is torch's current stream unless one is given.  The library must have been built
(`python -m paper_1806_00187_amd.build`); there is no fallback of any kind."""
from __future__ import annotations

import ctypes as C
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnmt.so")

NMT_OK, NMT_EINVAL, NMT_ESTATE, NMT_ENOMEM, NMT_EHIP = 0, -1, -2, -3, -4


class NmtError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"libnmt error {code}: {msg}")
        self.code = code


class nmt_config(C.Structure):
    _fields_ = [("enc_layers", C.c_int32), ("dec_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("d_ff", C.c_int32), ("vocab", C.c_int32), ("pad_id", C.c_int32), ("dropout", C.c_float),
                ("attn_dropout", C.c_float), ("act_dropout", C.c_float), ("label_smoothing", C.c_float), ("ln_eps", C.c_float), ("seed", C.c_uint64),
                ("max_sentences", C.c_int32), ("max_len", C.c_int32)]


class nmt_dropout(C.Structure):
    _fields_ = [("p", C.c_float), ("site", C.c_uint32), ("step", C.c_uint32), ("micro", C.c_uint32), ("seed", C.c_uint64),
                ("n_pos", C.c_int32), ("d_sent_uid", C.c_void_p)]


class nmt_segment(C.Structure):
    _fields_ = [("B", C.c_int32), ("S", C.c_int32), ("T", C.c_int32), ("micro_idx", C.c_uint32)]


class nmt_wgrad(C.Structure):
    _fields_ = [("d_dy", C.c_void_p), ("d_x", C.c_void_p), ("d_gw", C.c_void_p), ("d_gb", C.c_void_p), ("ld_dy", C.c_int32), ("ld_x", C.c_int32),
                ("ld_gw", C.c_int32), ("out", C.c_int32), ("in_", C.c_int32), ("rows", C.c_int32)]


class nmt_gated_norm(C.Structure):
    _fields_ = [("rows", C.c_int32), ("d", C.c_int32), ("type", C.c_int32), ("kind", C.c_int32), ("eps", C.c_float), ("resid_scale", C.c_float),
                ("rows_per_gate", C.c_int32), ("ld_x", C.c_int64), ("ld_y", C.c_int64), ("ld_h", C.c_int64), ("ld_n", C.c_int64),
                ("d_x", C.c_void_p), ("d_y", C.c_void_p), ("d_post_gain", C.c_void_p), ("d_post_shift", C.c_void_p), ("d_gate", C.c_void_p),
                ("d_pre_gain", C.c_void_p), ("d_pre_shift", C.c_void_p), ("d_h", C.c_void_p), ("d_n", C.c_void_p), ("d_stats", C.c_void_p)]


class nmt_gated_norm_grad(C.Structure):
    _fields_ = [("ld_dh", C.c_int64), ("ld_dn", C.c_int64), ("ld_dx", C.c_int64), ("ld_dy", C.c_int64), ("d_dh", C.c_void_p), ("d_dn", C.c_void_p),
                ("d_dx", C.c_void_p), ("d_dy", C.c_void_p), ("d_dpost_gain", C.c_void_p), ("d_dpost_shift", C.c_void_p), ("d_dgate", C.c_void_p),
                ("d_dpre_gain", C.c_void_p), ("d_dpre_shift", C.c_void_p), ("d_scratch", C.c_void_p), ("scratch_floats", C.c_int64)]


class nmt_adamw_tensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("weight_decay", C.c_float), ("lr_factor", C.c_float), ("d_master", C.c_void_p), ("d_m", C.c_void_p),
                ("d_v", C.c_void_p), ("d_m_scale", C.c_void_p), ("d_v_scale", C.c_void_p), ("d_grad", C.c_void_p), ("d_weights", C.c_void_p)]


class nmt_norm8(C.Structure):
    _fields_ = [("rows", C.c_int32), ("d", C.c_int32), ("type", C.c_int32), ("kind", C.c_int32), ("eps", C.c_float), ("resid_scale", C.c_float),
                ("ld_x", C.c_int64), ("ld_y", C.c_int64), ("ld_h", C.c_int64), ("ld_n", C.c_int64), ("ld_codes", C.c_int64), ("ld_scales", C.c_int64),
                ("d_x", C.c_void_p), ("d_y", C.c_void_p), ("d_gain", C.c_void_p), ("d_shift", C.c_void_p), ("d_h", C.c_void_p), ("d_n", C.c_void_p),
                ("d_codes", C.c_void_p), ("d_scales", C.c_void_p), ("d_stats", C.c_void_p)]


class nmt_gemm8(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32), ("batch", C.c_int32), ("type", C.c_int32), ("a_square", C.c_int32),
                ("b_square", C.c_int32), ("lda", C.c_int64), ("ldb", C.c_int64), ("ldc", C.c_int64), ("ld_add", C.c_int64), ("ld_sa", C.c_int64),
                ("ld_sb", C.c_int64), ("stride_a", C.c_int64), ("stride_b", C.c_int64), ("stride_c", C.c_int64), ("stride_add", C.c_int64),
                ("stride_bias", C.c_int64), ("stride_sa", C.c_int64), ("stride_sb", C.c_int64), ("d_a", C.c_void_p), ("d_b", C.c_void_p),
                ("d_sa", C.c_void_p), ("d_sb", C.c_void_p), ("d_bias", C.c_void_p), ("d_add", C.c_void_p), ("d_c", C.c_void_p),
                ("d_ranges", C.c_void_p), ("d_scratch", C.c_void_p), ("scratch_floats", C.c_int64)]


class nmt_expert_layer8(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("k", C.c_int32), ("experts", C.c_int32), ("d", C.c_int32), ("ff", C.c_int32), ("type", C.c_int32),
                ("act", C.c_int32), ("ld_x", C.c_int64), ("ld_add", C.c_int64), ("ld_out", C.c_int64), ("ld_up", C.c_int64), ("stride_up", C.c_int64),
                ("ld_up_scales", C.c_int64), ("stride_up_scales", C.c_int64), ("ld_down", C.c_int64), ("stride_down", C.c_int64),
                ("ld_down_scales", C.c_int64), ("stride_down_scales", C.c_int64), ("d_x", C.c_void_p), ("d_expert", C.c_void_p),
                ("d_weights", C.c_void_p), ("d_up", C.c_void_p), ("d_up_scales", C.c_void_p), ("d_down", C.c_void_p), ("d_down_scales", C.c_void_p),
                ("d_add", C.c_void_p), ("d_out", C.c_void_p), ("d_scratch", C.c_void_p), ("scratch_floats", C.c_int64)]


_P, _I32, _I64, _F, _U32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_uint32
_DP = C.POINTER(nmt_dropout)
_SP = C.POINTER(nmt_segment)

_SIGNATURES = {
    "nmt_last_error": (C.c_char_p, []),
    "nmt_create": (C.c_int, [C.POINTER(nmt_config), C.POINTER(_P)]),
    "nmt_destroy": (None, [_P]),
    "nmt_param_count": (_I64, [_P]),
    "nmt_param_tensors": (_I32, [_P]),
    "nmt_grad_scale": (C.c_float, [_P]),
    "nmt_param_info": (C.c_int, [_P, _I32, C.POINTER(C.c_char_p), C.POINTER(_I64), C.POINTER(_I32), C.POINTER(_I32)]),
    "nmt_workspace_bytes": (_I64, [_P, _I32, _I32, _I32]),
    "nmt_workspace_bytes_group": (_I64, [_P, _I32, _SP]),
    "nmt_bind": (C.c_int, [_P, _P, _P, _P, _P, _P, _P, _P, _I64]),
    "nmt_forward_loss": (C.c_int, [_P, _P, _P, _P, _I32, _I32, _I32, _F, _U32, _U32, _P, _I32, _P, _P, _P]),
    "nmt_forward_loss_group": (C.c_int, [_P, _I32, _SP, _P, _P, _P, _F, _U32, _P, _I32, _P, _P, _P]),
    "nmt_workspace_bytes_packed": (_I64, [_P, _I32, _I64, _I64]),
    "nmt_forward_loss_packed": (C.c_int, [_P, _I32, _P, _I64, _I64, _I32, _I32, _P, _P, _P, _F, _U32, _I32, _P, _P, _P]),
    "nmt_backward": (C.c_int, [_P, _P]),
    "nmt_accumulate": (C.c_int, [_P, _I32, _P]),
    "nmt_accumulate_loss": (C.c_int, [_P, _I32, _P, _P, _P]),
    "nmt_tuning": (C.c_int, [C.c_char_p, _I32]),
    "nmt_gemm_timing": (C.c_int, [C.POINTER(C.c_double), C.POINTER(_I64), C.POINTER(C.c_double)]),
    "nmt_debug_activation": (C.c_int, [_P, C.c_char_p, C.POINTER(_P), C.POINTER(_I64), C.POINTER(_I64)]),
    "nmt_check_overflow": (C.c_int, [_P, _F, _P, _P]),
    "nmt_adam_step": (C.c_int, [_P, _F, _F, _F, _F, _I32, _P, _P]),
    "nmt_finish_update": (C.c_int, [_P, _I32, _F, _F, _F, _F, _F, _I32, _P, _P]),
    "nmt_scaler_update": (C.c_int, [C.POINTER(C.c_float), C.POINTER(_I32), _I32, _I32]),
    "nmt_lr_schedule": (C.c_double, [_I64, C.c_double, _I64]),
    "nmt_op_gemm": (C.c_int, [_P, _I32, _I32, _P, _I32, _I32, _P, _I32, _I32, _I32, _I32, _P, _I32, _DP, _P, _P, _F, _P]),
    "nmt_op_gemm_f32": (C.c_int, [_P, _I32, _I32, _P, _I32, _I32, _P, _I32, _I32, _I32, _I32, _I32, _P]),
    "nmt_op_gemm_splitk": (C.c_int, [_P, _I32, _I32, _P, _I32, _I32, _P, _I32, _I32, _I32, _I32, _P, _I64, _I32, _P]),
    "nmt_op_wgrad_group": (C.c_int, [_I32, C.POINTER(nmt_wgrad), _F, _P, _I64, _I32, _I32, _P]),
    "nmt_op_attention_fwd": (C.c_int, [_P, _I32, _P, _I32, _P, _I32, _P, _I32, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _P]),
    "nmt_op_attention_bwd": (C.c_int, [_P, _I32, _P, _I32, _P, _I32, _P, _I32, _P, _I32, _P, _P, _I32, _P, _I32, _P, _I32, _P,
                                       _I32, _I32, _I32, _I32, _I32, _I32, _I32, _P]),
    "nmt_op_residual_layernorm_fwd": (C.c_int, [_P, _P, _P, _P, _P, _P, _I32, _I32, _F, _DP, _P]),
    "nmt_op_layernorm_bwd_scratch": (_I64, [_I32]),
    "nmt_op_residual_layernorm_bwd": (C.c_int, [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _P, _I32, _I32, _DP, _P]),
    "nmt_op_embed_fwd": (C.c_int, [_P, _P, _P, _I32, _I32, _I32, _DP, _P]),
    "nmt_op_softmax_xent": (C.c_int, [_P, _P, _P, _I32, _I32, _I32, _F, _F, _P, _P, _P]),
    "nmt_op_colsum_scratch": (_I64, [_I32]),
    "nmt_op_colsum": (C.c_int, [_P, _I32, _P, _P, _I32, _I32, _P]),
    "nmt_op_colsum_static": (C.c_int, [_P, _I32, _P, _I32, _I32, _P]),
    "nmt_op_embed_bwd_scratch": (_I64, [_I32, _I32, _I32]),
    "nmt_op_embed_bwd": (C.c_int, [_P, _P, _I32, _DP, _P, _P, _I32, _DP, _P, _I32, _I32, _P, _P]),
    "nmt_op_accumulate": (C.c_int, [_P, _P, _I64, _I32, _P]),
    "nmt_op_check_overflow": (C.c_int, [_P, _I64, _F, _P, _P]),
    "nmt_op_adam": (C.c_int, [_P, _P, _P, _P, _F, _P, _I64, _F, _F, _F, _F, _I32, _P, _P]),
    "nmt_op_dropout_mask": (C.c_int, [_P, _I32, _I32, _DP, _P]),
    "nmt_op_gated_norm_fwd": (C.c_int, [C.POINTER(nmt_gated_norm), _P]),
    "nmt_debug_gated_norm_grid": (C.c_int, [_I32, _I32, _I32, C.POINTER(_I64), C.POINTER(_I32)]),
    "nmt_op_gated_norm_bwd_scratch": (_I64, [_I32, _I32, _I32]),
    "nmt_op_gated_norm_bwd": (C.c_int, [C.POINTER(nmt_gated_norm), C.POINTER(nmt_gated_norm_grad), _P]),
    "nmt_op_expert_dispatch_scratch": (_I64, [_I32, _I32, _I32]),
    "nmt_op_expert_dispatch": (C.c_int, [_P, _I32, _I32, _I32, _I32, _P, _I64, _I32, _I32, _P, _I64, _P, _P, _P, _I64, _P]),
    "nmt_op_expert_combine": (C.c_int, [_P, _I64, _I32, _P, _P, _P, _I64, _P, _I64, _I32, _I32, _I32, _I32, _P]),
    "nmt_op_expert_combine_bwd": (C.c_int, [_P, _I64, _P, _I64, _I32, _P, _P, _P, _I64, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32, _P]),
    "nmt_adamw_table_bytes": (_I64, [_I32, C.POINTER(nmt_adamw_tensor)]),
    "nmt_adamw_create": (C.c_int, [_I32, C.POINTER(nmt_adamw_tensor), _I32, _I32, _I32, _P, _I64, _P, C.POINTER(_P)]),
    "nmt_adamw_destroy": (None, [_P]),
    "nmt_op_quantize8": (C.c_int, [_P, _I64, _I32, _I32, _I32, _I32, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P]),
    "nmt_op_norm8": (C.c_int, [_P, _P]),
    "nmt_op_gemm8_scratch": (_I64, [_I32, _I32, _I32, _I32, _I32]),
    "nmt_op_gemm8": (C.c_int, [_P, _P]),
    "nmt_debug_gemm8_form": (C.c_int, [_I32, _I32, _I32, _I32, _I32, _I32, _I32, C.POINTER(_I32), C.POINTER(_I32)]),
    "nmt_op_expert_layer8_scratch": (_I64, [_I32, _I32, _I32, _I32, _I32]),
    "nmt_op_expert_layer8": (C.c_int, [_P, _P]),
    "nmt_adamw_step": (C.c_int, [_P, C.c_double, C.c_double, C.c_double, C.c_double, _I32, _F, _P, _P]),
}

_lib = None


def load():
    """Loads libnmt.so and declares every entry point; raises if the library has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_1806_00187_amd.build`")
        # torch first: the library then binds to the HIP runtime torch has already loaded, the one that owns
        # the tensors' memory and streams (loaded the other way round, the process ends up with two runtimes
        # and the library's own sees no device)
        import torch  # noqa: F401
        lib = C.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _torch_types()
        _lib = lib
    return _lib


def exported_symbols():
    return sorted(_SIGNATURES)


def _check(rc):
    if rc != NMT_OK:
        raise NmtError(rc, load().nmt_last_error().decode())


def _p(t):
    """Device (or host) address of a torch tensor, or NULL."""
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is not None:
        return C.c_void_p(stream)
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _drop(drop):
    """drop: None or dict(p, site, step, micro, seed, n_pos, sent_uid=tensor|None)."""
    if drop is None:
        return None
    uid = drop.get("sent_uid")
    return C.byref(nmt_dropout(drop.get("p", 0.0), drop.get("site", 0), drop.get("step", 0), drop.get("micro", 0),
                               drop.get("seed", 0), drop["n_pos"], None if uid is None else uid.data_ptr()))


# ---- context ------------------------------------------------------------------------------------
def nmt_create(**cfg):
    c = nmt_config(**cfg)
    out = C.c_void_p()
    _check(load().nmt_create(C.byref(c), C.byref(out)))
    return out


def nmt_destroy(ctx):
    load().nmt_destroy(ctx)


def nmt_param_count(ctx):
    return load().nmt_param_count(ctx)


def nmt_grad_scale(ctx):
    return load().nmt_grad_scale(ctx)


def nmt_param_tensors(ctx):
    return load().nmt_param_tensors(ctx)


def nmt_param_info(ctx, idx):
    name, off, rows, cols = C.c_char_p(), C.c_int64(), C.c_int32(), C.c_int32()
    _check(load().nmt_param_info(ctx, idx, C.byref(name), C.byref(off), C.byref(rows), C.byref(cols)))
    return name.value.decode(), off.value, rows.value, cols.value


def nmt_workspace_bytes(ctx, B, S, T):
    n = load().nmt_workspace_bytes(ctx, B, S, T)
    if n < 0:
        _check(int(n))
    return n


def _segments(segs):
    """segs: sequence of (B, S, T, micro_idx)."""
    arr = (nmt_segment * len(segs))()
    for i, (B, S, T, micro) in enumerate(segs):
        arr[i] = nmt_segment(B, S, T, micro)
    return arr


def nmt_workspace_bytes_group(ctx, segs):
    n = load().nmt_workspace_bytes_group(ctx, len(segs), _segments(segs))
    if n < 0:
        _check(int(n))
    return n


def nmt_bind(ctx, w16, g16, master32=None, acc32=None, adam_m=None, adam_v=None, workspace=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().nmt_bind(ctx, _p(w16), _p(g16), _p(master32), _p(acc32), _p(adam_m), _p(adam_v), _p(workspace), ws_bytes))


# ---- the training step --------------------------------------------------------------------------
def nmt_forward_loss(ctx, src, tgt_in, tgt_out, loss_scale, step, micro_idx, loss_sum, ntok, sent_uid=None, training=True,
                     stream=None):
    B, S = src.shape
    T = tgt_in.shape[1]
    _check(load().nmt_forward_loss(ctx, _p(src), _p(tgt_in), _p(tgt_out), B, S, T, loss_scale, step, micro_idx, _p(sent_uid),
                                   1 if training else 0, _p(loss_sum), _p(ntok), _stream(stream)))


def nmt_forward_loss_group(ctx, segs, src, tgt_in, tgt_out, loss_scale, step, loss_sum, ntok, sent_uid=None, training=True,
                           stream=None):
    """segs: sequence of (B, S, T, micro_idx); src / tgt_in / tgt_out: flat int32 tensors holding the sub-batches one after
    another; sent_uid: one uint32 per sentence in the same order, or None."""
    _check(load().nmt_forward_loss_group(ctx, len(segs), _segments(segs), _p(src), _p(tgt_in), _p(tgt_out), loss_scale, step,
                                         _p(sent_uid), 1 if training else 0, _p(loss_sum), _p(ntok), _stream(stream)))


def nmt_workspace_bytes_packed(ctx, n_sent, n_src_tokens, n_tgt_tokens):
    n = load().nmt_workspace_bytes_packed(ctx, n_sent, n_src_tokens, n_tgt_tokens)
    if n < 0:
        _check(int(n))
    return n


def nmt_forward_loss_packed(ctx, sentences, n_src_tokens, n_tgt_tokens, max_src_len, max_tgt_len, src, tgt_in, tgt_out, loss_scale,
                            step, loss_sum, ntok, training=True, stream=None):
    """sentences: int32 device tensor [n_sent, 4] = (src_len, tgt_len, uid, micro_idx) per sentence; src / tgt_in / tgt_out: flat
    int32 device tensors of n_src_tokens / n_tgt_tokens ids, sentences back to back."""
    _check(load().nmt_forward_loss_packed(ctx, sentences.shape[0], _p(sentences), n_src_tokens, n_tgt_tokens, max_src_len, max_tgt_len,
                                          _p(src), _p(tgt_in), _p(tgt_out), loss_scale, step, 1 if training else 0, _p(loss_sum),
                                          _p(ntok), _stream(stream)))


def nmt_backward(ctx, stream=None):
    _check(load().nmt_backward(ctx, _stream(stream)))


def nmt_accumulate(ctx, first, stream=None):
    _check(load().nmt_accumulate(ctx, 1 if first else 0, _stream(stream)))


def nmt_accumulate_loss(ctx, first, loss_total, ntok_total, stream=None):
    _check(load().nmt_accumulate_loss(ctx, 1 if first else 0, _p(loss_total), _p(ntok_total), _stream(stream)))


def nmt_debug_activation(ctx, name):
    """(device address, rows, cols) of a saved fp16 activation of the last forward pass."""
    ptr, rows, cols = C.c_void_p(), C.c_int64(), C.c_int64()
    _check(load().nmt_debug_activation(ctx, name.encode(), C.byref(ptr), C.byref(rows), C.byref(cols)))
    return ptr.value, rows.value, cols.value


def nmt_gemm_timing():
    """(milliseconds, products, algorithmic FLOPs) of the GEMM products launched since the last call with "gemm_timing" on."""
    ms, n, fl = C.c_double(), C.c_int64(), C.c_double()
    _check(load().nmt_gemm_timing(C.byref(ms), C.byref(n), C.byref(fl)))
    return ms.value, n.value, fl.value


_TUNING_SET = {}   # what this process has set through nmt_tuning (the library has no call that reads a switch back)


def nmt_tuning(name, value=0):
    _check(load().nmt_tuning(name.encode(), int(value)))
    if name == "defaults":
        _TUNING_SET.clear()
    else:
        _TUNING_SET[name] = int(value)


def tuning_value(name, default):
    """The value last set for a launch-form switch through nmt_tuning, or `default` (the library's) if none was."""
    return _TUNING_SET.get(name, default)


def nmt_check_overflow(ctx, inv_scale, flag, stream=None):
    _check(load().nmt_check_overflow(ctx, inv_scale, _p(flag), _stream(stream)))


def nmt_adam_step(ctx, lr, beta1, beta2, eps, t, flag, stream=None):
    _check(load().nmt_adam_step(ctx, lr, beta1, beta2, eps, t, _p(flag), _stream(stream)))


def nmt_finish_update(ctx, first, inv_scale, lr, beta1, beta2, eps, t, flag, stream=None):
    _check(load().nmt_finish_update(ctx, 1 if first else 0, inv_scale, lr, beta1, beta2, eps, t, _p(flag), _stream(stream)))


def nmt_scaler_update(scale, clean, overflow, window=2000):
    s, c = C.c_float(scale), C.c_int32(clean)
    _check(load().nmt_scaler_update(C.byref(s), C.byref(c), 1 if overflow else 0, window))
    return s.value, c.value


def nmt_lr_schedule(t, peak, warmup=4000):
    return load().nmt_lr_schedule(t, peak, warmup)


# ---- kernel-level entry points -------------------------------------------------------------------
def nmt_op_gemm(A, a_t, lda, B, b_t, ldb, Cout, ldc, M, N, K, bias=None, relu=False, drop=None, add=None, relu_src=None,
                mask_scale=1.0, stream=None):
    _check(load().nmt_op_gemm(_p(A), int(a_t), lda, _p(B), int(b_t), ldb, _p(Cout), ldc, M, N, K, _p(bias), int(relu), _drop(drop),
                              _p(add), _p(relu_src), mask_scale, _stream(stream)))


def nmt_op_gemm_f32(A, a_t, lda, B, b_t, ldb, Cout, ldc, M, N, K, splits=1, stream=None):
    _check(load().nmt_op_gemm_f32(_p(A), int(a_t), lda, _p(B), int(b_t), ldb, _p(Cout), ldc, M, N, K, splits, _stream(stream)))


def nmt_op_gemm_splitk(A, a_t, lda, B, b_t, ldb, Cout, ldc, M, N, K, partial, splits=0, stream=None):
    _check(load().nmt_op_gemm_splitk(_p(A), int(a_t), lda, _p(B), int(b_t), ldb, _p(Cout), ldc, M, N, K, _p(partial), partial.numel(),
                                     splits, _stream(stream)))


def nmt_op_wgrad_group(products, out_scale=1.0, partial=None, tile=0, splits=0, stream=None):
    """products: list of (dy, ld_dy, x, ld_x, gw, ld_gw, gb or None, out, in, rows)."""
    arr = (nmt_wgrad * len(products))()
    for w, (dy, ld_dy, x, ld_x, gw, ld_gw, gb, n_out, n_in, rows) in zip(arr, products):
        w.d_dy, w.d_x, w.d_gw, w.d_gb = (None if t is None else t.data_ptr() for t in (dy, x, gw, gb))
        w.ld_dy, w.ld_x, w.ld_gw, w.out, w.in_, w.rows = ld_dy, ld_x, ld_gw, n_out, n_in, rows
    _check(load().nmt_op_wgrad_group(len(products), arr, out_scale, _p(partial), 0 if partial is None else partial.numel(), tile, splits,
                                     _stream(stream)))


def nmt_op_attention_fwd(Q, ldq, K, ldk, V, ldv, O, ldo, lse, key_ids, pad_id, causal, B, H, dh, Tq, Tk, stream=None):
    _check(load().nmt_op_attention_fwd(_p(Q), ldq, _p(K), ldk, _p(V), ldv, _p(O), ldo, _p(lse), _p(key_ids), pad_id, int(causal),
                                       B, H, dh, Tq, Tk, _stream(stream)))


def nmt_op_attention_bwd(Q, ldq, K, ldk, V, ldv, O, ldo, dO, lddo, lse, dQ, lddq, dK, lddk, dV, lddv, key_ids, pad_id, causal, B, H,
                         dh, Tq, Tk, stream=None):
    _check(load().nmt_op_attention_bwd(_p(Q), ldq, _p(K), ldk, _p(V), ldv, _p(O), ldo, _p(dO), lddo, _p(lse), _p(dQ), lddq, _p(dK),
                                       lddk, _p(dV), lddv, _p(key_ids), pad_id, int(causal), B, H, dh, Tq, Tk, _stream(stream)))


def nmt_op_residual_layernorm_fwd(sub, resid, gamma, beta, out, stats, rows, d, eps, drop=None, stream=None):
    _check(load().nmt_op_residual_layernorm_fwd(_p(sub), _p(resid), _p(gamma), _p(beta), _p(out), _p(stats), rows, d, eps, _drop(drop),
                                                _stream(stream)))


def nmt_op_layernorm_bwd_scratch(d):
    return load().nmt_op_layernorm_bwd_scratch(d)


def nmt_op_residual_layernorm_bwd(dout, sub, resid, gamma, stats, dy, dym, dgamma, dbeta, dbias, partial, rows, d, drop=None,
                                  stream=None):
    _check(load().nmt_op_residual_layernorm_bwd(_p(dout), _p(sub), _p(resid), _p(gamma), _p(stats), _p(dy), _p(dym), _p(dgamma),
                                                _p(dbeta), _p(dbias), _p(partial), rows, d, _drop(drop), _stream(stream)))


def nmt_op_embed_fwd(ids, E, x, rows, d, vocab, drop, stream=None):
    _check(load().nmt_op_embed_fwd(_p(ids), _p(E), _p(x), rows, d, vocab, _drop(drop), _stream(stream)))


def nmt_op_softmax_xent(logits, targets, row_loss, rows, V, pad_id, label_smoothing, loss_scale, loss_sum, ntok, stream=None):
    _check(load().nmt_op_softmax_xent(_p(logits), _p(targets), _p(row_loss), rows, V, pad_id, label_smoothing, loss_scale,
                                      _p(loss_sum), _p(ntok), _stream(stream)))


def nmt_op_colsum_scratch(cols):
    return load().nmt_op_colsum_scratch(cols)


def nmt_op_colsum(src, ld, dst, partial, rows, cols, stream=None):
    _check(load().nmt_op_colsum(_p(src), ld, _p(dst), _p(partial), rows, cols, _stream(stream)))


def nmt_op_colsum_static(src, ld, dst, rows, cols, stream=None):
    _check(load().nmt_op_colsum_static(_p(src), ld, _p(dst), rows, cols, _stream(stream)))


def nmt_op_embed_bwd_scratch(vocab, rows_total, d):
    return load().nmt_op_embed_bwd_scratch(vocab, rows_total, d)


def nmt_op_embed_bwd(ids_a, dx_a, rows_a, drop_a, ids_b, dx_b, rows_b, drop_b, gE, d, vocab, scratch, stream=None):
    _check(load().nmt_op_embed_bwd(_p(ids_a), _p(dx_a), rows_a, _drop(drop_a), _p(ids_b), _p(dx_b), rows_b, _drop(drop_b), _p(gE), d,
                                   vocab, _p(scratch), _stream(stream)))


def nmt_op_accumulate(g16, acc32, n, first, stream=None):
    _check(load().nmt_op_accumulate(_p(g16), _p(acc32), n, 1 if first else 0, _stream(stream)))


def nmt_op_check_overflow(acc32, n, inv_scale, flag, stream=None):
    _check(load().nmt_op_check_overflow(_p(acc32), n, inv_scale, _p(flag), _stream(stream)))


def nmt_op_adam(master32, m, v, g32, w16, n, lr, beta1, beta2, eps, t, flag, grad_scale=1.0, stream=None):
    _check(load().nmt_op_adam(_p(master32), _p(m), _p(v), _p(g32), grad_scale, _p(w16), n, lr, beta1, beta2, eps, t, _p(flag),
                              _stream(stream)))


def nmt_op_dropout_mask(keep, rows, n_cols, drop, stream=None):
    _check(load().nmt_op_dropout_mask(_p(keep), rows, n_cols, _drop(drop), _stream(stream)))


# ---- norms around a gated block, experts, AdamW ----------------------------------------------------
# These take sizes, types and distances between rows from their tensors and refuse tensors that do not fit each other; the call goes
# to the stream of the tensors' device.  A small call is bound by what is done here, so nothing is looked up twice.
NMT_F16, NMT_BF16, NMT_F32 = 0, 1, 2
NMT_NORM_LAYER, NMT_NORM_RMS, NMT_ONE_GATE = 0, 1, 2 ** 31 - 1
_MOST = 2 ** 31 - 1
_KINDS = {"layer": NMT_NORM_LAYER, "rms": NMT_NORM_RMS}
_TYPES = {}          # torch dtypes -> type codes; filled with _FLOAT and _INT when torch is there (load())
_FLOAT = _INT = _E4M3 = _torch = _raw_stream = _current_device = None


def _torch_types():
    global _FLOAT, _INT, _E4M3, _torch, _raw_stream, _current_device
    import torch
    _torch = torch
    # (what torch.cuda.current_stream looks up, without the Stream object around it: 0.1 us instead of 1)
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
    # (what torch.cuda.current_device asks, without looking whether the GPU is in use yet: there are tensors on it)
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _TYPES.update({torch.float16: NMT_F16, torch.bfloat16: NMT_BF16, torch.float32: NMT_F32})
    _FLOAT, _INT, _E4M3 = torch.float32, torch.int32, torch.float8_e4m3fn


def _refuse(msg, code=NMT_EINVAL):
    raise NmtError(code, msg)


def _type_code(dtype, who):
    code = _TYPES.get(dtype)
    if code is None:
        _refuse(f"{who}: rows of {dtype}: float16, bfloat16 or float32")
    return code


def _rows_of(t, who, what):
    """(rows, d, dtype, device) of the tensor that the others are held to."""
    if t is None or t.dim() != 2:
        _refuse(f"{who}: {what} is a two-dimensional tensor")
    rows, d = t.shape
    if rows > _MOST or d > _MOST:
        _refuse(f"{who}: {what} is {tuple(t.shape)}: sizes are of 32 bits")
    return rows, d, t.dtype, t.get_device()


def _matrix(t, rows, d, dtype, device, what):
    """Address of a [rows, d] tensor of that type on that device, and the distance between its rows."""
    if t.dtype is not dtype or t.get_device() != device or t.shape != (rows, d):
        _refuse(f"{what} is {tuple(t.shape)} {t.dtype} on {t.device}, not ({rows}, {d}) {dtype} on device {device}")
    ld, step = t.stride()
    if rows <= 1:
        ld = d
    if (step != 1 and d > 1) or ld < d:
        _refuse(f"{what} has strides {t.stride()}: rows whose elements lie side by side and that do not overlap are taken")
    return t.data_ptr(), ld


def _vector(t, n, dtype, device, what):
    """Address of a contiguous tensor of n elements."""
    if t.dtype is not dtype or t.get_device() != device or t.numel() != n or not t.is_contiguous():
        _refuse(f"{what} is {tuple(t.shape)} {t.dtype} on {t.device}, not {n} contiguous elements of {dtype} on device {device}")
    return t.data_ptr()


def _call(fn, device, stream, *args, out=None):
    """fn(*args, stream[, address of out]) with `device` as the current one; its current stream if none is given."""
    if device < 0:
        _refuse(f"{fn.__name__}: the tensors are not on a GPU")
    if stream is None:
        stream = _raw_stream(device)
    last = (stream,) if out is None else (stream, C.byref(out))
    if device == _current_device():
        rc = fn(*args, *last)
    else:
        with _torch.cuda.device(device):
            rc = fn(*args, *last)
    if rc != NMT_OK:
        _check(rc)


def _gates(gate, rows, rows_per_gate, who):
    """(rows of the gate, rows_per_gate)"""
    if rows == 0:       # (no gates, or the one that all rows share: the tensor says which)
        return (0, 1) if gate.numel() == 0 else (1, NMT_ONE_GATE)
    if rows_per_gate is None or rows_per_gate >= rows:
        return 1, rows
    if rows_per_gate < 1:
        _refuse(f"{who}: rows_per_gate must be at least 1")
    return -(-rows // rows_per_gate), rows_per_gate


def _norm_parts(a, rows, d, dtype, device, post, gate, pre, kind, rows_per_gate, resid_scale, who):
    """What the forward and the backward call take alike."""
    if kind not in _KINDS:
        _refuse(f"{who}: kind {kind!r}: 'layer' or 'rms'")
    a.rows, a.d, a.type, a.kind, a.resid_scale = rows, d, _type_code(dtype, who), _KINDS[kind], resid_scale
    if post is not None:
        gain, shift = post
        a.d_post_gain = _vector(gain, d, dtype, device, "the gain after the block")
        if shift is not None:
            a.d_post_shift = _vector(shift, d, dtype, device, "the shift after the block")
    if gate is not None:
        gates, a.rows_per_gate = _gates(gate, rows, rows_per_gate, who)
        a.d_gate = _vector(gate, gates * d, dtype, device, "the gate")
    if pre is not None:
        gain, shift = pre
        a.d_pre_gain = _vector(gain, d, dtype, device, "the gain before the next block")
        if shift is not None:
            a.d_pre_shift = _vector(shift, d, dtype, device, "the shift before the next block")


def nmt_op_gated_norm_fwd(x, y, h, n, stats=None, post=None, gate=None, pre=None, kind="layer", rows_per_gate=None, resid_scale=1.0, eps=1e-5,
                          stream=None):
    """h = resid_scale * x + gate * post(y), n = pre(h).  post, pre: (gain, shift or None) or None; rows_per_gate None: one gate for all rows.
    y None: n = pre(x); resid_scale is then 1."""
    lib = _lib or load()
    rows, d, dtype, device = _rows_of(x, "nmt_op_gated_norm_fwd", "x")
    a = nmt_gated_norm()
    _norm_parts(a, rows, d, dtype, device, post, gate, pre, kind, rows_per_gate, resid_scale, "nmt_op_gated_norm_fwd")
    a.eps = eps
    a.d_x, a.ld_x = _matrix(x, rows, d, dtype, device, "x")
    if y is not None:
        a.d_y, a.ld_y = _matrix(y, rows, d, dtype, device, "y")
    if h is not None:
        a.d_h, a.ld_h = _matrix(h, rows, d, dtype, device, "h")
    if n is not None:
        a.d_n, a.ld_n = _matrix(n, rows, d, dtype, device, "n")
    if stats is not None:
        a.d_stats = _vector(stats, 4 * rows, _FLOAT, device, "stats")
    _call(lib.nmt_op_gated_norm_fwd, device, stream, a)


def nmt_debug_gated_norm_grid(rows, d, dtype):
    """(work-groups, threads of each) of nmt_op_gated_norm_fwd's launch."""
    lib, groups, threads = _lib or load(), C.c_int64(), C.c_int32()
    _check(lib.nmt_debug_gated_norm_grid(rows, d, _type_code(dtype, "nmt_debug_gated_norm_grid"), C.byref(groups), C.byref(threads)))
    return groups.value, threads.value


def nmt_op_gated_norm_bwd_scratch(rows, d, rows_per_gate=None):
    _sizes("nmt_op_gated_norm_bwd_scratch", rows, d, rows_per_gate or 0)
    n = load().nmt_op_gated_norm_bwd_scratch(rows, d, rows_per_gate or max(rows, 1))
    if n < 0:
        _refuse(f"nmt_op_gated_norm_bwd_scratch: {rows} rows of {d}, {rows_per_gate} to a gate")
    return n


def nmt_op_gated_norm_bwd(dh, dn, y, h, stats, dx, dy, scratch, post=None, gate=None, pre=None, dpost=None, dgate=None, dpre=None, kind="layer",
                          rows_per_gate=None, resid_scale=1.0, stream=None):
    """Gradients of nmt_op_gated_norm_fwd (h: its x where there is no y, and resid_scale what the caller made that x with, if anything).  dpost, dpre: (of the gain, of the shift or None) or None."""
    lib = _lib or load()
    rows, d, dtype, device = _rows_of(dx, "nmt_op_gated_norm_bwd", "dx")
    a, g = nmt_gated_norm(), nmt_gated_norm_grad()
    _norm_parts(a, rows, d, dtype, device, post, gate, pre, kind, rows_per_gate, resid_scale, "nmt_op_gated_norm_bwd")
    g.d_dx, g.ld_dx = _matrix(dx, rows, d, dtype, device, "dx")
    if y is not None:
        a.d_y, a.ld_y = _matrix(y, rows, d, dtype, device, "y")
    if h is not None:
        a.d_h, a.ld_h = _matrix(h, rows, d, dtype, device, "h")
    if dh is not None:
        g.d_dh, g.ld_dh = _matrix(dh, rows, d, dtype, device, "dh")
    if dn is not None:
        g.d_dn, g.ld_dn = _matrix(dn, rows, d, dtype, device, "dn")
    if dy is not None:
        g.d_dy, g.ld_dy = _matrix(dy, rows, d, dtype, device, "dy")
    if stats is not None:
        a.d_stats = _vector(stats, 4 * rows, _FLOAT, device, "stats")
    if dpost is not None:
        gain, shift = dpost
        if gain is not None:
            g.d_dpost_gain = _vector(gain, d, dtype, device, "the gradient of the gain after the block")
        if shift is not None:
            g.d_dpost_shift = _vector(shift, d, dtype, device, "the gradient of the shift after the block")
    if dgate is not None:
        g.d_dgate = _vector(dgate, 0 if gate is None else gate.numel(), dtype, device, "the gate's gradient")
    if dpre is not None:
        gain, shift = dpre
        if gain is not None:
            g.d_dpre_gain = _vector(gain, d, dtype, device, "the gradient of the gain before the next block")
        if shift is not None:
            g.d_dpre_shift = _vector(shift, d, dtype, device, "the gradient of the shift before the next block")
    if scratch is not None:
        g.scratch_floats = scratch.numel()
        g.d_scratch = _vector(scratch, g.scratch_floats, _FLOAT, device, "scratch")
    _call(lib.nmt_op_gated_norm_bwd, device, stream, a, g)


def nmt_op_expert_dispatch_scratch(tokens, k, experts):
    _sizes("nmt_op_expert_dispatch_scratch", tokens, k, experts)
    n = load().nmt_op_expert_dispatch_scratch(tokens, k, experts)
    if n < 0:
        _check(int(n))
    return n


def _lists(t, who, what):
    if t is None or t.dim() != 2 or t.dtype is not _INT or not t.is_contiguous():
        _refuse(f"{who}: {what} is a contiguous [tokens, k] tensor of int32")
    tokens, k = t.shape
    if tokens > _MOST or k > _MOST:
        _refuse(f"{who}: {what} is {tuple(t.shape)}: sizes are of 32 bits")
    return tokens, k, t.get_device()


def _sizes(who, *sizes):
    for n in sizes:
        if not 0 <= n <= _MOST:
            _refuse(f"{who}: {n} is no size of 32 bits")


def nmt_op_expert_dispatch(expert, experts, capacity, x, rows, slot, ranges, scratch, stream=None):
    """expert [tokens, k] int32; x [tokens, d], rows: [experts * capacity, d], or [tokens * k, d] without a capacity (both None: the lists alone);
    slot [tokens, k], ranges [experts, 2] int32; scratch: int32."""
    lib = _lib or load()
    who = "nmt_op_expert_dispatch"
    tokens, k, device = _lists(expert, who, "expert")
    _sizes(who, experts, capacity)
    d = code = ld_x = ld_rows = 0
    x_ = rows_ = scratch_ = None
    if x is not None and rows is not None:
        _, d, dtype, _ = _rows_of(x, who, "x")
        code = _type_code(dtype, who)
        x_, ld_x = _matrix(x, tokens, d, dtype, device, "x")
        rows_, ld_rows = _matrix(rows, experts * capacity if capacity else tokens * k, d, dtype, device, "rows")
    elif x is not rows:
        _refuse(f"{who}: tokens and the experts' rows belong together")
    held = 0 if scratch is None else scratch.numel()
    if held:
        scratch_ = _vector(scratch, held, _INT, device, "scratch")
    _call(lib.nmt_op_expert_dispatch, device, stream, expert.data_ptr(), tokens, k, experts, capacity, x_, ld_x, d, code, rows_, ld_rows,
          _vector(slot, tokens * k, _INT, device, "slot"), _vector(ranges, 2 * experts, _INT, device, "ranges"), scratch_, held)


def nmt_op_expert_combine(rows, slot, weights, out, add=None, stream=None):
    """out[t] = add[t] + sum over j of weights[t, j] * rows[slot[t, j]]; weights fp32 [tokens, k] or None (1)."""
    lib, who = _lib or load(), "nmt_op_expert_combine"
    tokens, k, device = _lists(slot, who, "slot")
    n, d, dtype, _ = _rows_of(rows, who, "rows")
    rows_, ld_rows = _matrix(rows, n, d, dtype, device, "rows")
    out_, ld_out = _matrix(out, tokens, d, dtype, device, "out")
    add_, ld_add = (None, 0) if add is None else _matrix(add, tokens, d, dtype, device, "add")
    _call(lib.nmt_op_expert_combine, device, stream, rows_, ld_rows, n, slot.data_ptr(),
          None if weights is None else _vector(weights, tokens * k, _FLOAT, device, "weights"), add_, ld_add, out_, ld_out, tokens, k, d,
          _type_code(dtype, who))


def nmt_op_expert_combine_bwd(dout, rows, slot, weights, drows, dweights, ranges=None, capacity=0, stream=None):
    """drows[slot[t, j]] = weights[t, j] * dout[t], dweights[t, j] = <dout[t], rows[slot[t, j]]>; rows and dweights may both be None."""
    lib, who = _lib or load(), "nmt_op_expert_combine_bwd"
    tokens, k, device = _lists(slot, who, "slot")
    n, d, dtype, _ = _rows_of(drows, who, "drows")
    _sizes(who, capacity)
    drows_, ld_drows = _matrix(drows, n, d, dtype, device, "drows")
    dout_, ld_dout = _matrix(dout, tokens, d, dtype, device, "dout")
    rows_, ld_rows = (None, 0) if rows is None else _matrix(rows, n, d, dtype, device, "rows")
    experts, ranges_ = 1, None
    if ranges is not None:
        experts = ranges.shape[0]
        ranges_ = _vector(ranges, 2 * experts, _INT, device, "ranges")
    elif capacity:
        _refuse(f"{who}: a capacity needs the experts' ranges")
    _call(lib.nmt_op_expert_combine_bwd, device, stream, dout_, ld_dout, rows_, ld_rows, n, slot.data_ptr(),
          None if weights is None else _vector(weights, tokens * k, _FLOAT, device, "weights"), drows_, ld_drows,
          None if dweights is None else _vector(dweights, tokens * k, _FLOAT, device, "dweights"), ranges_, experts, capacity, tokens, k, d,
          _type_code(dtype, who))


def _adamw_tensors(tensors, who):
    """tensors: list of dict(master, m, v, grad, weights or None, m_scale, v_scale (8-bit states: else None), weight_decay, lr_factor).  Returns the C
    array, the bits of a state and the types of gradients and weights."""
    import torch
    arr = (nmt_adamw_tensor * len(tensors))()
    bits, grad_type, weights_type = 32, None, None
    for i, (a, t) in enumerate(zip(arr, tensors)):
        master, m, v, grad, weights = t["master"], t["m"], t["v"], t["grad"], t.get("weights")
        n = master.numel()
        e8 = m.dtype is torch.float8_e4m3fn
        if i == 0:
            bits = 8 if e8 else 32
        if e8 != (bits == 8):
            _refuse(f"{who}: states of 8 and of 32 bits in one list")
        state = torch.float8_e4m3fn if e8 else torch.float32
        if grad_type is None:
            grad_type = grad.dtype
        if weights is not None and weights_type is None:
            weights_type = weights.dtype
        device = master.get_device()
        vec = lambda x, size, dtype, what: None if x is None else _vector(x, size, dtype, device, f"{what} of tensor {i}")
        blocks = -(-n // 256) if e8 else 0
        a.n, a.weight_decay, a.lr_factor = n, t.get("weight_decay", 0.0), t.get("lr_factor", 1.0)
        a.d_master, a.d_m, a.d_v = vec(master, n, torch.float32, "master"), vec(m, n, state, "m"), vec(v, n, state, "v")
        a.d_grad, a.d_weights = vec(grad, n, grad_type, "grad"), vec(weights, n, weights_type, "weights")
        if e8:
            a.d_m_scale = vec(t.get("m_scale"), blocks, torch.float32, "m_scale")
            a.d_v_scale = vec(t.get("v_scale"), blocks, torch.float32, "v_scale")
        if device != tensors[0]["master"].get_device():
            _refuse(f"{who}: tensors on several devices")
    return arr, bits, grad_type or torch.float32, weights_type or torch.float32


def nmt_adamw_table_bytes(tensors):
    arr = (nmt_adamw_tensor * len(tensors))()
    for a, t in zip(arr, tensors):
        a.n = t["master"].numel()
    n = load().nmt_adamw_table_bytes(len(tensors), arr)
    if n < 0:
        _check(int(n))
    return n


class AdamwPlan:
    """The handle of nmt_adamw_create; keeps the tensors it was made for."""

    def __init__(self, handle, device, keep):
        self.handle, self.device, self.keep = handle, device, keep


def nmt_adamw_create(tensors, table, stream=None):
    """tensors: list of dict(master=, m=, v=, grad=, weights= or None, weight_decay=, lr_factor=) of tensors of equal sizes, master fp32; m and v fp32, or
    float8_e4m3fn with m_scale= and v_scale= (fp32, one element per 256).  table: uint8 tensor of nmt_adamw_table_bytes(tensors) bytes."""
    lib, who = _lib or load(), "nmt_adamw_create"
    arr, bits, grad_type, weights_type = _adamw_tensors(tensors, who)
    out = C.c_void_p()
    device = (tensors[0]["master"] if tensors else table).get_device()
    size = table.numel() * table.element_size()
    _call(lib.nmt_adamw_create, device, stream, len(tensors), arr, bits, _type_code(grad_type, who), _type_code(weights_type, who),
          _vector(table, table.numel(), table.dtype, device, "the table"), size, out=out)
    return AdamwPlan(out, device, ([dict(t) for t in tensors], table))


def nmt_adamw_destroy(plan):
    if plan.handle is not None:
        load().nmt_adamw_destroy(plan.handle)
        plan.handle = plan.keep = None


def nmt_adamw_step(plan, lr, beta1, beta2, eps, t, grad_scale=1.0, flag=None, stream=None):
    if plan.handle is None:
        _refuse("nmt_adamw_step: the plan has been given back")
    _call(_lib.nmt_adamw_step, plan.device, stream, plan.handle, lr, beta1, beta2, eps, t, grad_scale,
          None if flag is None else _vector(flag, 1, _INT, plan.device, "flag"))


# ---- matrices held in 8 bits -----------------------------------------------------------------------
# Codes are float8_e4m3fn [rows, d], scales fp32 [blocks of 128 columns, rows], or [blocks of columns, blocks of 128 rows] where 128 x 128 elements share one.
NMT_ACT_RELU, NMT_ACT_SILU_GATE = 0, 1
_ACTS = {"relu": NMT_ACT_RELU, "silu_gate": NMT_ACT_SILU_GATE}


def nmt_op_quantize8(x, codes=None, scales=None, codes_t=None, scales_t=None, square=False, stream=None):
    """x [rows, d] into codes [rows, d] with scales [ceil(d / 128), rows], and into codes_t [d, rows] with scales_t [ceil(rows / 128), d], its transpose; either pair may be None.
    square: scales [ceil(d / 128), ceil(rows / 128)], and transposed."""
    lib, who = _lib or load(), "nmt_op_quantize8"
    rows, d, dtype, device = _rows_of(x, who, "x")
    x_, ld_x = _matrix(x, rows, d, dtype, device, "x")
    down, across = -(-rows // 128), -(-d // 128)
    codes_ = scales_ = codes_t_ = scales_t_ = None
    ld_codes = ld_scales = ld_codes_t = ld_scales_t = 0
    if codes is not None:
        codes_, ld_codes = _matrix(codes, rows, d, _E4M3, device, "codes")
    if scales is not None:
        scales_, ld_scales = _matrix(scales, across, down if square else rows, _FLOAT, device, "scales")
    if codes_t is not None:
        codes_t_, ld_codes_t = _matrix(codes_t, d, rows, _E4M3, device, "codes_t")
    if scales_t is not None:
        scales_t_, ld_scales_t = _matrix(scales_t, down, across if square else d, _FLOAT, device, "scales_t")
    _call(lib.nmt_op_quantize8, device, stream, x_, ld_x, rows, d, _type_code(dtype, who), 1 if square else 0, codes_, ld_codes, scales_, ld_scales,
          codes_t_, ld_codes_t, scales_t_, ld_scales_t)


# The structs of these calls as bytes, in one go: field by field they cost 2 us more.
_NORM8, _GEMM8, _LAYER8 = struct.Struct("4i2f6q9Q"), struct.Struct("7i13q9Qq"), struct.Struct("7i11q10Qq")
for _s, _c in ((_NORM8, nmt_norm8), (_GEMM8, nmt_gemm8), (_LAYER8, nmt_expert_layer8)):
    assert _s.size == C.sizeof(_c), _c


def nmt_op_norm8(x, y, h, codes, scales, gain, shift=None, n=None, stats=None, kind="rms", resid_scale=1.0, eps=1e-5, stream=None):
    """h = resid_scale * x + y, n = norm(h) * gain + shift in 8 bits: codes [rows, d], scales [ceil(d / 128), rows]; n itself as well if a tensor is given.  y None: h is x, and
    h None."""
    lib, who = _lib or load(), "nmt_op_norm8"
    rows, d, dtype, device = _rows_of(x, who, "x")
    if kind not in _KINDS:
        _refuse(f"{who}: kind {kind!r}: 'layer' or 'rms'")
    if not (abs(resid_scale) < 3.4e38 and abs(eps) < 3.4e38):
        _refuse(f"{who}: resid_scale {resid_scale} and eps {eps} are numbers of 32 bits")
    x_, ld_x = _matrix(x, rows, d, dtype, device, "x")
    y_, ld_y = (0, 0) if y is None else _matrix(y, rows, d, dtype, device, "y")
    h_, ld_h = (0, 0) if h is None else _matrix(h, rows, d, dtype, device, "h")
    n_, ld_n = (0, 0) if n is None else _matrix(n, rows, d, dtype, device, "n")
    codes_, ld_codes = _matrix(codes, rows, d, _E4M3, device, "codes")
    scales_, ld_scales = _matrix(scales, -(-d // 128), rows, _FLOAT, device, "scales")
    _call(lib.nmt_op_norm8, device, stream,
          _NORM8.pack(rows, d, _type_code(dtype, who), _KINDS[kind], eps, resid_scale, ld_x, ld_y, ld_h, ld_n, ld_codes, ld_scales, x_, y_,
                      _vector(gain, d, dtype, device, "the gain"), 0 if shift is None else _vector(shift, d, dtype, device, "the shift"), h_, n_, codes_, scales_,
                      0 if stats is None else _vector(stats, 4 * rows, _FLOAT, device, "stats")))


def _stack(t, batch, rows, d, dtype, device, what):
    """(address, distance between rows, distance between matrices) of a [rows, d] tensor, or of a [batch, rows, d] one."""
    strides, shape = t.stride(), t.shape
    if batch == 1 and shape == (rows, d) and strides[1] == 1 and strides[0] >= d and rows > 1 and t.dtype is dtype and t.get_device() == device:
        return t.data_ptr(), strides[0], 0
    if t.dtype is dtype and t.get_device() == device and (shape == (batch, rows, d) or (batch == 1 and shape == (rows, d))):
        ld, step = strides[-2:]
        if rows <= 1:
            ld = d
        stride = strides[0] if batch > 1 else 0
        if (step == 1 or d <= 1) and ld >= d and stride >= 0:
            return t.data_ptr(), ld, stride
        _refuse(f"{what} has strides {strides}: rows whose elements lie side by side and that do not overlap are taken")
    _refuse(f"{what} is {tuple(shape)} {t.dtype} on {t.device}, not ({batch}, {rows}, {d}) {dtype} on device {device}")


def _scale_lines(scales, rows, what):
    """Whether these are the scales of 128 x 128 elements each, and how many lie side by side."""
    shape = scales.shape
    lines = shape[-1] if len(shape) in (2, 3) else -1
    if lines == rows:
        return 0, rows
    if lines != -(-rows // 128):
        _refuse(f"{what} are {tuple(scales.shape)}: a column for each of {rows} rows, or for each 128 of them")
    return 1, lines


def nmt_op_gemm8_scratch(M, N, K, batch=1, ranges=False):
    _sizes("nmt_op_gemm8_scratch", M, N, K, batch)
    n = load().nmt_op_gemm8_scratch(M, N, K, batch, 1 if ranges else 0)
    if n < 0:
        _check(int(n))
    return n


def nmt_debug_gemm8_form(M, N, K, dtype, batch=1, ranges=False, b_square=True):
    """(edge of the tiles, pieces along k) of such a call of nmt_op_gemm8."""
    lib, tile, splits = _lib or load(), C.c_int32(), C.c_int32()
    _check(lib.nmt_debug_gemm8_form(M, N, K, batch, 1 if ranges else 0, _type_code(dtype, "nmt_debug_gemm8_form"), 1 if b_square else 0, C.byref(tile), C.byref(splits)))
    return tile.value, splits.value


def nmt_op_gemm8(a, a_scales, b, b_scales, c, bias=None, add=None, ranges=None, scratch=None, stream=None):
    """c = a b^T + bias + add: a [M, K] and b [N, K] in 8 bits, c and add [M, N], bias [N]; or a, b, c, add and their scales with a dimension of products in front (bias then [batch, N]).
    ranges [experts, 2]: a, c and add are [M, .], expert e's rows those of its range, b [experts, N, K] and bias [experts, N]."""
    lib, who = _lib or load(), "nmt_op_gemm8"
    if c is None or a is None or b is None:
        _refuse(f"{who}: a, b and c are tensors of two or three dimensions")
    c_shape, a_shape = c.shape, a.shape
    if len(c_shape) not in (2, 3) or len(a_shape) not in (2, 3):
        _refuse(f"{who}: a, b and c are tensors of two or three dimensions")
    device, dtype = c.get_device(), c.dtype
    *many, M, N = c_shape
    K = a_shape[-1]
    batch = own = many[0] if many else 1        # (own: products that have an a and a c of their own)
    ranges_ = add_ = bias_ = scratch_ = ld_add = stride_add = stride_bias = held = 0
    if ranges is not None:
        if many or len(a_shape) == 3:
            _refuse(f"{who}: experts' rows lie in one matrix")
        batch = b.shape[0] if b.dim() == 3 else 1
        ranges_ = _vector(ranges, 2 * batch, _INT, device, "ranges")
    if M > _MOST or N > _MOST or K > _MOST or batch > _MOST:
        _sizes(who, M, N, K, batch)
    a_, lda, stride_a = _stack(a, own, M, K, _E4M3, device, "a")
    b_, ldb, stride_b = _stack(b, batch, N, K, _E4M3, device, "b")
    c_, ldc, stride_c = _stack(c, own, M, N, dtype, device, "c")
    if M <= 1:
        lda = -(-K // 16) * 16
    if N <= 1:
        ldb = -(-K // 16) * 16
    a_square, a_lines = _scale_lines(a_scales, M, "a's scales")
    b_square, b_lines = _scale_lines(b_scales, N, "b's scales")
    blocks = -(-K // 128)
    sa_, ld_sa, stride_sa = _stack(a_scales, own, blocks, a_lines, _FLOAT, device, "a's scales")
    sb_, ld_sb, stride_sb = _stack(b_scales, batch, blocks, b_lines, _FLOAT, device, "b's scales")
    if add is not None:
        add_, ld_add, stride_add = _stack(add, own, M, N, dtype, device, "add")
    if bias is not None:
        if batch == 1 and bias.dim() == 1:
            bias_ = _vector(bias, N, dtype, device, "bias")
        else:
            bias_, _, stride_bias = _stack(bias.unsqueeze(-2), batch, 1, N, dtype, device, "bias")
    if scratch is not None:
        held = scratch.numel()
        scratch_ = _vector(scratch, held, _FLOAT, device, "scratch")
    _call(lib.nmt_op_gemm8, device, stream,
          _GEMM8.pack(M, N, K, batch, _type_code(dtype, who), a_square, b_square, lda, ldb, ldc, ld_add, ld_sa, ld_sb, stride_a, stride_b, stride_c, stride_add,
                      stride_bias, stride_sa, stride_sb, a_, b_, sa_, sb_, bias_, add_, c_, ranges_, scratch_, held))


def nmt_op_expert_layer8_scratch(tokens, k, experts, d, ff):
    _sizes("nmt_op_expert_layer8_scratch", tokens, k, experts, d, ff)
    n = load().nmt_op_expert_layer8_scratch(tokens, k, experts, d, ff)
    if n < 0:
        _check(int(n))
    return n


def nmt_op_expert_layer8(x, expert, weights, up, up_scales, down, down_scales, out, scratch, add=None, act="relu", stream=None):
    """out[t] = add[t] + sum over j of weights[t, j] * down[e] act(up[e] x[t]), e = expert[t, j]: x, out, add [tokens, d], expert int32 and weights fp32 (or None: 1) [tokens, k], up [experts,
    ff, d] (act "silu_gate": [experts, 2 ff, d]) and down [experts, d, ff] in 8 bits with scales of 128 x 128."""
    lib, who = _lib or load(), "nmt_op_expert_layer8"
    tokens, d, dtype, device = _rows_of(x, who, "x")
    n, k, _ = _lists(expert, who, "expert")
    if act not in _ACTS:
        _refuse(f"{who}: act {act!r}: 'relu' or 'silu_gate'")
    if n != tokens or down is None or down.dim() != 3 or up is None or up.dim() != 3:
        _refuse(f"{who}: experts of {n} tokens of {tokens}, up and down of three dimensions")
    experts, _, ff = down.shape
    _sizes(who, experts, ff)
    wide = 2 * ff if act == "silu_gate" else ff
    x_, ld_x = _matrix(x, tokens, d, dtype, device, "x")
    out_, ld_out = _matrix(out, tokens, d, dtype, device, "out")
    add_, ld_add = (0, 0) if add is None else _matrix(add, tokens, d, dtype, device, "add")
    up_, ld_up, stride_up = _stack(up, experts, wide, d, _E4M3, device, "up")
    down_, ld_down, stride_down = _stack(down, experts, d, ff, _E4M3, device, "down")
    if wide <= 1:
        ld_up = -(-d // 16) * 16
    if d <= 1:
        ld_down = -(-ff // 16) * 16
    us_, ld_us, stride_us = _stack(up_scales, experts, -(-d // 128), -(-wide // 128), _FLOAT, device, "up's scales")
    ds_, ld_ds, stride_ds = _stack(down_scales, experts, -(-ff // 128), -(-d // 128), _FLOAT, device, "down's scales")
    scratch_ = held = 0
    if scratch is not None:
        held = scratch.numel()
        scratch_ = _vector(scratch, held, _FLOAT, device, "scratch")
    _call(lib.nmt_op_expert_layer8, device, stream,
          _LAYER8.pack(tokens, k, experts, d, ff, _type_code(dtype, who), _ACTS[act], ld_x, ld_add, ld_out, ld_up, stride_up, ld_us, stride_us, ld_down, stride_down,
                       ld_ds, stride_ds, x_, _vector(expert, tokens * k, _INT, device, "expert"),
                       0 if weights is None else _vector(weights, tokens * k, _FLOAT, device, "weights"), up_, us_, down_, ds_, add_, out_, scratch_, held))
