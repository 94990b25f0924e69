"""ctypes binding of libnmt.so: one Python function per C entry point, same names, argument
marshalling only.  Device buffers are torch tensors (their data_ptr() is passed through); the HIP
stream is torch's current stream unless one is given.  The library must have been built
(`python -m paper_1806_00187_amd.build`); there is no fallback of any kind."""
from __future__ import annotations

import ctypes as C
import os

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
    "nmt_op_gated_norm_bwd_scratch": (_I64, [_I32, _I32, _I32]),
    "nmt_op_gated_norm_bwd": (C.c_int, [C.POINTER(nmt_gated_norm), C.POINTER(nmt_gated_norm_grad), _P]),
    "nmt_op_expert_dispatch_scratch": (_I64, [_I32, _I32, _I32]),
    "nmt_op_expert_dispatch": (C.c_int, [_P, _I32, _I32, _I32, _I32, _P, _I64, _I32, _I32, _P, _I64, _P, _P, _P, _P]),
    "nmt_op_expert_combine": (C.c_int, [_P, _I64, _I32, _P, _P, _P, _I64, _P, _I64, _I32, _I32, _I32, _I32, _P]),
    "nmt_op_expert_combine_bwd": (C.c_int, [_P, _I64, _P, _I64, _I32, _P, _P, _P, _I64, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32, _P]),
    "nmt_adamw_table_bytes": (_I64, [_I32, C.POINTER(nmt_adamw_tensor)]),
    "nmt_adamw_create": (C.c_int, [_I32, C.POINTER(nmt_adamw_tensor), _I32, _I32, _I32, _P, _I64, _P, C.POINTER(_P)]),
    "nmt_adamw_destroy": (None, [_P]),
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
# to the stream of the tensors' device.
NMT_F16, NMT_BF16, NMT_F32 = 0, 1, 2
NMT_NORM_LAYER, NMT_NORM_RMS = 0, 1
_KINDS = {"layer": NMT_NORM_LAYER, "rms": NMT_NORM_RMS}


def _refuse(msg):
    raise NmtError(NMT_EINVAL, msg)


def _type_code(dtype, who):
    import torch
    if dtype is torch.float16:
        return NMT_F16
    if dtype is torch.bfloat16:
        return NMT_BF16
    if dtype is torch.float32:
        return NMT_F32
    _refuse(f"{who}: rows of {dtype}: float16, bfloat16 or float32")


def _matrix(t, rows, d, like, who, what):
    """(address, distance between rows) of a [rows, d] tensor of the type and device of `like`; (None, 0) of None."""
    if t is None:
        return None, 0
    if t.dtype is not like.dtype or t.device != like.device or t.dim() != 2 or t.shape[0] != rows or t.shape[1] != d:
        _refuse(f"{who}: {what} is {tuple(t.shape)} {t.dtype} on {t.device}, not ({rows}, {d}) {like.dtype} on {like.device}")
    ld, step = t.stride()
    if (step != 1 and d > 1) or (ld < d and rows > 1):
        _refuse(f"{who}: {what} has strides {(ld, step)}: rows whose elements lie side by side and that do not overlap are taken")
    return t.data_ptr(), (ld if rows > 1 else d)


def _vector(t, n, dtype, like, who, what):
    """Address of a contiguous tensor of n elements, or None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != like.device or t.numel() != n or not t.is_contiguous():
        _refuse(f"{who}: {what} is {tuple(t.shape)} {t.dtype} on {t.device}, not {n} contiguous elements of {dtype} on {like.device}")
    return t.data_ptr()


def _on(like, stream, call, *args):
    """call(*args, stream) with the device of `like` as the current one."""
    import torch
    device = like.device
    if device.type != "cuda":
        _refuse(f"the tensors are on {device}")
    if stream is None:
        stream = torch.cuda.current_stream(device).cuda_stream
    if device.index == torch.cuda.current_device():
        _check(call(*args, stream))
    else:
        with torch.cuda.device(device):
            _check(call(*args, stream))


def _pair(p):
    return (None, None) if p is None else p


def _gated_norm(who, first, x, y, h, n, stats, post, gate, pre, kind, rows_per_gate, resid_scale, eps):
    if first is None or first.dim() != 2:
        _refuse(f"{who}: the rows are [rows, d] tensors")
    rows, d = first.shape
    T = first.dtype
    if kind not in _KINDS:
        _refuse(f"{who}: kind {kind!r}: 'layer' or 'rms'")
    gates = 0
    if gate is not None:
        rows_per_gate = rows_per_gate or max(rows, 1)
        if rows_per_gate < 1:
            _refuse(f"{who}: rows_per_gate must be at least 1")
        gates = 1 if rows_per_gate >= rows else -(-rows // rows_per_gate)
    x_, ld_x = _matrix(x, rows, d, first, who, "x")
    y_, ld_y = _matrix(y, rows, d, first, who, "y")
    h_, ld_h = _matrix(h, rows, d, first, who, "h")
    n_, ld_n = _matrix(n, rows, d, first, who, "n")
    post_gain, post_shift = _pair(post)
    pre_gain, pre_shift = _pair(pre)
    import torch
    return nmt_gated_norm(rows, d, _type_code(T, who), _KINDS[kind], eps, resid_scale, min(rows_per_gate or 1, 2 ** 31 - 1), ld_x, ld_y, ld_h, ld_n,
                          x_, y_, _vector(post_gain, d, T, first, who, "the gain after the block"),
                          _vector(post_shift, d, T, first, who, "the shift after the block"), _vector(gate, gates * d, T, first, who, "the gate"),
                          _vector(pre_gain, d, T, first, who, "the gain before the next block"),
                          _vector(pre_shift, d, T, first, who, "the shift before the next block"), h_, n_,
                          _vector(stats, 4 * rows, torch.float32, first, who, "stats"))


def nmt_op_gated_norm_fwd(x, y, h, n, stats=None, post=None, gate=None, pre=None, kind="layer", rows_per_gate=None, resid_scale=1.0, eps=1e-5,
                          stream=None):
    """h = resid_scale * x + gate * post(y), n = pre(h).  post, pre: (gain, shift or None) or None; rows_per_gate None: one gate for all rows."""
    a = _gated_norm("nmt_op_gated_norm_fwd", x, x, y, h, n, stats, post, gate, pre, kind, rows_per_gate, resid_scale, eps)
    _on(x, stream, load().nmt_op_gated_norm_fwd, C.byref(a))


def nmt_op_gated_norm_bwd_scratch(rows, d, rows_per_gate=None):
    n = load().nmt_op_gated_norm_bwd_scratch(rows, d, rows_per_gate or max(rows, 1))
    if n < 0:
        _refuse(f"nmt_op_gated_norm_bwd_scratch: {rows} rows of {d}, {rows_per_gate} to a gate")
    return n


def nmt_op_gated_norm_bwd(dh, dn, y, h, stats, dx, dy, scratch, post=None, gate=None, pre=None, dpost=None, dgate=None, dpre=None, kind="layer",
                          rows_per_gate=None, resid_scale=1.0, stream=None):
    """Gradients of nmt_op_gated_norm_fwd (h: its x where there is no y).  dpost, dpre: (of the gain, of the shift or None) or None."""
    import torch
    who = "nmt_op_gated_norm_bwd"
    a = _gated_norm(who, dx, None, y, h, None, stats, post, gate, pre, kind, rows_per_gate, resid_scale, 1.0)
    rows, d, T = a.rows, a.d, dx.dtype
    (dh_, ld_dh), (dn_, ld_dn) = _matrix(dh, rows, d, dx, who, "dh"), _matrix(dn, rows, d, dx, who, "dn")
    (dx_, ld_dx), (dy_, ld_dy) = _matrix(dx, rows, d, dx, who, "dx"), _matrix(dy, rows, d, dx, who, "dy")
    dpost_gain, dpost_shift = _pair(dpost)
    dpre_gain, dpre_shift = _pair(dpre)
    vec = lambda t, what: _vector(t, d, T, dx, who, what)
    g = nmt_gated_norm_grad(ld_dh, ld_dn, ld_dx, ld_dy, dh_, dn_, dx_, dy_, vec(dpost_gain, "the gradient of the gain after the block"),
                            vec(dpost_shift, "the gradient of the shift after the block"),
                            _vector(dgate, 0 if gate is None else gate.numel(), T, dx, who, "the gate's gradient"),
                            vec(dpre_gain, "the gradient of the gain before the next block"),
                            vec(dpre_shift, "the gradient of the shift before the next block"),
                            None if scratch is None else _vector(scratch, scratch.numel(), torch.float32, dx, who, "scratch"),
                            0 if scratch is None else scratch.numel())
    _on(dx, stream, load().nmt_op_gated_norm_bwd, C.byref(a), C.byref(g))


def nmt_op_expert_dispatch_scratch(tokens, k, experts):
    n = load().nmt_op_expert_dispatch_scratch(tokens, k, experts)
    if n < 0:
        _check(int(n))
    return n


def _lists(t, who, what):
    import torch
    if t is None or t.dim() != 2 or t.dtype is not torch.int32 or not t.is_contiguous():
        _refuse(f"{who}: {what} is a contiguous [tokens, k] tensor of int32")
    return t.shape


def nmt_op_expert_dispatch(expert, experts, capacity, x, rows, slot, ranges, scratch, stream=None):
    """expert [tokens, k] int32; x [tokens, d], rows: [experts * capacity, d], or [tokens * k, d] without a capacity (both None: the lists alone);
    slot [tokens, k], ranges [experts, 2] int32."""
    import torch
    who = "nmt_op_expert_dispatch"
    tokens, k = _lists(expert, who, "expert")
    type_ = d = ld_x = ld_rows = 0
    x_ = rows_ = None
    if (x is None) != (rows is None):
        _refuse(f"{who}: tokens and the experts' rows belong together")
    if x is not None:
        if x.dim() != 2:
            _refuse(f"{who}: x is [tokens, d]")
        d, type_ = x.shape[1], _type_code(x.dtype, who)
        x_, ld_x = _matrix(x, tokens, d, x, who, "x")
        rows_, ld_rows = _matrix(rows, experts * capacity if capacity else tokens * k, d, x, who, "rows")
    I = torch.int32
    need = nmt_op_expert_dispatch_scratch(tokens, k, experts)
    if need and (scratch is None or scratch.numel() < need):
        raise NmtError(NMT_ENOMEM, f"{who}: scratch of {0 if scratch is None else scratch.numel()} elements, {need} needed")
    if x is not None and x.device != expert.device:
        _refuse(f"{who}: expert is on {expert.device}, x on {x.device}")
    _on(expert, stream, load().nmt_op_expert_dispatch, expert.data_ptr(), tokens, k, experts, capacity, x_, ld_x, d, type_, rows_, ld_rows,
        _vector(slot, tokens * k, I, expert, who, "slot"), _vector(ranges, 2 * experts, I, expert, who, "ranges"),
        None if scratch is None else _vector(scratch, scratch.numel(), I, expert, who, "scratch"))


def nmt_op_expert_combine(rows, slot, weights, out, add=None, stream=None):
    """out[t] = add[t] + sum over j of weights[t, j] * rows[slot[t, j]]; weights fp32 [tokens, k] or None (1)."""
    import torch
    who = "nmt_op_expert_combine"
    tokens, k = _lists(slot, who, "slot")
    if rows is None or rows.dim() != 2:
        _refuse(f"{who}: rows is [rows, d]")
    n, d = rows.shape
    (rows_, ld_rows), (out_, ld_out), (add_, ld_add) = (_matrix(rows, n, d, rows, who, "rows"), _matrix(out, tokens, d, rows, who, "out"),
                                                        _matrix(add, tokens, d, rows, who, "add"))
    if slot.device != rows.device:
        _refuse(f"{who}: slot is on {slot.device}, rows on {rows.device}")
    _on(rows, stream, load().nmt_op_expert_combine, rows_, ld_rows, n, slot.data_ptr(),
        _vector(weights, tokens * k, torch.float32, rows, who, "weights"), add_, ld_add, out_, ld_out, tokens, k, d, _type_code(rows.dtype, who))


def nmt_op_expert_combine_bwd(dout, rows, slot, weights, drows, dweights, ranges=None, capacity=0, stream=None):
    """drows[slot[t, j]] = weights[t, j] * dout[t], dweights[t, j] = <dout[t], rows[slot[t, j]]>; rows and dweights may both be None."""
    import torch
    who = "nmt_op_expert_combine_bwd"
    tokens, k = _lists(slot, who, "slot")
    if drows is None or drows.dim() != 2:
        _refuse(f"{who}: drows is [rows, d]")
    n, d = drows.shape
    (dout_, ld_dout), (rows_, ld_rows), (drows_, ld_drows) = (_matrix(dout, tokens, d, drows, who, "dout"), _matrix(rows, n, d, drows, who, "rows"),
                                                              _matrix(drows, n, d, drows, who, "drows"))
    if slot.device != drows.device:
        _refuse(f"{who}: slot is on {slot.device}, drows on {drows.device}")
    if capacity and ranges is None:
        _refuse(f"{who}: a capacity needs the experts' ranges")
    experts = 1 if ranges is None else ranges.shape[0]
    _on(drows, stream, load().nmt_op_expert_combine_bwd, dout_, ld_dout, rows_, ld_rows, n, slot.data_ptr(),
        _vector(weights, tokens * k, torch.float32, drows, who, "weights"), drows_, ld_drows,
        _vector(dweights, tokens * k, torch.float32, drows, who, "dweights"),
        _vector(ranges, 2 * experts, torch.int32, drows, who, "ranges"), experts, capacity, tokens, k, d, _type_code(drows.dtype, who))


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
        vec = lambda x, size, dtype, what: _vector(x, size, dtype, master, who, f"{what} of tensor {i}")
        blocks = -(-n // 256) if e8 else 0
        a.n, a.weight_decay, a.lr_factor = n, t.get("weight_decay", 0.0), t.get("lr_factor", 1.0)
        a.d_master, a.d_m, a.d_v = vec(master, n, torch.float32, "master"), vec(m, n, state, "m"), vec(v, n, state, "v")
        a.d_grad, a.d_weights = vec(grad, n, grad_type, "grad"), vec(weights, n, weights_type, "weights")
        if e8:
            a.d_m_scale = vec(t.get("m_scale"), blocks, torch.float32, "m_scale")
            a.d_v_scale = vec(t.get("v_scale"), blocks, torch.float32, "v_scale")
        if master.device != tensors[0]["master"].device:
            _refuse(f"{who}: tensors on {tensors[0]['master'].device} and on {master.device}")
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
    who = "nmt_adamw_create"
    arr, bits, grad_type, weights_type = _adamw_tensors(tensors, who)
    out = C.c_void_p()
    like = tensors[0]["master"] if tensors else table
    if table.device != like.device or not table.is_contiguous():
        _refuse(f"{who}: the table is contiguous and on the tensors' device")
    _on(like, stream, lambda s: load().nmt_adamw_create(len(tensors), arr, bits, _type_code(grad_type, who), _type_code(weights_type, who), table.data_ptr(),
                                                       table.numel() * table.element_size(), s, C.byref(out)))
    return AdamwPlan(out, like, (list(tensors), table))


def nmt_adamw_destroy(plan):
    if plan.handle is not None:
        load().nmt_adamw_destroy(plan.handle)
        plan.handle = plan.keep = None


def nmt_adamw_step(plan, lr, beta1, beta2, eps, t, grad_scale=1.0, flag=None, stream=None):
    import torch
    if plan.handle is None:
        _refuse("nmt_adamw_step: the plan has been given back")
    _on(plan.device, stream, load().nmt_adamw_step, plan.handle, lr, beta1, beta2, eps, t, grad_scale,
        _vector(flag, 1, torch.int32, plan.device, "nmt_adamw_step", "flag"))
