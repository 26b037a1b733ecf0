"""ctypes binding of libmrl.so: same names as the C ABI, argument marshalling only.

Tensors are torch tensors used as device (or pinned host) memory; every step of the path runs
inside the library's CUDA kernels.  There is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

from .build import LIB_PATH

OK = 0
F32, BF16, E4M3 = 0, 1, 2
ADV_MEAN_ONLY, ADV_GROUP_ZNORM, ADV_BATCH_ZNORM = 0, 1, 2
PICK_NONE, PICK_FIRST, PICK_SHORTEST, PICK_ALL, PICK_SEEDED = 0, 1, 2, 3, 4
AGG_TOKEN_MEAN, AGG_SEQ_MEAN_TOKEN_MEAN = 0, 1
RATIO_TOKEN, RATIO_SEQUENCE = 0, 1
KL_K1, KL_K2, KL_K3 = 0, 1, 2
FLAG_ACCUMULATE_LOSS, FLAG_SKIP_ZERO_ROWS, FLAG_ACCUMULATE_DW, FLAG_PAIR_TILES = 1, 2, 4, 8
WS_TOKEN_LOGPROBS, WS_POLICY_LOSS, WS_FUSED_LMHEAD, WS_THL_WORD_ALIGN = 0, 1, 2, 3
WS_RMSNORM_BWD, WS_GRAD_NORM, WS_ADAMW, WS_DISTILL = 4, 5, 6, 7
DEV_BAD_TOKEN_ID, DEV_TIMEOUT, DEV_BAD_WORD_MAP, DEV_NONFINITE_GRAD, DEV_BAD_LIST = 1, 2, 4, 8, 16
ROUND_NEAREST, ROUND_SEEDED = 0, 1
STATE_BLOCK = 256
DISTILL_FORWARD, DISTILL_REVERSE = 0, 1
REST_EVENT, REST_NONE = 0, 1
MAX_TOP, SCALE_BLOCK = 128, 128

EXPORTS = ("mrl_group_advantages", "mrl_token_logprobs", "mrl_policy_loss_fwd_bwd",
           "mrl_fused_lmhead_loss_fwd_bwd", "mrl_workspace_bytes", "mrl_status_string", "mrl_version",
           "mrl_profile_dominant_kernel", "mrl_policy_loss_fwd_bwd_static", "mrl_thl_word_align_logprobs",
           "mrl_policy_loss_fwd_bwd_host", "mrl_host_pipeline_workspace_bytes", "mrl_profile_last_kernel",
           "mrl_rmsnorm_residual_fwd", "mrl_rmsnorm_residual_bwd", "mrl_grad_norm", "mrl_adamw_step",
           "mrl_e4m3_quantize", "mrl_e4m3_product", "mrl_top_logprobs", "mrl_distill_loss_fwd_bwd")
STATIC_MAX_ROWS, STATIC_MAX_SEQS = 65536, 65536
ERR_STATIC_SCRATCH_TOO_SMALL = 8


class AdvParams(C.Structure):
    _fields_ = [("mode", C.c_int32), ("ddof", C.c_int32), ("eps", C.c_float),
                ("sgt_success_thr", C.c_float), ("sgt_negative_thr", C.c_float),
                ("sgt_pick", C.c_int32), ("seed", C.c_uint64)]


class LossParams(C.Structure):
    _fields_ = [("eps_lo", C.c_float), ("eps_hi", C.c_float), ("agg_mode", C.c_int32),
                ("flags", C.c_uint32), ("pg_denominator", C.c_double), ("seq_denominator", C.c_double),
                ("nll_coeff", C.c_float), ("ratio_level", C.c_int32), ("entropy", C.c_void_p),
                ("logp_ref", C.c_void_p), ("kl_coeff", C.c_float), ("kl_estimator", C.c_int32),
                ("kl_loss", C.c_void_p)]


class NormParams(C.Structure):
    _fields_ = [("eps", C.c_float), ("weight_offset", C.c_float), ("group", C.c_int32), ("flags", C.c_uint32)]


class TensorSlotStruct(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("param", C.c_void_p), ("master", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("numel", C.c_int64), ("rng_first", C.c_uint64),
                ("weight_decay", C.c_float), ("grad_dtype", C.c_int32), ("param_dtype", C.c_int32),
                ("state_dtype", C.c_int32)]


class AdamwParams(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("step", C.c_int64), ("seed", C.c_uint64), ("rounding", C.c_int32), ("flags", C.c_uint32),
                ("lr_dev", C.c_void_p), ("step_dev", C.c_void_p)]


class DistillParams(C.Structure):
    _fields_ = [("temperature", C.c_float), ("coeff", C.c_float), ("direction", C.c_int32), ("rest", C.c_int32),
                ("rest_floor", C.c_float), ("flags", C.c_uint32), ("denominator", C.c_double)]


class MrlError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built (there is no other code path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2605_07244_b200.build` "
                               "(or __graft_entry__.build()) first; there is no CPU fallback")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        L.mrl_group_advantages.argtypes = [vp, vp, i32, i32, i32, i32, C.POINTER(AdvParams), vp, vp, vp, vp, vp, vp, vp]
        L.mrl_group_advantages.restype = C.c_int
        L.mrl_token_logprobs.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, vp, vp, vp, sz, vp]
        L.mrl_token_logprobs.restype = C.c_int
        L.mrl_policy_loss_fwd_bwd.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, i32, vp, vp, vp, vp,
                                              C.POINTER(LossParams), vp, i64, vp, vp, vp, vp, vp, sz, vp]
        L.mrl_policy_loss_fwd_bwd.restype = C.c_int
        L.mrl_policy_loss_fwd_bwd_static.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, i32, vp, vp, vp, vp,
                                                     C.POINTER(LossParams), vp, i64, vp, vp, vp, vp, vp]
        L.mrl_policy_loss_fwd_bwd_static.restype = C.c_int
        L.mrl_policy_loss_fwd_bwd_host.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, i32, vp, vp, vp, vp,
                                                   C.POINTER(LossParams), vp, i64, vp, vp, vp, vp, i64, vp, sz, vp]
        L.mrl_policy_loss_fwd_bwd_host.restype = C.c_int
        L.mrl_host_pipeline_workspace_bytes.argtypes = [i64, i64, i32, i32, i64]
        L.mrl_host_pipeline_workspace_bytes.restype = sz
        L.mrl_fused_lmhead_loss_fwd_bwd.argtypes = [vp, vp, i64, i32, i32, vp, vp, vp, i32, vp, vp, vp, vp,
                                                    C.POINTER(LossParams), vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.mrl_fused_lmhead_loss_fwd_bwd.restype = C.c_int
        L.mrl_thl_word_align_logprobs.argtypes = [vp, vp, vp, vp, vp, vp, i32, i64, i64, i64, C.c_float, vp, vp, vp, vp,
                                                  vp, sz, vp]
        L.mrl_thl_word_align_logprobs.restype = C.c_int
        L.mrl_rmsnorm_residual_fwd.argtypes = [vp, i64, vp, i64, i32, vp, i32, i64, i32, C.POINTER(NormParams), vp, i64,
                                               vp, i64, vp, i64, vp, vp, vp]
        L.mrl_rmsnorm_residual_fwd.restype = C.c_int
        L.mrl_rmsnorm_residual_bwd.argtypes = [vp, i64, vp, i64, vp, i64, i32, vp, i32, vp, i64, i32, C.POINTER(NormParams),
                                               vp, i64, vp, vp, sz, vp]
        L.mrl_rmsnorm_residual_bwd.restype = C.c_int
        L.mrl_grad_norm.argtypes = [vp, i32, C.c_float, vp, vp, vp, sz, vp]
        L.mrl_grad_norm.restype = C.c_int
        L.mrl_adamw_step.argtypes = [vp, i32, C.POINTER(AdamwParams), vp, vp, vp, sz, vp]
        L.mrl_adamw_step.restype = C.c_int
        L.mrl_e4m3_quantize.argtypes = [vp, i64, i32, i64, i32, i32, vp, i64, vp, vp]
        L.mrl_e4m3_quantize.restype = C.c_int
        L.mrl_e4m3_product.argtypes = [vp, i64, vp, vp, i64, vp, i64, i32, i32, i32, vp, i64, vp, vp]
        L.mrl_e4m3_product.restype = C.c_int
        L.mrl_top_logprobs.argtypes = [vp, i32, i64, i32, i64, vp, vp, C.c_float, i32, vp, vp, vp, vp, vp, vp, vp]
        L.mrl_top_logprobs.restype = C.c_int
        L.mrl_distill_loss_fwd_bwd.argtypes = [vp, i32, i64, i32, i64, vp, vp, i32, vp, vp, C.POINTER(DistillParams), vp, i64,
                                               vp, vp, vp, vp, vp, sz, vp]
        L.mrl_distill_loss_fwd_bwd.restype = C.c_int
        L.mrl_workspace_bytes.argtypes = [i32, i64, i32, i32, i32, i32]
        L.mrl_workspace_bytes.restype = sz
        L.mrl_status_string.argtypes = [C.c_int]
        L.mrl_status_string.restype = C.c_char_p
        L.mrl_profile_dominant_kernel.argtypes = [C.POINTER(vp), C.POINTER(vp), i32]
        L.mrl_profile_dominant_kernel.restype = C.c_int
        L.mrl_profile_last_kernel.argtypes = []
        L.mrl_profile_last_kernel.restype = C.c_char_p
        L.mrl_version.argtypes = []
        L.mrl_version.restype = C.c_int
        _lib = L
    return _lib


def _p(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise MrlError(3, "dtype")


def _check(code: int, where: str):
    if code != OK:
        raise MrlError(code, where)


def status_string(code: int) -> str:
    return lib().mrl_status_string(code).decode()


def version() -> int:
    return lib().mrl_version()


def workspace_bytes(which: int, N: int, V: int, H: int = 0, dtype: int = BF16, S: int = 0) -> int:
    return int(lib().mrl_workspace_bytes(which, N, V, H, dtype, S))


def mrl_group_advantages(rewards, seq_len, learner: int, ap: AdvParams, adv_own=None, adv_pool=None,
                         rescue=None, pick=None, nll_seq_weight=None, n_gated=None, stream=None):
    P, M, G = rewards.shape
    _check(lib().mrl_group_advantages(_p(rewards), _p(seq_len), P, M, G, learner, C.byref(ap), _p(adv_own),
                                      _p(adv_pool), _p(rescue), _p(pick), _p(nll_seq_weight), _p(n_gated),
                                      _stream(stream)), "mrl_group_advantages")


def mrl_token_logprobs(logits, ids, mask, logp, lse=None, status=None, workspace=None, V=None, stream=None):
    N = logits.shape[0]
    V = logits.shape[1] if V is None else V
    ld = logits.stride(0) if N > 1 else max(logits.shape[1], V)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().mrl_token_logprobs(_p(logits), _dtype_code(logits), N, V, ld, _p(ids), _p(mask), _p(logp),
                                    _p(lse), _p(status), _p(workspace), ws_bytes, _stream(stream)),
           "mrl_token_logprobs")


def mrl_policy_loss_fwd_bwd(logits, ids, mask, cu_seqlens, adv_seq, logp_old, tok_weight, nll_weight,
                            lp: LossParams, dlogits, logp, loss, stats=None, status=None, workspace=None,
                            V=None, stream=None):
    N = logits.shape[0]
    V = logits.shape[1] if V is None else V
    S = cu_seqlens.numel() - 1
    ld = logits.stride(0) if N > 1 else max(logits.shape[1], V)
    ld_out = ld if dlogits is None else (dlogits.stride(0) if N > 1 else max(dlogits.shape[1], V))
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().mrl_policy_loss_fwd_bwd(_p(logits), _dtype_code(logits), N, V, ld, _p(ids), _p(mask),
                                         _p(cu_seqlens), S, _p(adv_seq), _p(logp_old), _p(tok_weight),
                                         _p(nll_weight), C.byref(lp), _p(dlogits), ld_out, _p(logp), _p(loss),
                                         _p(stats), _p(status), _p(workspace), ws_bytes, _stream(stream)),
           "mrl_policy_loss_fwd_bwd")


def mrl_policy_loss_fwd_bwd_static(logits, ids, mask, cu_seqlens, adv_seq, logp_old, tok_weight, nll_weight,
                                   lp: LossParams, dlogits, logp, loss, stats=None, status=None, V=None,
                                   stream=None):
    """mrl_policy_loss_fwd_bwd without a workspace argument: for callers that cannot allocate device
    memory, the library's own fixed scratch array is used (N <= STATIC_MAX_ROWS, S <= STATIC_MAX_SEQS)."""
    N = logits.shape[0]
    V = logits.shape[1] if V is None else V
    S = cu_seqlens.numel() - 1
    ld = logits.stride(0) if N > 1 else max(logits.shape[1], V)
    ld_out = ld if dlogits is None else (dlogits.stride(0) if N > 1 else max(dlogits.shape[1], V))
    _check(lib().mrl_policy_loss_fwd_bwd_static(_p(logits), _dtype_code(logits), N, V, ld, _p(ids), _p(mask),
                                                _p(cu_seqlens), S, _p(adv_seq), _p(logp_old), _p(tok_weight),
                                                _p(nll_weight), C.byref(lp), _p(dlogits), ld_out, _p(logp),
                                                _p(loss), _p(stats), _p(status), _stream(stream)),
           "mrl_policy_loss_fwd_bwd_static")


def host_pipeline_workspace_bytes(N: int, ld: int, dtype: int, S: int, slab_rows: int) -> int:
    return int(lib().mrl_host_pipeline_workspace_bytes(N, ld, dtype, S, slab_rows))


def mrl_policy_loss_fwd_bwd_host(h_logits, h_ids, h_mask, h_cu_seqlens, h_adv_seq, h_logp_old, h_tok_weight,
                                 h_nll_weight, lp: LossParams, h_dlogits, h_logp, h_loss, h_stats, h_status,
                                 slab_rows: int, workspace, V=None, stream=None):
    """The logits-in pass on HOST tensors (pinned for overlap), pipelined in micro-batches of whole sequences over
    three staging buffers in `workspace` (device).  Asynchronous: synchronise `stream` before reading the outputs."""
    for t in (h_logits, h_ids, h_mask, h_cu_seqlens, h_adv_seq, h_logp_old, h_tok_weight, h_nll_weight, h_dlogits,
              h_logp, h_loss, h_stats, h_status):
        if t is not None and t.is_cuda:
            raise MrlError(1, "mrl_policy_loss_fwd_bwd_host takes host tensors")
    N = h_logits.shape[0]
    V = h_logits.shape[1] if V is None else V
    S = h_cu_seqlens.numel() - 1
    ld = h_logits.stride(0) if N > 1 else max(h_logits.shape[1], V)
    ld_out = ld if h_dlogits is None else (h_dlogits.stride(0) if N > 1 else max(h_dlogits.shape[1], V))
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().mrl_policy_loss_fwd_bwd_host(_p(h_logits), _dtype_code(h_logits), N, V, ld, _p(h_ids), _p(h_mask),
                                              _p(h_cu_seqlens), S, _p(h_adv_seq), _p(h_logp_old), _p(h_tok_weight),
                                              _p(h_nll_weight), C.byref(lp), _p(h_dlogits), ld_out, _p(h_logp),
                                              _p(h_loss), _p(h_stats), _p(h_status), int(slab_rows), _p(workspace),
                                              ws_bytes, _stream(stream)), "mrl_policy_loss_fwd_bwd_host")


def mrl_fused_lmhead_loss_fwd_bwd(hidden, W, ids, mask, cu_seqlens, adv_seq, logp_old, tok_weight, nll_weight,
                                  lp: LossParams, dHidden, dW, logp, loss, stats=None, status=None,
                                  workspace=None, stream=None):
    N, H = hidden.shape
    V = W.shape[0]
    S = cu_seqlens.numel() - 1
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().mrl_fused_lmhead_loss_fwd_bwd(_p(hidden), _p(W), N, H, V, _p(ids), _p(mask), _p(cu_seqlens), S,
                                               _p(adv_seq), _p(logp_old), _p(tok_weight), _p(nll_weight),
                                               C.byref(lp), _p(dHidden), _p(dW), _p(logp), _p(loss), _p(stats),
                                               _p(status), _p(workspace), ws_bytes, _stream(stream)),
           "mrl_fused_lmhead_loss_fwd_bwd")


def mrl_thl_word_align_logprobs(src_logp, src_word, src_cu, tgt_word, tgt_cu, word_cu, total_words, ignore_value,
                                out, src_total=None, tgt_total=None, status=None, workspace=None, stream=None):
    Bn = src_cu.numel() - 1
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().mrl_thl_word_align_logprobs(_p(src_logp), _p(src_word), _p(src_cu), _p(tgt_word), _p(tgt_cu),
                                             _p(word_cu), Bn, src_word.numel(), out.numel(), int(total_words),
                                             float(ignore_value), _p(out),
                                             _p(src_total), _p(tgt_total), _p(status), _p(workspace), ws_bytes,
                                             _stream(stream)), "mrl_thl_word_align_logprobs")


# ---- the norm before the LM head, the gradient norm and the update: the argument checks that need the tensors' shapes.
# (Written for little time per call: the smallest calls take the GPU three microseconds.)

_CODES = {torch.float32: F32, torch.bfloat16: BF16}
_CODE_TYPES = (torch.float8_e4m3fn, torch.uint8)      # how e4m3 codes may be held


def _stream_of(device: int, stream, where):
    """Handle of `stream`, or of the current stream of the tensors' device, which has to be the current device."""
    if device < 0 or device != torch.cuda.current_device():
        raise MrlError(1, f"{where}: tensors of the current device are wanted")
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _row_stride(t, shape, dtype, device, where):
    """Row stride of a tensor of [N, H] rows whose columns are adjacent; 0 for none."""
    if t is None:
        return 0
    if t.dtype is not dtype and not (dtype is None and t.dtype in _CODE_TYPES):
        raise MrlError(3, where)
    if t.shape != shape or t.get_device() != device:
        raise MrlError(1, where)
    if t.is_contiguous():
        return shape[1]
    ld, step = t.stride()
    if (shape[1] > 1 and step != 1) or (shape[0] > 1 and ld < shape[1]):
        raise MrlError(1, where)
    return ld if shape[0] > 1 else shape[1]


def _float_vector(t, n, device, where):
    """Address of a contiguous float32 tensor of n elements."""
    if t is None:
        return None
    if t.dtype is not torch.float32:
        raise MrlError(3, where)
    if t.numel() != n or t.get_device() != device or not t.is_contiguous():
        raise MrlError(1, where)
    return t.data_ptr()


def _vector(t, n, dtypes, device, where):
    """Address of a contiguous tensor of n elements of one of the types."""
    if t is None:
        return None
    if t.dtype not in dtypes:
        raise MrlError(3, where)
    if t.numel() != n or t.get_device() != device or not t.is_contiguous():
        raise MrlError(1, where)
    return t.data_ptr()


def _workspace(t, device, where):
    """Address and bytes of a workspace."""
    if t is None:
        return None, 0
    if t.get_device() != device or not t.is_contiguous():
        raise MrlError(1, where)
    return t.data_ptr(), t.nbytes


_F32_ONLY = (torch.float32,)


def mrl_rmsnorm_residual_fwd(x, residual, weight, np: NormParams, h_out=None, y=None, y8=None, scales=None, rstd=None,
                             stream=None):
    where = "mrl_rmsnorm_residual_fwd"
    shape, dtype, dev = x.shape, x.dtype, x.get_device()
    N, H = shape
    code = _CODES.get(dtype)
    if code is None:
        raise MrlError(3, where)
    st = _stream_of(dev, stream, where)
    w = _vector(weight, H, _CODES, dev, where)
    ld_x, ld_r = _row_stride(x, shape, dtype, dev, where), _row_stride(residual, shape, dtype, dev, where)
    ld_h, ld_y = _row_stride(h_out, shape, dtype, dev, where), _row_stride(y, shape, dtype, dev, where)
    ld_8 = _row_stride(y8, shape, None, dev, where)
    group = np.group
    code = lib().mrl_rmsnorm_residual_fwd(
        x.data_ptr(), ld_x, None if residual is None else residual.data_ptr(), ld_r, code, w, _CODES[weight.dtype], N, H, np,
        None if h_out is None else h_out.data_ptr(), ld_h, None if y is None else y.data_ptr(), ld_y,
        None if y8 is None else y8.data_ptr(), ld_8,
        _float_vector(scales, N * (-(-H // group) if group > 0 else 1), dev, where), _float_vector(rstd, N, dev, where), st)
    if code != OK:
        raise MrlError(code, where)


def mrl_rmsnorm_residual_bwd(dy, dh, h, weight, rstd, np: NormParams, dx, dweight=None, workspace=None, stream=None):
    where = "mrl_rmsnorm_residual_bwd"
    shape, dtype, dev = dy.shape, dy.dtype, dy.get_device()
    N, H = shape
    code = _CODES.get(dtype)
    if code is None:
        raise MrlError(3, where)
    st = _stream_of(dev, stream, where)
    w = _vector(weight, H, _CODES, dev, where)
    ld_dy, ld_dh = _row_stride(dy, shape, dtype, dev, where), _row_stride(dh, shape, dtype, dev, where)
    ld_h, ld_dx = _row_stride(h, shape, dtype, dev, where), _row_stride(dx, shape, dtype, dev, where)
    ws, ws_bytes = _workspace(workspace, dev, where)
    code = lib().mrl_rmsnorm_residual_bwd(
        dy.data_ptr(), ld_dy, None if dh is None else dh.data_ptr(), ld_dh, h.data_ptr(), ld_h, code, w, _CODES[weight.dtype],
        _float_vector(rstd, N, dev, where), N, H, np, dx.data_ptr(), ld_dx, _float_vector(dweight, H, dev, where), ws, ws_bytes,
        st)
    if code != OK:
        raise MrlError(code, where)


class TensorSlot:
    """One tensor of mrl_grad_norm / mrl_adamw_step: contiguous CUDA tensors of one size.  A gradient norm needs `grad`
    alone; 8-bit states are uint8 or float8_e4m3fn tensors with `m_scale`, `v_scale` of ceil(numel / STATE_BLOCK).

    The addresses are those of now: a tensor that is allocated anew later on (a gradient that autograd makes again after
    `p.grad = None`, a parameter whose `.data` is exchanged) needs a new slot.  Where `param` is a leaf and `grad` its `.grad`, a call
    after that has become another tensor is refused; other gradients are the caller's to keep in place."""

    def __init__(self, grad, param=None, master=None, m=None, v=None, m_scale=None, v_scale=None, weight_decay=0.0,
                 rng_first=0):
        n, dev, where = grad.numel(), grad.get_device(), "TensorSlot"
        codes = m is not None and m.dtype in _CODE_TYPES
        kind = _CODE_TYPES if codes else _F32_ONLY
        blocks = -(-n // STATE_BLOCK)
        self.struct = TensorSlotStruct(
            _vector(grad, n, _CODES, dev, where), _vector(param, n, _CODES, dev, where), _float_vector(master, n, dev, where),
            _vector(m, n, kind, dev, where), _vector(v, n, kind, dev, where), _float_vector(m_scale, blocks, dev, where),
            _float_vector(v_scale, blocks, dev, where), n, rng_first, weight_decay, _CODES[grad.dtype],
            F32 if param is None else _CODES[param.dtype], E4M3 if codes else F32)
        self.device = dev
        self.tensors = (grad, param, master, m, v, m_scale, v_scale)
        self.updates = None if param is None or n == 0 else param.data_ptr()
        self.watched = param is not None and param.requires_grad and param.is_leaf and param.grad is grad


class TensorList:
    """The table of a step's tensors: built once for tensors that stay where they are, which it keeps alive (see TensorSlot)."""

    def __init__(self, slots):
        self.slots = list(slots)
        if any(s.device != self.slots[0].device for s in self.slots):
            raise MrlError(1, "TensorList: tensors on several devices")
        params = [s.updates for s in self.slots if s.updates is not None]
        if len(set(params)) != len(params):
            raise MrlError(1, "TensorList: a parameter is there twice")
        self.device = self.slots[0].device if self.slots else torch.cuda.current_device()
        self.n = len(self.slots)
        self.table = (TensorSlotStruct * self.n)(*[s.struct for s in self.slots])
        self.address = C.addressof(self.table) if self.n else None
        self.watched = [(s.tensors[1], s.tensors[0]) for s in self.slots if s.watched]

    def check(self, where):
        """Refuses a list whose parameters have got other gradients since it was built."""
        for param, grad in self.watched:
            if param.grad is not grad:
                raise MrlError(1, f"{where}: a parameter's gradient is another tensor than in the list")


def mrl_grad_norm(tensors: TensorList, max_norm: float, norm=None, coef=None, workspace=None, stream=None):
    where, dev = "mrl_grad_norm", tensors.device
    if tensors.watched:
        tensors.check(where)
    st = _stream_of(dev, stream, where)
    ws, ws_bytes = _workspace(workspace, dev, where)
    code = lib().mrl_grad_norm(tensors.address, tensors.n, max_norm, _float_vector(norm, 1, dev, where),
                               _float_vector(coef, 1, dev, where), ws, ws_bytes, st)
    if code != OK:
        raise MrlError(code, where)


def mrl_adamw_step(tensors: TensorList, ap: AdamwParams, grad_scale=None, status=None, workspace=None, stream=None):
    where, dev = "mrl_adamw_step", tensors.device
    if tensors.watched:
        tensors.check(where)
    st = _stream_of(dev, stream, where)
    ws, ws_bytes = _workspace(workspace, dev, where)
    code = lib().mrl_adamw_step(tensors.address, tensors.n, ap, _float_vector(grad_scale, 1, dev, where),
                                _vector(status, 1, (torch.int32,), dev, where), ws, ws_bytes, st)
    if code != OK:
        raise MrlError(code, where)


# ---- a frozen model scored in 8 bits, its top tokens, and the loss that learns from them

_I32_ONLY, _U8_ONLY, _I64_ONLY = (torch.int32,), (torch.uint8,), (torch.int64,)


def _row_code(t, where):
    code = _CODES.get(t.dtype)
    if code is None:
        raise MrlError(3, where)
    return code


def mrl_e4m3_quantize(x, codes, scales, block_rows: int, stream=None):
    """Codes uint8 or float8_e4m3fn like x, scales float32 of ceil(N / block_rows) x ceil(H / 128)."""
    where, shape, dev = "mrl_e4m3_quantize", x.shape, x.get_device()
    N, H = shape
    code, st = _row_code(x, where), _stream_of(dev, stream, where)
    n_scales = -(-N // block_rows) * -(-H // SCALE_BLOCK) if block_rows > 0 else 0
    code = lib().mrl_e4m3_quantize(x.data_ptr(), _row_stride(x, shape, x.dtype, dev, where), code, N, H, block_rows,
                                   codes.data_ptr(), _row_stride(codes, shape, None, dev, where),
                                   _float_vector(scales, n_scales, dev, where), st)
    if code != OK:
        raise MrlError(code, where)


def mrl_e4m3_product(x8, x_scales, w8, w_scales, out, status=None, stream=None):
    """out[N, V] (bf16 or float32) of rows x8[N, H] and weights w8[V, H]; codes uint8 or float8_e4m3fn."""
    where, dev = "mrl_e4m3_product", x8.get_device()
    (N, H), V = x8.shape, w8.shape[0]
    code, st = _row_code(out, where), _stream_of(dev, stream, where)
    blocks = -(-H // SCALE_BLOCK)
    code = lib().mrl_e4m3_product(
        x8.data_ptr(), _row_stride(x8, x8.shape, None, dev, where), _float_vector(x_scales, N * blocks, dev, where),
        w8.data_ptr(), _row_stride(w8, (V, H), None, dev, where),
        _float_vector(w_scales, -(-V // SCALE_BLOCK) * blocks, dev, where), N, H, V, code, out.data_ptr(),
        _row_stride(out, (N, V), out.dtype, dev, where), _vector(status, 1, _I32_ONLY, dev, where), st)
    if code != OK:
        raise MrlError(code, where)


def mrl_top_logprobs(logits, ids, mask, temperature: float, logp=None, lse=None, entropy=None, top_ids=None, top_logp=None,
                     status=None, stream=None):
    """`top` is the number of columns of top_ids and top_logp (none: 0)."""
    where, shape, dev = "mrl_top_logprobs", logits.shape, logits.get_device()
    N, V = shape
    code, st = _row_code(logits, where), _stream_of(dev, stream, where)
    top = 0 if top_ids is None else top_ids.shape[-1]
    code = lib().mrl_top_logprobs(
        logits.data_ptr(), code, N, V, _row_stride(logits, shape, logits.dtype, dev, where),
        _vector(ids, N, _I32_ONLY, dev, where), _vector(mask, N, _U8_ONLY, dev, where), temperature, top,
        _float_vector(logp, N, dev, where), _float_vector(lse, N, dev, where), _float_vector(entropy, N, dev, where),
        _vector(top_ids, N * top, _I32_ONLY, dev, where), _float_vector(top_logp, N * top, dev, where),
        _vector(status, 1, _I32_ONLY, dev, where), st)
    if code != OK:
        raise MrlError(code, where)


def mrl_distill_loss_fwd_bwd(logits, top_ids, top_logp, mask, row_weight, dp: DistillParams, dlogits, row_kl, loss, stats=None,
                             status=None, workspace=None, stream=None):
    where, shape, dev = "mrl_distill_loss_fwd_bwd", logits.shape, logits.get_device()
    N, V = shape
    code, st = _row_code(logits, where), _stream_of(dev, stream, where)
    top = top_ids.shape[-1]
    ld, ld_out = _row_stride(logits, shape, logits.dtype, dev, where), _row_stride(dlogits, shape, logits.dtype, dev, where)
    ws, ws_bytes = _workspace(workspace, dev, where)
    code = lib().mrl_distill_loss_fwd_bwd(
        logits.data_ptr(), code, N, V, ld, _vector(top_ids, N * top, _I32_ONLY, dev, where),
        _float_vector(top_logp, N * top, dev, where), top, _vector(mask, N, _U8_ONLY, dev, where),
        _float_vector(row_weight, N, dev, where), dp, None if dlogits is None else dlogits.data_ptr(), ld_out or ld,
        _float_vector(row_kl, N, dev, where), _float_vector(loss, 1, dev, where), _vector(stats, 2, _I64_ONLY, dev, where),
        _vector(status, 1, _I32_ONLY, dev, where), ws, ws_bytes, st)
    if code != OK:
        raise MrlError(code, where)


class DominantKernelTimer:
    """Registers n CUDA-event pairs around the dominant kernel of the following calls; `elapsed_ms()`
    returns the duration of every recorded launch (after a synchronise)."""

    def __init__(self, n: int):
        self.n = n
        self.start = [torch.cuda.Event(enable_timing=True) for _ in range(n)]
        self.stop = [torch.cuda.Event(enable_timing=True) for _ in range(n)]
        for e in self.start + self.stop:      # torch creates the CUDA event lazily: force it
            e.record()
        torch.cuda.synchronize()
        self._a = (C.c_void_p * n)(*[e.cuda_event for e in self.start])
        self._b = (C.c_void_p * n)(*[e.cuda_event for e in self.stop])

    def __enter__(self):
        _check(lib().mrl_profile_dominant_kernel(self._a, self._b, self.n), "mrl_profile_dominant_kernel")
        return self

    def __exit__(self, *exc):
        self.last_kernel = lib().mrl_profile_last_kernel().decode()
        lib().mrl_profile_dominant_kernel(None, None, 0)

    def elapsed_ms(self, count: int):
        return [self.start[i].elapsed_time(self.stop[i]) for i in range(min(count, self.n))]
