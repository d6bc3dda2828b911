"""ctypes binding of the C ABI in include/moe.h (argument marshalling only).

Every function here has the name of the C entry point it calls and the same
arguments. Tensors may be passed as torch tensors (their ``data_ptr()`` is used),
as integer device addresses, or as None (NULL). ``stream`` may be a
``torch.cuda.Stream``, an integer handle, or None for the current torch stream.
A non-OK status raises ``MoEError`` carrying moe_last_error().

There is no fallback: if ``libmoe.so`` is missing this module raises on import.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmoe.so")

MOE_OK, MOE_ERR_INVALID_ARG, MOE_ERR_CUDA, MOE_ERR_DEVICE_CHECK, MOE_ERR_TIMEOUT, \
    MOE_ERR_UNSUPPORTED = range(6)
MOE_F32, MOE_BF16 = 0, 1
MOE_PAIRS_OFF, MOE_PAIRS_ALL, MOE_PAIRS_AUTO = 0, 1, 2
MOE_SCORE_SOFTMAX, MOE_SCORE_SIGMOID = 0, 1
CKPT_BLOCK = 128  # columns of a row that share a scale in an 8-bit checkpoint


class MoEError(RuntimeError):
    def __init__(self, status: int, fn: str, msg: str):
        super().__init__(f"{fn}: status {status} ({msg})")
        self.status = status


class moe_config(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int64),
        ("d_model", ctypes.c_int32),
        ("n_experts", ctypes.c_int32),
        ("d_ff", ctypes.c_int32),
        ("top_k", ctypes.c_int32),
        ("n_parties", ctypes.c_int32),
        ("n_shared", ctypes.c_int32),
        ("d_ff_shared", ctypes.c_int32),
        ("normalize_topk", ctypes.c_int32),
        ("aux_alpha", ctypes.c_float),
        ("dtype", ctypes.c_int32),
    ]


assert ctypes.sizeof(moe_config) == 48


class moe_gate_rule(ctypes.Structure):
    _fields_ = [
        ("score", ctypes.c_int32),
        ("n_groups", ctypes.c_int32),
        ("top_groups", ctypes.c_int32),
        ("group_top", ctypes.c_int32),
        ("scale", ctypes.c_float),
    ]


assert ctypes.sizeof(moe_gate_rule) == 20


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build the CUDA library first "
            "(python -m paper_2506_02965_gb300.build); there is no CPU fallback")
    return ctypes.CDLL(LIB_PATH)


_lib = _load()
P = ctypes.c_void_p
_CFG = ctypes.POINTER(moe_config)
_RULE = ctypes.POINTER(moe_gate_rule)
_I64, _I32, _INT, _F32, _SIZE = ctypes.c_int64, ctypes.c_int32, ctypes.c_int, ctypes.c_float, ctypes.c_size_t

# name -> argtypes (after the config pointer where present)
_SIGS = {
    "moe_workspace_size": [_CFG, ctypes.POINTER(ctypes.c_size_t)],
    "moe_route": [_CFG] + [P] * 10,
    "moe_route_from_logits": [_CFG] + [P] * 7,
    "moe_aux_loss": [_CFG] + [P] * 6,
    "moe_dispatch": [_CFG] + [P] * 7 + [ctypes.c_size_t, P],
    "moe_dispatch_noalloc": [_CFG] + [P] * 7,
    "moe_dispatch_owner": [_CFG] + [P] * 10 + [ctypes.c_size_t, P],
    "moe_expert_ffn_fwd": [_CFG] + [P] * 15,
    "moe_combine_fwd": [_CFG] + [P] * 6,
    "moe_combine_bwd": [_CFG] + [P] * 7,
    "moe_expert_ffn_bwd": [_CFG] + [P] * 23,
    "moe_route_bwd": [_CFG] + [P] * 13 + [ctypes.c_size_t, P],
    "moe_dispatch_bwd": [_CFG] + [P] * 6,
    "moe_device_status": [P, ctypes.POINTER(ctypes.c_int32)],
    "moe_set_wait_limit_ns": [ctypes.c_uint64],
    "moe_set_gemm_pairs": [ctypes.c_int],
    "moe_mse_loss": [_CFG] + [P] * 5 + [ctypes.c_size_t, P],
    "moe_expert_ffn_bwd_kernels": [_CFG, ctypes.POINTER(ctypes.c_int32)],
    "moe_sgd_update": [P, P, P, ctypes.c_int64, ctypes.c_int64, P, ctypes.c_float, ctypes.c_int, P],
    "moe_gather_rows": [P, P, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, P, P],
    "moe_gate": [_CFG, _RULE] + [P] * 8,
    "moe_route_gate": [_CFG, _RULE] + [P] * 11,
    "moe_gate_bwd": [_CFG, _RULE] + [P] * 12 + [_SIZE, P],
    "moe_gate_balance": [_CFG, P, _F32, P, P, P],
    "moe_layer_norm_fwd": [_I64, _I32, _INT] + [P] * 4 + [_F32] + [P] * 7,
    "moe_layer_norm_workspace_size": [_I64, _I32, ctypes.POINTER(_SIZE)],
    "moe_layer_norm_bwd": [_I64, _I32, _INT] + [P] * 12 + [_SIZE, P],
    "moe_ckpt_pack": [_I64, _I32, _INT] + [P] * 4,
    "moe_ckpt_unpack": [_I64, _I32, _INT] + [P] * 4,
    "moe_ckpt_swiglu_bwd": [_I64, _I32, _INT] + [P] * 6,
    "moe_expert_ffn_bwd_ckpt": [_CFG] + [P] * 25,
    "moe_embed_fwd": [_I64, _I32, _I32, _INT, P, P, _F32, P, P],
    "moe_embed_workspace_size": [_I64, _I32, _I32, ctypes.POINTER(_SIZE)],
    "moe_embed_bwd": [_I64, _I32, _I32, _INT, P, P, _F32, _INT, P, P, _SIZE, P],
    "moe_vocab_loss_workspace_size": [_I64, _I32, _I32, _INT, _INT, ctypes.POINTER(_SIZE)],
    "moe_vocab_loss": [_I64, _I32, _I32, _INT] + [P] * 9 + [_SIZE, P],
    "moe_orthogonalise_workspace_size": [_I32, _I32, _I32, _INT, ctypes.POINTER(_SIZE)],
    "moe_orthogonalise": [_I32, _I32, _I32, _INT, P, P, _F32, _INT, P, _I32, _F32, P, P, P, _SIZE, P],
}
for _n, _a in _SIGS.items():
    f = getattr(_lib, _n)
    f.argtypes = _a
    f.restype = ctypes.c_int
for _n in ("moe_status_string",):
    getattr(_lib, _n).argtypes = [ctypes.c_int]
    getattr(_lib, _n).restype = ctypes.c_char_p
for _n in ("moe_last_error", "moe_version"):
    getattr(_lib, _n).argtypes = []
    getattr(_lib, _n).restype = ctypes.c_char_p

EXPORTED = list(_SIGS) + ["moe_status_string", "moe_last_error", "moe_version"]


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


_current_stream = None


def _raw_stream_getter():
    """The current torch stream's handle. The raw getter where torch has it (0.1 us a call against 3 to 5 through a
    Stream object, of a launch's 3)."""
    global _current_stream
    import torch
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    _current_stream = lambda: raw(device())  # noqa: E731
    return _current_stream()


def _stream(s):
    if s is None:
        return _current_stream() if _current_stream is not None else _raw_stream_getter()
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(st: int, fn: str):
    if st != MOE_OK:
        raise MoEError(st, fn, _lib.moe_last_error().decode())


def _call(fn: str, cfg, *args, stream=None):
    c = getattr(_lib, fn)
    conv = []
    for a, ty in zip(args, c.argtypes[1:]):
        conv.append(a if ty is ctypes.c_size_t else _ptr(a))
    _check(c(ctypes.byref(cfg), *conv, _stream(stream)), fn)


def make_config(T, d_model, n_experts, d_ff, top_k, n_parties=1, n_shared=0, d_ff_shared=0,
                normalize_topk=0, aux_alpha=0.01, dtype=MOE_BF16) -> moe_config:
    return moe_config(int(T), int(d_model), int(n_experts), int(d_ff), int(top_k), int(n_parties),
                      int(n_shared), int(d_ff_shared), int(normalize_topk), float(aux_alpha),
                      int(dtype))


def moe_version() -> str:
    return _lib.moe_version().decode()


def moe_status_string(s: int) -> str:
    return _lib.moe_status_string(s).decode()


def moe_last_error() -> str:
    return _lib.moe_last_error().decode()


def moe_workspace_size(cfg) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.moe_workspace_size(ctypes.byref(cfg), ctypes.byref(n)), "moe_workspace_size")
    return n.value


def moe_set_wait_limit_ns(ns: int):
    _check(_lib.moe_set_wait_limit_ns(int(ns)), "moe_set_wait_limit_ns")


def moe_set_gemm_pairs(on: int):
    _check(_lib.moe_set_gemm_pairs(int(on)), "moe_set_gemm_pairs")


def moe_device_status(stream=None) -> int:
    code = ctypes.c_int32(0)
    _check(_lib.moe_device_status(_stream(stream), ctypes.byref(code)), "moe_device_status")
    return code.value


def moe_route(cfg, x, w_router, router_bias, party_offsets, logits, probs, topk_idx, topk_w,
              counts, stream=None):
    _call("moe_route", cfg, x, w_router, router_bias, party_offsets, logits, probs, topk_idx,
          topk_w, counts, stream=stream)


def moe_route_from_logits(cfg, logits, party_offsets, probs, topk_idx, topk_w, counts,
                          stream=None):
    _call("moe_route_from_logits", cfg, logits, party_offsets, probs, topk_idx, topk_w, counts,
          stream=stream)


def moe_aux_loss(cfg, probs, counts, party_offsets, loss, aux_coef, stream=None):
    _call("moe_aux_loss", cfg, probs, counts, party_offsets, loss, aux_coef, stream=stream)


def moe_dispatch(cfg, topk_idx, x, offsets, slot_of, token_of, x_perm, workspace,
                 workspace_bytes, stream=None):
    _call("moe_dispatch", cfg, topk_idx, x, offsets, slot_of, token_of, x_perm, workspace,
          int(workspace_bytes), stream=stream)


def moe_dispatch_noalloc(cfg, topk_idx, x, offsets, slot_of, token_of, x_perm, stream=None):
    _call("moe_dispatch_noalloc", cfg, topk_idx, x, offsets, slot_of, token_of, x_perm,
          stream=stream)


def moe_dispatch_owner(cfg, topk_idx, x, party_offsets, group_expert, offsets, slot_of, token_of,
                       x_perm, send_counts, workspace, workspace_bytes, stream=None):
    _call("moe_dispatch_owner", cfg, topk_idx, x, party_offsets, group_expert, offsets, slot_of,
          token_of, x_perm, send_counts, workspace, int(workspace_bytes), stream=stream)


def moe_expert_ffn_fwd(cfg, x_perm, offsets, w1, w2, h_gu, act, y_perm, x=None, ws1=None,
                       ws2=None, h_gu_sh=None, act_sh=None, y_sh=None, group_expert=None,
                       stream=None):
    _call("moe_expert_ffn_fwd", cfg, x_perm, offsets, w1, w2, h_gu, act, y_perm, x, ws1, ws2,
          h_gu_sh, act_sh, y_sh, group_expert, stream=stream)


def moe_expert_ffn_bwd_kernels(cfg) -> int:
    n = ctypes.c_int32(0)
    _check(_lib.moe_expert_ffn_bwd_kernels(ctypes.byref(cfg), ctypes.byref(n)), "moe_expert_ffn_bwd_kernels")
    return int(n.value)


def moe_mse_loss(cfg, out, target, loss, dout, workspace, workspace_bytes, stream=None):
    _call("moe_mse_loss", cfg, out, target, loss, dout, workspace, workspace_bytes, stream=stream)


def moe_sgd_update(w, dw, n_groups, group_elems, group_counts, lr, dtype, w_master=None, stream=None):
    _check(_lib.moe_sgd_update(_ptr(w), _ptr(dw), _ptr(w_master), int(n_groups), int(group_elems),
                               _ptr(group_counts), float(lr), int(dtype), _stream(stream)), "moe_sgd_update")


def moe_gather_rows(src, rows, n_rows, n_src_rows, row_elems, dtype, dst, stream=None):
    _check(_lib.moe_gather_rows(_ptr(src), _ptr(rows), int(n_rows), int(n_src_rows), int(row_elems),
                                int(dtype), _ptr(dst), _stream(stream)), "moe_gather_rows")


def moe_combine_fwd(cfg, y_perm, topk_w, slot_of, y_sh, out, stream=None):
    _call("moe_combine_fwd", cfg, y_perm, topk_w, slot_of, y_sh, out, stream=stream)


def moe_combine_bwd(cfg, dout, y_perm, topk_w, slot_of, dy_perm, dtopk_w, stream=None):
    _call("moe_combine_bwd", cfg, dout, y_perm, topk_w, slot_of, dy_perm, dtopk_w, stream=stream)


def moe_expert_ffn_bwd(cfg, x_perm, offsets, w1, w2, h_gu, act, dy_perm, dh, dx_perm, dw1, dw2,
                       x=None, dout=None, ws1=None, ws2=None, h_gu_sh=None, act_sh=None,
                       dh_sh=None, dx_sh=None, dws1=None, dws2=None, group_expert=None,
                       stream=None):
    _call("moe_expert_ffn_bwd", cfg, x_perm, offsets, w1, w2, h_gu, act, dy_perm, dh, dx_perm,
          dw1, dw2, x, dout, ws1, ws2, h_gu_sh, act_sh, dh_sh, dx_sh, dws1, dws2, group_expert,
          stream=stream)


def moe_route_bwd(cfg, x, w_router, probs, topk_idx, topk_w, dtopk_w, aux_coef, party_offsets,
                  dlogits, dw_router, dbias, dx_router, workspace, workspace_bytes, stream=None):
    _call("moe_route_bwd", cfg, x, w_router, probs, topk_idx, topk_w, dtopk_w, aux_coef,
          party_offsets, dlogits, dw_router, dbias, dx_router, workspace, int(workspace_bytes),
          stream=stream)


def moe_dispatch_bwd(cfg, dx_perm, slot_of, dx_router, dx_sh, dx, stream=None):
    _call("moe_dispatch_bwd", cfg, dx_perm, slot_of, dx_router, dx_sh, dx, stream=stream)


# ------------------------------------------------------------------ operators around the layer
# These also check what a tensor is before its address is taken: on the GPU, dense, of the right
# element type and as many elements as the call's sizes say (moe_expert_ffn_bwd_ckpt's: at least as many; a
# workspace: of at least the bytes that the call is told). The kinds: MOE_F32, MOE_BF16 and
_I32T, _I8T = 2, 3
_kinds = None


def _check_arr(fn, name, t, kind, n):
    """Address of a dense GPU tensor of n elements of `kind`; an address or None as it is."""
    if t is None or type(t) is int:
        return t
    global _kinds
    if _kinds is None:
        import torch
        _kinds = (torch.float32, torch.bfloat16, torch.int32, torch.int8)
    if t.numel() == n and t.is_cuda and t.is_contiguous() and t.dtype is _kinds[kind]:
        return t.data_ptr()
    raise MoEError(MOE_ERR_INVALID_ARG, fn, f"{name}: expected a dense GPU tensor of {n} elements of {_kinds[kind]}, got "
                                            f"{tuple(t.shape)} {t.dtype}, strides {t.stride()}, on {t.device}")


def _arr(fn, name, t, kind, n):
    """_check_arr; from the first tensor on in C++ (csrc/marshal.cpp), where that is built for this torch."""
    global _arr
    if t is None or type(t) is int:
        return t
    import torch
    from importlib import machinery, util
    try:
        spec = util.spec_from_loader("_marshal", machinery.ExtensionFileLoader("_marshal", os.path.join(HERE, "_marshal.so")))
        m = util.module_from_spec(spec)
        m.set_slow(_check_arr)
        # one that was built for another torch does not read this one's tensors
        _arr = m.addr if m.torch_version == torch.__version__.split("+")[0] else _check_arr
    except (ImportError, OSError):
        _arr = _check_arr
    return _arr(fn, name, t, kind, n)


def _room(fn, name, t, kind, n):
    """_arr for a buffer that may hold more than n elements."""
    if t is None or isinstance(t, int):
        return t
    return _arr(fn, name, t, kind, max(n, t.numel()))


def _work(fn, t, nbytes):
    """Address of a dense GPU tensor, of any element type, that holds nbytes; an address or None as it is."""
    if t is None or isinstance(t, int):
        return t
    if t.is_cuda and t.is_contiguous() and t.numel() * t.element_size() >= nbytes:
        return t.data_ptr()
    raise MoEError(MOE_ERR_INVALID_ARG, fn, f"workspace: expected a dense GPU tensor of {nbytes} bytes, got {tuple(t.shape)} {t.dtype}, "
                                            f"strides {t.stride()}, on {t.device}")


def _dtype_of(fn, dtype):
    if dtype != MOE_F32 and dtype != MOE_BF16:
        raise MoEError(MOE_ERR_INVALID_ARG, fn, f"unknown dtype {dtype}")
    return int(dtype)


def ckpt_blocks(cols: int) -> int:
    """Scales per row of an 8-bit checkpoint of `cols` columns."""
    return -(-cols // CKPT_BLOCK)


def make_gate_rule(score=MOE_SCORE_SOFTMAX, n_groups=1, top_groups=1, group_top=1, scale=1.0) -> moe_gate_rule:
    return moe_gate_rule(int(score), int(n_groups), int(top_groups), int(group_top), float(scale))


def _gate_arrays(fn, cfg, logits, balance_bias, party_offsets, scores, topk_idx, topk_w, counts):
    T, E, k, Pn = cfg.T, cfg.n_experts, cfg.top_k, cfg.n_parties
    return (_arr(fn, "logits", logits, MOE_F32, T * E), _arr(fn, "balance_bias", balance_bias, MOE_F32, Pn * E),
            _arr(fn, "party_offsets", party_offsets, _I32T, Pn + 1), _arr(fn, "scores", scores, MOE_F32, T * E),
            _arr(fn, "topk_idx", topk_idx, _I32T, T * k), _arr(fn, "topk_w", topk_w, MOE_F32, T * k),
            _arr(fn, "counts", counts, _I32T, Pn * E))


def moe_gate(cfg, rule, logits, balance_bias, party_offsets, scores, topk_idx, topk_w, counts, stream=None):
    a = _gate_arrays("moe_gate", cfg, logits, balance_bias, party_offsets, scores, topk_idx, topk_w, counts)
    _check(_lib.moe_gate(cfg, rule, *a, _stream(stream)), "moe_gate")


def moe_route_gate(cfg, rule, x, w_router, router_bias, balance_bias, party_offsets, logits, scores, topk_idx, topk_w, counts,
                   stream=None):
    fn = "moe_route_gate"
    T, E, d, Pn = cfg.T, cfg.n_experts, cfg.d_model, cfg.n_parties
    logits, balance_bias, party_offsets, scores, topk_idx, topk_w, counts = _gate_arrays(
        fn, cfg, logits, balance_bias, party_offsets, scores, topk_idx, topk_w, counts)
    dt = _dtype_of(fn, cfg.dtype)
    _check(_lib.moe_route_gate(cfg, rule, _arr(fn, "x", x, dt, T * d), _arr(fn, "w_router", w_router, dt, Pn * E * d),
                               _arr(fn, "router_bias", router_bias, MOE_F32, Pn * E), balance_bias, party_offsets, logits, scores,
                               topk_idx, topk_w, counts, _stream(stream)), fn)


def moe_gate_bwd(cfg, rule, logits, topk_idx, dtopk_w, aux_coef, party_offsets, dlogits, x=None, w_router=None, dw_router=None,
                 dbias=None, dx_router=None, workspace=None, workspace_bytes=0, stream=None):
    fn = "moe_gate_bwd"
    T, E, d, k, Pn = cfg.T, cfg.n_experts, cfg.d_model, cfg.top_k, cfg.n_parties
    dt = _dtype_of(fn, cfg.dtype)
    _check(_lib.moe_gate_bwd(cfg, rule, _arr(fn, "logits", logits, MOE_F32, T * E), _arr(fn, "topk_idx", topk_idx, _I32T, T * k),
                             _arr(fn, "dtopk_w", dtopk_w, MOE_F32, T * k), _arr(fn, "aux_coef", aux_coef, MOE_F32, Pn * E),
                             _arr(fn, "party_offsets", party_offsets, _I32T, Pn + 1), _arr(fn, "dlogits", dlogits, MOE_F32, T * E),
                             _arr(fn, "x", x, dt, T * d), _arr(fn, "w_router", w_router, dt, Pn * E * d),
                             _arr(fn, "dw_router", dw_router, dt, Pn * E * d), _arr(fn, "dbias", dbias, MOE_F32, Pn * E),
                             _arr(fn, "dx_router", dx_router, dt, T * d),
                             _work(fn, workspace, workspace_bytes) if dw_router is not None else None, int(workspace_bytes),
                             _stream(stream)), fn)


def moe_gate_balance(cfg, counts, rate, bias_in, bias_out, stream=None):
    fn, n = "moe_gate_balance", cfg.n_parties * cfg.n_experts
    _check(_lib.moe_gate_balance(cfg, _arr(fn, "counts", counts, _I32T, n), rate, _arr(fn, "bias_in", bias_in, MOE_F32, n),
                                 _arr(fn, "bias_out", bias_out, MOE_F32, n), _stream(stream)), fn)


def moe_layer_norm_workspace_size(rows, d) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.moe_layer_norm_workspace_size(int(rows), int(d), ctypes.byref(n)), "moe_layer_norm_workspace_size")
    return n.value


def moe_layer_norm_fwd(rows, d, dtype, x, residual, gamma, beta, eps, h, y, mean=None, rstd=None, h_q=None, h_scale=None,
                       stream=None):
    fn, n = "moe_layer_norm_fwd", rows * d
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_layer_norm_fwd(rows, d, dt, _arr(fn, "x", x, dt, n), _arr(fn, "residual", residual, dt, n),
                                   _arr(fn, "gamma", gamma, MOE_F32, d), _arr(fn, "beta", beta, MOE_F32, d), eps,
                                   _arr(fn, "h", h, dt, n), _arr(fn, "y", y, dt, n), _arr(fn, "mean", mean, MOE_F32, rows),
                                   _arr(fn, "rstd", rstd, MOE_F32, rows), _arr(fn, "h_q", h_q, _I8T, n),
                                   _arr(fn, "h_scale", h_scale, MOE_F32, rows * ckpt_blocks(d)), _stream(stream)), fn)


def moe_layer_norm_bwd(rows, d, dtype, dy, h, h_q, h_scale, mean, rstd, gamma, dh, dx, dgamma, dbeta, workspace,
                       workspace_bytes, stream=None):
    fn, n = "moe_layer_norm_bwd", rows * d
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_layer_norm_bwd(rows, d, dt, _arr(fn, "dy", dy, dt, n), _arr(fn, "h", h, dt, n), _arr(fn, "h_q", h_q, _I8T, n),
                                   _arr(fn, "h_scale", h_scale, MOE_F32, rows * ckpt_blocks(d)), _arr(fn, "mean", mean, MOE_F32, rows),
                                   _arr(fn, "rstd", rstd, MOE_F32, rows), _arr(fn, "gamma", gamma, MOE_F32, d),
                                   _arr(fn, "dh", dh, dt, n), _arr(fn, "dx", dx, dt, n), _arr(fn, "dgamma", dgamma, MOE_F32, d),
                                   _arr(fn, "dbeta", dbeta, MOE_F32, d), _work(fn, workspace, workspace_bytes), int(workspace_bytes),
                                   _stream(stream)), fn)


def moe_ckpt_pack(rows, cols, dtype, x, q, scale, stream=None):
    fn, n = "moe_ckpt_pack", rows * cols
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_ckpt_pack(rows, cols, dt, _arr(fn, "x", x, dt, n), _arr(fn, "q", q, _I8T, n),
                              _arr(fn, "scale", scale, MOE_F32, rows * ckpt_blocks(cols)), _stream(stream)), fn)


def moe_ckpt_unpack(rows, cols, dtype, q, scale, x, stream=None):
    fn, n = "moe_ckpt_unpack", rows * cols
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_ckpt_unpack(rows, cols, dt, _arr(fn, "q", q, _I8T, n),
                                _arr(fn, "scale", scale, MOE_F32, rows * ckpt_blocks(cols)), _arr(fn, "x", x, dt, n),
                                _stream(stream)), fn)


def moe_ckpt_swiglu_bwd(rows, d_ff, dtype, q, scale, dact, act, dh, stream=None):
    fn, n = "moe_ckpt_swiglu_bwd", rows * d_ff
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_ckpt_swiglu_bwd(rows, d_ff, dt, _arr(fn, "q", q, _I8T, 2 * n),
                                    _arr(fn, "scale", scale, MOE_F32, rows * ckpt_blocks(2 * d_ff)),
                                    _arr(fn, "dact", dact, dt, n), _arr(fn, "act", act, dt, n), _arr(fn, "dh", dh, dt, 2 * n),
                                    _stream(stream)), fn)


def moe_expert_ffn_bwd_ckpt(cfg, x_perm, offsets, w1, w2, gu_q, gu_scale, dy_perm, dact, act, dh, dx_perm, dw1, dw2, x=None,
                            dout=None, ws1=None, ws2=None, h_gu_sh=None, act_sh=None, dh_sh=None, dx_sh=None, dws1=None,
                            dws2=None, group_expert=None, stream=None):
    fn = "moe_expert_ffn_bwd_ckpt"
    T, d, E, F, S, Fs, dt = cfg.T, cfg.d_model, cfg.n_experts, cfg.d_ff, cfg.n_shared, cfg.d_ff_shared, _dtype_of(fn, cfg.dtype)
    TK, some = T * cfg.top_k, T > 0

    # what the call does not use (without tokens all but the weights' gradients, without shared experts theirs) is not looked at
    def at(name, t, n, kind=dt, used=some):
        return _room(fn, name, t, kind, n) if used else None

    def sh(name, t, n, used=some):
        return at(name, t, n, used=S > 0 and used)

    _check(_lib.moe_expert_ffn_bwd_ckpt(
        cfg, at("x_perm", x_perm, TK * d), at("offsets", offsets, E + 1, _I32T), at("w1", w1, E * 2 * F * d),
        at("w2", w2, E * d * F), at("gu_q", gu_q, TK * 2 * F, _I8T), at("gu_scale", gu_scale, TK * ckpt_blocks(2 * F), MOE_F32),
        at("dy_perm", dy_perm, TK * d), at("dact", dact, TK * F), at("act", act, TK * F), at("dh", dh, TK * 2 * F),
        at("dx_perm", dx_perm, TK * d), at("dw1", dw1, E * 2 * F * d, used=True), at("dw2", dw2, E * d * F, used=True),
        sh("x", x, T * d), sh("dout", dout, T * d), sh("ws1", ws1, S * 2 * Fs * d), sh("ws2", ws2, S * d * Fs),
        sh("h_gu_sh", h_gu_sh, S * T * 2 * Fs), sh("act_sh", act_sh, S * T * Fs), sh("dh_sh", dh_sh, S * T * 2 * Fs),
        sh("dx_sh", dx_sh, S * T * d), sh("dws1", dws1, S * 2 * Fs * d, used=True), sh("dws2", dws2, S * d * Fs, used=True),
        at("group_expert", group_expert, E, _I32T), _stream(stream)), fn)


# ------------------------------------------------------------------ around a stack of blocks
def moe_embed_fwd(T, d, V, dtype, ids, w, scale, out, stream=None):
    fn = "moe_embed_fwd"
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_embed_fwd(T, d, V, dt, _arr(fn, "ids", ids, _I32T, T), _arr(fn, "w", w, dt, V * d), scale,
                              _arr(fn, "out", out, dt, T * d), _stream(stream)), fn)


def moe_embed_workspace_size(T, d, V) -> int:
    n = ctypes.c_size_t(0)
    _check(_lib.moe_embed_workspace_size(int(T), int(d), int(V), ctypes.byref(n)), "moe_embed_workspace_size")
    return n.value


def moe_embed_bwd(T, d, V, dtype, ids, dout, scale, accumulate, dw, workspace, workspace_bytes, stream=None):
    fn = "moe_embed_bwd"
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_embed_bwd(T, d, V, dt, _arr(fn, "ids", ids, _I32T, T), _arr(fn, "dout", dout, dt, T * d), scale, accumulate,
                              _arr(fn, "dw", dw, dt, V * d), _work(fn, workspace, workspace_bytes), workspace_bytes,
                              _stream(stream)), fn)


def moe_vocab_loss_workspace_size(T, d, V, dtype, with_grads) -> int:
    fn, n = "moe_vocab_loss_workspace_size", ctypes.c_size_t(0)
    _check(_lib.moe_vocab_loss_workspace_size(int(T), int(d), int(V), _dtype_of(fn, dtype), int(bool(with_grads)), ctypes.byref(n)), fn)
    return n.value


def moe_vocab_loss(T, d, V, dtype, h, w, target, weight, loss, token_loss, dh, dw, workspace, workspace_bytes, stream=None):
    fn = "moe_vocab_loss"
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_vocab_loss(T, d, V, dt, _arr(fn, "h", h, dt, T * d), _arr(fn, "w", w, dt, V * d), _arr(fn, "target", target, _I32T, T),
                               _arr(fn, "weight", weight, MOE_F32, T), _arr(fn, "loss", loss, MOE_F32, 1),
                               _arr(fn, "token_loss", token_loss, MOE_F32, T), _arr(fn, "dh", dh, dt, T * d),
                               _arr(fn, "dw", dw, dt, V * d), _work(fn, workspace, workspace_bytes), workspace_bytes,
                               _stream(stream)), fn)


def moe_orthogonalise_workspace_size(groups, rows, cols, dtype) -> int:
    fn, n = "moe_orthogonalise_workspace_size", ctypes.c_size_t(0)
    _check(_lib.moe_orthogonalise_workspace_size(int(groups), int(rows), int(cols), _dtype_of(fn, dtype), ctypes.byref(n)), fn)
    return n.value


def moe_orthogonalise(groups, rows, cols, dtype, dw, momentum, beta, nesterov, group_counts, steps, scale, momentum_out, out, workspace,
                      workspace_bytes, stream=None):
    fn, n = "moe_orthogonalise", groups * rows * cols
    dt = _dtype_of(fn, dtype)
    _check(_lib.moe_orthogonalise(groups, rows, cols, dt, _arr(fn, "dw", dw, dt, n), _arr(fn, "momentum", momentum, MOE_F32, n), beta,
                                  nesterov, _arr(fn, "group_counts", group_counts, _I32T, groups), steps, scale,
                                  _arr(fn, "momentum_out", momentum_out, MOE_F32, n), _arr(fn, "out", out, dt, n),
                                  _work(fn, workspace, workspace_bytes), workspace_bytes, _stream(stream)), fn)
