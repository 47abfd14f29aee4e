"""ctypes binding of libpmpe (include/pmpe.h): argument marshalling only.

Every function has the name of the C entry point and takes torch tensors (or None)
where the C call takes device pointers; the HIP stream defaults to torch's current
stream. A negative status raises PmpeError. Every step of the layer runs in the HIP
kernels of libpmpe; if the library is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes
import os
from array import array
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# Only the library built in the package directory is loaded: it is the code that
# enforces the policy mask and writes the execution audit.
LIB_PATH = os.path.join(_PKG, "libpmpe.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is not built; run `python -m paper_2608_06690_amd.build` "
        "(or __graft_entry__.build()) first")

_lib = ctypes.CDLL(LIB_PATH)

PMPE_OK = 0
PMPE_F32 = 0
PMPE_BF16 = 1
PMPE_FP8_E4M3 = 2
PMPE_GATE_RENORM_TOPK = 0
PMPE_GATE_POOL_SOFTMAX = 1
PMPE_ROUTE_MASKED = 0
PMPE_ROUTE_SOFT = 1
PMPE_POLICY_ALLOW = 0xA11C0DE5
PMPE_POLICY_DENY = 0x00000000
PMPE_DEV_PRIV_ROUTER_MISSING = 0x1
PMPE_DEV_PRIV_WEIGHTS_MISSING = 0x2

STATUS_NAMES = {
    0: "PMPE_OK", -1: "PMPE_ERR_NULL", -2: "PMPE_ERR_SHAPE", -3: "PMPE_ERR_K_EXCEEDS_POOL",
    -4: "PMPE_ERR_DTYPE", -5: "PMPE_ERR_ALIGN", -6: "PMPE_ERR_WORKSPACE", -7: "PMPE_ERR_LAUNCH",
    -8: "PMPE_ERR_TAG_MISMATCH", -9: "PMPE_ERR_SCRATCH",
}
PMPE_ERR_TAG_MISMATCH = -8
PMPE_ERR_SCRATCH = -9
PMPE_NOALLOC_SCRATCH_BYTES = 2 << 20
PMPE_LORA_GATE_ROW = 0
PMPE_LORA_GATE_TILE = 1
PMPE_LORA_GATE_POSTHOC = 2
PMPE_LORA_TILE_ROWS = 64
PMPE_SCORE_SOFTMAX = 0
PMPE_SCORE_SIGMOID = 1
PMPE_POOL_PUBLIC = 0
PMPE_POOL_PRIVATE = 1
PMPE_POOL_MIXED = 2


class PmpeError(RuntimeError):
    def __init__(self, status: int, call: str):
        self.status = status
        msg = _lib.pmpe_status_string(status).decode()
        super().__init__(f"{call}: {STATUS_NAMES.get(status, status)} ({msg})")


class LayerDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "hidden", "inter", "n_pub", "n_priv", "top_k", "n_shared", "shared_inter",
        "act_dtype", "w_dtype", "gate_mode", "route_mode")]


class CacheTag(ctypes.Structure):
    """pmpe_cache_tag: resolved decision (1 allow, 0 deny), model revision digest and
    checkpoint fingerprint (32 bytes each)."""
    _fields_ = [("decision", ctypes.c_uint32), ("model_revision", ctypes.c_uint8 * 32),
                ("checkpoint_fingerprint", ctypes.c_uint8 * 32)]


def make_cache_tag(decision: int, model_revision: bytes, checkpoint_fingerprint: bytes) -> CacheTag:
    if len(model_revision) != 32 or len(checkpoint_fingerprint) != 32:
        raise ValueError("model_revision and checkpoint_fingerprint are 32-byte digests")
    t = CacheTag()
    t.decision = decision
    t.model_revision[:] = list(model_revision)
    t.checkpoint_fingerprint[:] = list(checkpoint_fingerprint)
    return t


class ForwardArgs(ctypes.Structure):
    """pmpe_forward_args: the buffers of one layer forward."""
    POINTERS = (
        "x", "wr_pub", "wr_priv", "logit_bias", "policy_word", "topk_idx", "topk_gate", "allow", "kgap",
        "expert_count", "expert_offset", "row_token", "token_row", "x_perm", "w13_pub", "w2_pub", "w13_priv",
        "w2_priv", "w13_sh", "w2_sh", "w13s_pub", "w2s_pub", "w13s_priv", "w2s_priv", "y_shared", "y_perm", "ab",
        "out", "audit_token_rows", "audit_priv_calls", "req_offset", "req_private_rows", "total_private_rows",
        "deny_violations", "dev_status", "ws")
    _fields_ = [(n, ctypes.c_void_p) for n in POINTERS] + [
        ("ws_bytes", ctypes.c_size_t), ("R", ctypes.c_int32), ("ffn", ctypes.c_int32), ("failed", ctypes.c_int32)]


class ScoreRule(ctypes.Structure):
    """pmpe_score_rule: how pmpe_select and pmpe_route_scored choose and weight experts."""
    _fields_ = [(n, ctypes.c_int32) for n in ("score", "group_top", "n_group_pub", "topk_group_pub", "n_group_priv",
                                              "topk_group_priv")] + [("scale", ctypes.c_float)]


def make_score_rule(score: int = 1, groups=(1, 1), groups_priv=(1, 1), group_top: int = 2,
                    scale: float = 1.0) -> ScoreRule:
    """A score rule; groups and groups_priv are (groups, groups that stay) of the two pools."""
    return ScoreRule(score, group_top, groups[0], groups[1], groups_priv[0], groups_priv[1], scale)


_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_SZ = ctypes.c_size_t
_DESC = ctypes.POINTER(LayerDesc)

_lib.pmpe_version.restype = _I32
_lib.pmpe_version.argtypes = []
_lib.pmpe_status_string.restype = ctypes.c_char_p
_lib.pmpe_status_string.argtypes = [_I32]
_lib.pmpe_workspace_bytes.restype = _SZ
_lib.pmpe_workspace_bytes.argtypes = [_DESC, _I32]
_lib.pmpe_check_desc.restype = _I32
_lib.pmpe_check_desc.argtypes = [_DESC, _I32]
_lib.pmpe_route.restype = _I32
_lib.pmpe_route.argtypes = [_DESC, _I32] + [_P] * 10 + [_P, _SZ, _P]
_lib.pmpe_dispatch.restype = _I32
_lib.pmpe_dispatch.argtypes = [_DESC, _I32] + [_P] * 7 + [_P, _SZ, _P]
_lib.pmpe_dispatch_noalloc.restype = _I32
_lib.pmpe_dispatch_noalloc.argtypes = [_DESC, _I32] + [_P] * 7 + [_P]
_lib.pmpe_expert_ffn.restype = _I32
_lib.pmpe_expert_ffn.argtypes = [_DESC, _I32] + [_P] * 16 + [_P, _SZ, _P]
_lib.pmpe_combine.restype = _I32
_lib.pmpe_combine.argtypes = [_DESC, _I32] + [_P] * 5 + [_P]
_lib.pmpe_audit.restype = _I32
_lib.pmpe_audit.argtypes = [_DESC, _I32, _P, _P, _P, _I32, _P, _P, _P, _P]

_lib.pmpe_layer_forward.restype = _I32
_lib.pmpe_layer_forward.argtypes = [_DESC, _I32, ctypes.POINTER(ForwardArgs), _P]

_lib.pmpe_backward_workspace_bytes.restype = _SZ
_lib.pmpe_backward_workspace_bytes.argtypes = [_DESC, _I32]
_lib.pmpe_backward.restype = _I32
_lib.pmpe_backward.argtypes = [_DESC, _I32] + [_P] * 28 + [_P, _SZ, _P]
_lib.pmpe_transpose_experts.restype = _I32
_lib.pmpe_transpose_experts.argtypes = [_P, _P, _I32, _I32, _I32, _P]
_lib.pmpe_expert_ffn_train.restype = _I32
_lib.pmpe_expert_ffn_train.argtypes = [_DESC, _I32] + [_P] * 17 + [_P, _SZ, _P]
_lib.pmpe_expert_ffn_fp8.restype = _I32
_lib.pmpe_expert_ffn_fp8.argtypes = [_DESC, _I32] + [_P] * 17 + [_P, _SZ, _P]
_lib.pmpe_expert_ffn_lora_workspace_bytes.restype = _SZ
_lib.pmpe_expert_ffn_lora_workspace_bytes.argtypes = [_DESC, _I32]
_lib.pmpe_expert_ffn_lora.restype = _I32
_lib.pmpe_expert_ffn_lora.argtypes = ([_DESC, _I32] + [_P] * 13 + [_I32, ctypes.c_float, _I32]
                                      + [_P] * 3 + [_P, _SZ, _P])
_lib.pmpe_adamw.restype = _I32
_lib.pmpe_adamw.argtypes = [_P, _I32, _P, _P, _P, _P, ctypes.c_uint64, _I32] + [ctypes.c_float] * 5 + [_P]
_lib.pmpe_route_record.restype = _I32
_lib.pmpe_route_record.argtypes = [_DESC, _I32, _I32, _P, _P, _P, _I32, _P, _P]
_lib.pmpe_cache_tag_check.restype = _I32
_lib.pmpe_cache_tag_check.argtypes = [ctypes.POINTER(CacheTag), ctypes.POINTER(CacheTag)]
_lib.pmpe_fingerprint_workspace_bytes.restype = _SZ
_lib.pmpe_fingerprint_workspace_bytes.argtypes = [ctypes.c_uint64]
_lib.pmpe_fingerprint.restype = _I32
_lib.pmpe_fingerprint.argtypes = [_P, ctypes.c_uint64, _P, _P, _SZ, _P]

_lib.pmpe_rmsnorm.restype = _I32
_lib.pmpe_rmsnorm.argtypes = [_I32] * 3 + [_P] * 3 + [_I32, ctypes.c_float] + [_P] * 6
_lib.pmpe_rmsnorm_backward_workspace_bytes.restype = _SZ
_lib.pmpe_rmsnorm_backward_workspace_bytes.argtypes = [_I32, _I32]
_lib.pmpe_rmsnorm_backward.restype = _I32
_lib.pmpe_rmsnorm_backward.argtypes = [_I32] * 3 + [_P, _I32] + [_P] * 3 + [_I32] + [_P] * 4 + [_SZ, _P]
_RULE = ctypes.POINTER(ScoreRule)
_lib.pmpe_select.restype = _I32
_lib.pmpe_select.argtypes = [_DESC, _RULE, _I32, _P, _I32] + [_P] * 8
_lib.pmpe_select_backward.restype = _I32
_lib.pmpe_select_backward.argtypes = [_DESC, _RULE, _I32, _P, _I32] + [_P] * 4
_lib.pmpe_route_scored.restype = _I32
_lib.pmpe_route_scored.argtypes = [_DESC, _RULE, _I32] + [_P] * 12 + [_P, _SZ, _P]
_lib.pmpe_backward_scored.restype = _I32
_lib.pmpe_backward_scored.argtypes = [_DESC, _RULE, _I32] + [_P] * 29 + [_P, _SZ, _P]
_lib.pmpe_grad_norm_workspace_bytes.restype = _SZ
_lib.pmpe_grad_norm_workspace_bytes.argtypes = [_P, _I32]
_lib.pmpe_grad_norm.restype = _I32
_lib.pmpe_grad_norm.argtypes = [_P, _P, _P, _I32, ctypes.c_double, _P, _P, _SZ, _P]
_lib.pmpe_clip_grads.restype = _I32
_lib.pmpe_clip_grads.argtypes = [_P, _P, _P, _P, _I32, _P, _P]
_lib.pmpe_adamw_clipped.restype = _I32
_lib.pmpe_adamw_clipped.argtypes = [_P, _I32, _P, _P, _P, _P, ctypes.c_uint64, _I32] + [ctypes.c_float] * 5 + [_P, _P]
_lib.pmpe_expert_ffn_mx_workspace_bytes.restype = _SZ
_lib.pmpe_expert_ffn_mx_workspace_bytes.argtypes = [_DESC, _I32]
_lib.pmpe_expert_ffn_mx.restype = _I32
_lib.pmpe_expert_ffn_mx.argtypes = [_DESC, _I32] + [_P] * 17 + [_P, _SZ, _P]

EXPORTED = ["pmpe_version", "pmpe_status_string", "pmpe_workspace_bytes", "pmpe_check_desc",
            "pmpe_route", "pmpe_dispatch", "pmpe_expert_ffn", "pmpe_combine", "pmpe_audit",
            "pmpe_fingerprint_workspace_bytes", "pmpe_fingerprint", "pmpe_backward_workspace_bytes",
            "pmpe_backward", "pmpe_expert_ffn_train", "pmpe_route_record", "pmpe_cache_tag_check",
            "pmpe_expert_ffn_lora_workspace_bytes", "pmpe_expert_ffn_lora", "pmpe_adamw",
            "pmpe_transpose_experts", "pmpe_expert_ffn_fp8", "pmpe_layer_forward",
            "pmpe_rmsnorm", "pmpe_rmsnorm_backward_workspace_bytes", "pmpe_rmsnorm_backward",
            "pmpe_select", "pmpe_select_backward", "pmpe_route_scored", "pmpe_backward_scored",
            "pmpe_grad_norm_workspace_bytes", "pmpe_grad_norm", "pmpe_clip_grads", "pmpe_adamw_clipped",
            "pmpe_expert_ffn_mx_workspace_bytes", "pmpe_expert_ffn_mx"]

PMPE_FP_LEAF_BYTES = 1024
PMPE_FP_FANOUT = 16


def lib() -> ctypes.CDLL:
    return _lib


def make_desc(hidden: int, inter: int, n_pub: int, n_priv: int, top_k: int, n_shared: int = 0,
              shared_inter: int = 0, bf16: bool = True, gate_mode: int = PMPE_GATE_RENORM_TOPK,
              route_mode: int = 0) -> LayerDesc:
    dt = PMPE_BF16 if bf16 else PMPE_F32
    return LayerDesc(hidden, inter, n_pub, n_priv, top_k, n_shared, shared_inter, dt, dt, gate_mode,
                     route_mode)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libpmpe must be contiguous")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        # (the stream object that the public call makes costs 2.8 us, a third of a small call)
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(status: int, call: str) -> None:
    if status != PMPE_OK:
        raise PmpeError(status, call)


def pmpe_version() -> int:
    return int(_lib.pmpe_version())


def pmpe_workspace_bytes(desc: LayerDesc, T: int) -> int:
    return int(_lib.pmpe_workspace_bytes(ctypes.byref(desc), T))


def pmpe_check_desc(desc: LayerDesc, T: int) -> int:
    return int(_lib.pmpe_check_desc(ctypes.byref(desc), T))


def pmpe_route(desc, T, x, wr_pub, wr_priv, logit_bias, policy_word, topk_idx, topk_gate, allow,
               kgap, dev_status, ws, stream=None) -> None:
    _check(_lib.pmpe_route(ctypes.byref(desc), T, _ptr(x), _ptr(wr_pub), _ptr(wr_priv),
                           _ptr(logit_bias), _ptr(policy_word), _ptr(topk_idx), _ptr(topk_gate),
                           _ptr(allow), _ptr(kgap), _ptr(dev_status), _ptr(ws),
                           0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)),
           "pmpe_route")


def pmpe_dispatch(desc, T, topk_idx, x, expert_count, expert_offset, row_token, token_row, x_perm,
                  ws, stream=None) -> None:
    _check(_lib.pmpe_dispatch(ctypes.byref(desc), T, _ptr(topk_idx), _ptr(x), _ptr(expert_count),
                              _ptr(expert_offset), _ptr(row_token), _ptr(token_row), _ptr(x_perm),
                              _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
                              _stream(stream)), "pmpe_dispatch")


def pmpe_dispatch_noalloc(desc, T, topk_idx, x, expert_count, expert_offset, row_token, token_row,
                          x_perm, stream=None) -> None:
    """pmpe_dispatch with the library's own per-device scratch array (no workspace)."""
    _check(_lib.pmpe_dispatch_noalloc(ctypes.byref(desc), T, _ptr(topk_idx), _ptr(x),
                                      _ptr(expert_count), _ptr(expert_offset), _ptr(row_token),
                                      _ptr(token_row), _ptr(x_perm), _stream(stream)),
           "pmpe_dispatch_noalloc")


def pmpe_expert_ffn(desc, T, x_perm, x, expert_count, expert_offset, row_token, w13_pub, w2_pub,
                    w13_priv, w2_priv, w13_sh, w2_sh, y_shared, y_perm, audit_token_rows,
                    audit_priv_calls, dev_status, ws, stream=None) -> None:
    _check(_lib.pmpe_expert_ffn(
        ctypes.byref(desc), T, _ptr(x_perm), _ptr(x), _ptr(expert_count), _ptr(expert_offset),
        _ptr(row_token), _ptr(w13_pub), _ptr(w2_pub), _ptr(w13_priv), _ptr(w2_priv), _ptr(w13_sh),
        _ptr(w2_sh), _ptr(y_shared), _ptr(y_perm), _ptr(audit_token_rows), _ptr(audit_priv_calls),
        _ptr(dev_status), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
        _stream(stream)), "pmpe_expert_ffn")


def pmpe_combine(desc, T, y_perm, token_row, topk_gate, y_shared, out, stream=None) -> None:
    _check(_lib.pmpe_combine(ctypes.byref(desc), T, _ptr(y_perm), _ptr(token_row), _ptr(topk_gate),
                             _ptr(y_shared), _ptr(out), _stream(stream)), "pmpe_combine")


def pmpe_audit(desc, T, audit_token_rows, allow, req_offset, R, req_private_rows,
               total_private_rows, deny_violations, stream=None) -> None:
    _check(_lib.pmpe_audit(ctypes.byref(desc), T, _ptr(audit_token_rows), _ptr(allow),
                           _ptr(req_offset), R, _ptr(req_private_rows), _ptr(total_private_rows),
                           _ptr(deny_violations), _stream(stream)), "pmpe_audit")


PMPE_FFN_PLAIN = 0
PMPE_FFN_TRAIN = 1
PMPE_FFN_FP8 = 2
_FFN_CALLS = ("pmpe_expert_ffn", "pmpe_expert_ffn_train", "pmpe_expert_ffn_fp8")


def pmpe_layer_forward(desc, T, tensors, R, ffn=PMPE_FFN_PLAIN, stream=None) -> None:
    """The five calls of a layer forward in one: `tensors` in the order of
    ForwardArgs.POINTERS (None where the C call takes NULL). An error names the call."""
    ptrs = [None if t is None else t.data_ptr() if t.is_contiguous() else _ptr(t) for t in tensors]
    ws = tensors[-1]
    a = ForwardArgs(*ptrs, 0 if ws is None else ws.numel() * ws.element_size(), R, ffn, 0)
    status = _lib.pmpe_layer_forward(ctypes.byref(desc), T, ctypes.byref(a), _stream(stream))
    if status != PMPE_OK:
        raise PmpeError(status, ("pmpe_route", "pmpe_dispatch", _FFN_CALLS[ffn], "pmpe_combine",
                                 "pmpe_audit")[a.failed])


def pmpe_backward_workspace_bytes(desc: LayerDesc, T: int) -> int:
    return int(_lib.pmpe_backward_workspace_bytes(ctypes.byref(desc), T))


def pmpe_expert_ffn_train(desc, T, x_perm, x, expert_count, expert_offset, row_token, w13_pub,
                          w2_pub, w13_priv, w2_priv, w13_sh, w2_sh, y_shared, y_perm,
                          audit_token_rows, audit_priv_calls, dev_status, ab, ws,
                          stream=None) -> None:
    _check(_lib.pmpe_expert_ffn_train(
        ctypes.byref(desc), T, _ptr(x_perm), _ptr(x), _ptr(expert_count), _ptr(expert_offset),
        _ptr(row_token), _ptr(w13_pub), _ptr(w2_pub), _ptr(w13_priv), _ptr(w2_priv), _ptr(w13_sh),
        _ptr(w2_sh), _ptr(y_shared), _ptr(y_perm), _ptr(audit_token_rows), _ptr(audit_priv_calls),
        _ptr(dev_status), _ptr(ab), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
        _stream(stream)), "pmpe_expert_ffn_train")


def pmpe_backward(desc, T, x, dout, topk_idx, topk_gate, expert_count, expert_offset, row_token,
                  token_row, y_perm, wr_pub, wr_priv, w13_pub, w2_pub, w13_priv, w2_priv,
                  logit_bias, w13_sh, w2_sh, w2t_pub, w13t_pub, w2t_priv, w13t_priv, ab, dx,
                  dw13_priv, dw2_priv, dwr_priv,
                  grad_rows, ws, stream=None) -> None:
    _check(_lib.pmpe_backward(
        ctypes.byref(desc), T, _ptr(x), _ptr(dout), _ptr(topk_idx), _ptr(topk_gate),
        _ptr(expert_count), _ptr(expert_offset), _ptr(row_token), _ptr(token_row), _ptr(y_perm),
        _ptr(wr_pub), _ptr(wr_priv), _ptr(w13_pub), _ptr(w2_pub), _ptr(w13_priv), _ptr(w2_priv),
        _ptr(logit_bias), _ptr(w13_sh), _ptr(w2_sh), _ptr(w2t_pub), _ptr(w13t_pub),
        _ptr(w2t_priv), _ptr(w13t_priv), _ptr(ab), _ptr(dx), _ptr(dw13_priv), _ptr(dw2_priv), _ptr(dwr_priv), _ptr(grad_rows), _ptr(ws),
        0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)), "pmpe_backward")


def pmpe_fingerprint_workspace_bytes(nbytes: int) -> int:
    return int(_lib.pmpe_fingerprint_workspace_bytes(nbytes))


def pmpe_fingerprint(data: Optional[torch.Tensor], digest: torch.Tensor, ws: Optional[torch.Tensor],
                     nbytes: Optional[int] = None, stream=None) -> None:
    """Fingerprint the bytes of `data` (all of them unless `nbytes` is given) into the
    32-byte device tensor `digest`."""
    if nbytes is None:
        nbytes = 0 if data is None else data.numel() * data.element_size()
    _check(_lib.pmpe_fingerprint(_ptr(data), nbytes, _ptr(digest), _ptr(ws),
                                 0 if ws is None else ws.numel() * ws.element_size(),
                                 _stream(stream)), "pmpe_fingerprint")


def fingerprint_tensors(*tensors: torch.Tensor, stream=None) -> torch.Tensor:
    """One fingerprint of several device tensors: the fingerprint of the concatenation of
    their fingerprints, in argument order. Returns a 32-byte uint8 device tensor."""
    if not tensors:
        raise ValueError("fingerprint_tensors needs at least one tensor")
    dev = tensors[0].device
    digests = torch.empty((len(tensors), 32), dtype=torch.uint8, device=dev)
    ws_bytes = max(pmpe_fingerprint_workspace_bytes(t.numel() * t.element_size()) for t in tensors)
    ws_bytes = max(ws_bytes, pmpe_fingerprint_workspace_bytes(32 * len(tensors)))
    ws = torch.empty(max(ws_bytes, 1), dtype=torch.uint8, device=dev)
    for i, t in enumerate(tensors):
        pmpe_fingerprint(t, digests[i], ws, stream=stream)
    root = torch.empty(32, dtype=torch.uint8, device=dev)
    pmpe_fingerprint(digests, root, ws, stream=stream)
    return root


def pmpe_route_record(desc, T, layer, topk_idx, allow, req_offset, R, rec, stream=None) -> None:
    """rec: [T, 4] int32 device tensor (pmpe_route_rec per token)."""
    _check(_lib.pmpe_route_record(ctypes.byref(desc), T, layer, _ptr(topk_idx), _ptr(allow),
                                  _ptr(req_offset), R, _ptr(rec), _stream(stream)),
           "pmpe_route_record")


def pmpe_cache_tag_check(cache: Optional[CacheTag], request: Optional[CacheTag]) -> bool:
    """True when the cached state may serve the request (every tag field equal)."""
    st = _lib.pmpe_cache_tag_check(None if cache is None else ctypes.byref(cache),
                                   None if request is None else ctypes.byref(request))
    if st not in (PMPE_OK, PMPE_ERR_TAG_MISMATCH):
        raise PmpeError(st, "pmpe_cache_tag_check")
    return st == PMPE_OK


def pmpe_expert_ffn_lora_workspace_bytes(desc: LayerDesc, T: int) -> int:
    return int(_lib.pmpe_expert_ffn_lora_workspace_bytes(ctypes.byref(desc), T))


def pmpe_expert_ffn_lora(desc, T, x_perm, x, expert_count, expert_offset, row_token, policy_word,
                         w13_pub, w2_pub, a13, b1, b3, a2, b2, rank, scale, gate, y_perm,
                         lora_rows, dev_status, ws, stream=None) -> None:
    _check(_lib.pmpe_expert_ffn_lora(
        ctypes.byref(desc), T, _ptr(x_perm), _ptr(x), _ptr(expert_count), _ptr(expert_offset),
        _ptr(row_token), _ptr(policy_word), _ptr(w13_pub), _ptr(w2_pub), _ptr(a13), _ptr(b1),
        _ptr(b3), _ptr(a2), _ptr(b2), rank, scale, gate, _ptr(y_perm), _ptr(lora_rows),
        _ptr(dev_status), _ptr(ws), 0 if ws is None else ws.numel() * ws.element_size(),
        _stream(stream)), "pmpe_expert_ffn_lora")


def pmpe_adamw(param: torch.Tensor, master: Optional[torch.Tensor], grad: torch.Tensor,
               m: torch.Tensor, v: torch.Tensor, step: int, lr: float, beta1: float, beta2: float,
               eps: float, weight_decay: float, stream=None) -> None:
    """One AdamW step of one parameter tensor (fp32, or bf16 with an fp32 master copy)."""
    dt = PMPE_BF16 if param.dtype == torch.bfloat16 else PMPE_F32
    _check(_lib.pmpe_adamw(_ptr(param), dt, _ptr(master), _ptr(grad), _ptr(m), _ptr(v),
                           param.numel(), step, lr, beta1, beta2, eps, weight_decay,
                           _stream(stream)), "pmpe_adamw")


def pmpe_transpose_experts(src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
    """dst[e] = src[e]^T for a bf16 stack src [n, rows, cols] into dst [n, cols, rows]."""
    n, rows, cols = src.shape
    if tuple(dst.shape) != (n, cols, rows):
        raise ValueError("dst must be [n, cols, rows]")
    _check(_lib.pmpe_transpose_experts(_ptr(src), _ptr(dst), n, rows, cols, _stream(stream)),
           "pmpe_transpose_experts")


def pmpe_expert_ffn_fp8(desc, T, x_perm, x, expert_count, expert_offset, row_token, w13_pub,
                        w2_pub, w13_priv, w2_priv, w13s_pub, w2s_pub, w13s_priv, w2s_priv, y_perm,
                        audit_token_rows, audit_priv_calls, dev_status, ws, stream=None) -> None:
    """Expert FFN with fp8 (e4m3, uint8 storage) weights and fp32 power-of-two row scales."""
    _check(_lib.pmpe_expert_ffn_fp8(
        ctypes.byref(desc), T, _ptr(x_perm), _ptr(x), _ptr(expert_count), _ptr(expert_offset),
        _ptr(row_token), _ptr(w13_pub), _ptr(w2_pub), _ptr(w13_priv), _ptr(w2_priv),
        _ptr(w13s_pub), _ptr(w2s_pub), _ptr(w13s_priv), _ptr(w2s_priv), _ptr(y_perm),
        _ptr(audit_token_rows), _ptr(audit_priv_calls), _ptr(dev_status), _ptr(ws),
        0 if ws is None else ws.numel() * ws.element_size(), _stream(stream)), "pmpe_expert_ffn_fp8")


_DTYPES = {torch.float32: PMPE_F32, torch.bfloat16: PMPE_BF16}


def _dtype(t: torch.Tensor, name: str) -> int:
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return _DTYPES[t.dtype]


def _here(t: torch.Tensor, name: str) -> int:
    """The device index of `t`, which has to be the current HIP device: the call's stream is one of its streams."""
    dev = t.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, not on the current HIP device")
    return dev


def _arg(t: Optional[torch.Tensor], name: str, shape, dtype, dev: int) -> Optional[int]:
    """Pointer of `t`, which is None or a contiguous tensor of this shape, one of these types and this device."""
    if t is None:
        return None
    if t.dtype in dtype and t.get_device() == dev and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be a contiguous {list(shape)} of {' or '.join(map(str, dtype))} on device {dev}, "
                     f"not {list(t.shape)} of {t.dtype} on {t.device} with strides {t.stride()}")


def _arg_n(t: Optional[torch.Tensor], name: str, n: int, dtype, dev: int) -> Optional[int]:
    """The same for a tensor of n elements, of any shape."""
    if t is None:
        return None
    if t.dtype in dtype and t.get_device() == dev and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name} must be contiguous, {n} elements of {' or '.join(map(str, dtype))} on device {dev}, "
                     f"not {list(t.shape)} of {t.dtype} on {t.device} with strides {t.stride()}")


def _work(ws: Optional[torch.Tensor], dev: int):
    """Pointer and bytes of a workspace on this device (None and 0 for None)."""
    if ws is None:
        return None, 0
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"the workspace must be contiguous on device {dev}, not on {ws.device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


_F32, _BF16, _U8, _I32T = (torch.float32,), (torch.bfloat16,), (torch.uint8,), (torch.int32,)
_WORDS, _FLOATS = (torch.int32, torch.uint32), tuple(_DTYPES)


def pmpe_rmsnorm(x, residual, weight, eps: float, sum_out, out, out_q, out_scale, rstd, stream=None) -> None:
    """Residual add and RMS norm of x [T, H] (bf16 or fp32): r = x + residual into sum_out,
    the norm of r into out and, in 8 bits, into out_q [T, H] with out_scale [T, H / 32]
    (uint8); each output may be None."""
    dev, shape, act = _here(x, "x"), x.shape, (x.dtype,)
    T, H = shape
    _check(_lib.pmpe_rmsnorm(
        T, H, _dtype(x, "x"), _ptr(x), _arg(residual, "residual", shape, act, dev), _arg(weight, "weight", (H,), _FLOATS, dev),
        _DTYPES[weight.dtype], eps, _arg(sum_out, "sum_out", shape, act, dev), _arg(out, "out", shape, act, dev),
        _arg(out_q, "out_q", shape, _U8, dev), _arg(out_scale, "out_scale", (T, H // 32), _U8, dev),
        _arg(rstd, "rstd", (T,), _F32, dev), _stream(stream)), "pmpe_rmsnorm")


def pmpe_rmsnorm_backward_workspace_bytes(T: int, H: int) -> int:
    return int(_lib.pmpe_rmsnorm_backward_workspace_bytes(T, H))


def pmpe_rmsnorm_backward(dy, dres, r, weight, rstd, dx, dweight, ws, stream=None) -> None:
    """Gradients of pmpe_rmsnorm: dx [T, H] (of r's type) and dweight [H] fp32 or None."""
    dev, shape, act = _here(r, "r"), r.shape, (r.dtype,)
    T, H = shape
    _check(_lib.pmpe_rmsnorm_backward(
        T, H, _dtype(r, "r"), _arg(dy, "dy", shape, (torch.float32, r.dtype), dev), _dtype(dy, "dy"),
        _arg(dres, "dres", shape, act, dev), _ptr(r), _arg(weight, "weight", (H,), _FLOATS, dev), _DTYPES[weight.dtype],
        _arg(rstd, "rstd", (T,), _F32, dev), _arg(dx, "dx", shape, act, dev), _arg(dweight, "dweight", (H,), _F32, dev),
        *_work(ws, dev), _stream(stream)), "pmpe_rmsnorm_backward")


def pmpe_select(desc, rule, T, logits, select_bias, policy_word, topk_idx, topk_gate, topk_logit, allow, margin,
                stream=None) -> None:
    """Selection and gates by `rule` from router logits [T, n_pub + n_priv] (fp32 or bf16)."""
    dev, E, n = _here(logits, "logits"), desc.n_pub + desc.n_priv, T * desc.top_k
    _check(_lib.pmpe_select(
        ctypes.byref(desc), ctypes.byref(rule), T, _arg(logits, "logits", (T, E), _FLOATS, dev), _DTYPES[logits.dtype],
        _arg(select_bias, "select_bias", (E,), _F32, dev), _arg_n(policy_word, "policy_word", T, _WORDS, dev),
        _arg_n(topk_idx, "topk_idx", n, _I32T, dev), _arg_n(topk_gate, "topk_gate", n, _F32, dev),
        _arg_n(topk_logit, "topk_logit", n, _F32, dev), _arg_n(allow, "allow", T, _U8, dev),
        _arg_n(margin, "margin", T, _F32, dev), _stream(stream)), "pmpe_select")


def pmpe_select_backward(desc, rule, T, logits, topk_idx, dgate, dlogits, stream=None) -> None:
    """Gradient dlogits [T, n_pub + n_priv] fp32 of pmpe_select's gates for their gradient dgate."""
    dev, E, n = _here(logits, "logits"), desc.n_pub + desc.n_priv, T * desc.top_k
    _check(_lib.pmpe_select_backward(
        ctypes.byref(desc), ctypes.byref(rule), T, _arg(logits, "logits", (T, E), _FLOATS, dev), _DTYPES[logits.dtype],
        _arg_n(topk_idx, "topk_idx", n, _I32T, dev), _arg_n(dgate, "dgate", n, _F32, dev),
        _arg(dlogits, "dlogits", (T, E), _F32, dev), _stream(stream)), "pmpe_select_backward")


def pmpe_route_scored(desc, rule, T, x, wr_pub, wr_priv, logit_bias, select_bias, policy_word, topk_idx, topk_gate,
                      topk_logit, allow, margin, dev_status, ws, stream=None) -> None:
    """pmpe_route with the selection and gates of a score rule."""
    dev, H, P, n = _here(x, "x"), desc.hidden, desc.n_priv, T * desc.top_k
    E = desc.n_pub + P
    _check(_lib.pmpe_route_scored(
        ctypes.byref(desc), ctypes.byref(rule), T, _arg_n(x, "x", T * H, _BF16 if desc.act_dtype == PMPE_BF16 else _F32, dev),
        _arg_n(wr_pub, "wr_pub", desc.n_pub * H, _F32, dev), _arg_n(wr_priv, "wr_priv", P * H, _F32, dev),
        _arg_n(logit_bias, "logit_bias", E, _F32, dev), _arg_n(select_bias, "select_bias", E, _F32, dev),
        _arg_n(policy_word, "policy_word", T, _WORDS, dev), _arg_n(topk_idx, "topk_idx", n, _I32T, dev),
        _arg_n(topk_gate, "topk_gate", n, _F32, dev), _arg_n(topk_logit, "topk_logit", n, _F32, dev),
        _arg_n(allow, "allow", T, _U8, dev), _arg_n(margin, "margin", T, _F32, dev),
        _arg_n(dev_status, "dev_status", 1, _WORDS, dev), *_work(ws, dev), _stream(stream)), "pmpe_route_scored")


def pmpe_backward_scored(desc, rule, T, topk_logit, x, dout, topk_idx, topk_gate, expert_count, expert_offset,
                         row_token, token_row, y_perm, wr_pub, wr_priv, w13_pub, w2_pub, w13_priv, w2_priv,
                         logit_bias, w13_sh, w2_sh, w2t_pub, w13t_pub, w2t_priv, w13t_priv, ab, dx, dw13_priv,
                         dw2_priv, dwr_priv, grad_rows, ws, stream=None) -> None:
    """pmpe_backward of a layer that routed by `rule` (pmpe_route_scored)."""
    dev, H, I, N, P, n = _here(x, "x"), desc.hidden, desc.inter, desc.n_pub, desc.n_priv, T * desc.top_k
    E, S = N + P, desc.n_shared * desc.shared_inter
    _check(_lib.pmpe_backward_scored(
        ctypes.byref(desc), ctypes.byref(rule), T, _arg_n(topk_logit, "topk_logit", n, _F32, dev),
        _arg_n(x, "x", T * H, _BF16, dev), _arg_n(dout, "dout", T * H, _BF16, dev), _arg_n(topk_idx, "topk_idx", n, _I32T, dev),
        _arg_n(topk_gate, "topk_gate", n, _F32, dev), _arg_n(expert_count, "expert_count", E, _I32T, dev),
        _arg_n(expert_offset, "expert_offset", E + 1, _I32T, dev), _arg_n(row_token, "row_token", n, _I32T, dev),
        _arg_n(token_row, "token_row", n, _I32T, dev), _arg_n(y_perm, "y_perm", n * H, _BF16, dev),
        _arg_n(wr_pub, "wr_pub", N * H, _F32, dev), _arg_n(wr_priv, "wr_priv", P * H, _F32, dev),
        _arg_n(w13_pub, "w13_pub", N * 2 * I * H, _BF16, dev), _arg_n(w2_pub, "w2_pub", N * H * I, _BF16, dev),
        _arg_n(w13_priv, "w13_priv", P * 2 * I * H, _BF16, dev), _arg_n(w2_priv, "w2_priv", P * H * I, _BF16, dev),
        _arg_n(logit_bias, "logit_bias", E, _F32, dev), _arg_n(w13_sh, "w13_sh", 2 * S * H, _BF16, dev),
        _arg_n(w2_sh, "w2_sh", H * S, _BF16, dev), _arg_n(w2t_pub, "w2t_pub", N * I * H, _BF16, dev),
        _arg_n(w13t_pub, "w13t_pub", N * H * 2 * I, _BF16, dev), _arg_n(w2t_priv, "w2t_priv", P * I * H, _BF16, dev),
        _arg_n(w13t_priv, "w13t_priv", P * H * 2 * I, _BF16, dev), _arg_n(ab, "ab", n * 2 * I, _F32, dev),
        _arg_n(dx, "dx", T * H, _F32, dev), _arg_n(dw13_priv, "dw13_priv", P * 2 * I * H, _F32, dev),
        _arg_n(dw2_priv, "dw2_priv", P * H * I, _F32, dev), _arg_n(dwr_priv, "dwr_priv", P * H, _F32, dev),
        _arg_n(grad_rows, "grad_rows", P, _WORDS, dev), *_work(ws, dev), _stream(stream)), "pmpe_backward_scored")


class GradList:
    """A list of gradients (fp32 or bf16 tensors of one device) with the arrays that
    pmpe_grad_norm and pmpe_clip_grads take; a program whose gradients stay in the same
    tensors makes it once (0.13 ms for 500 tensors, where the calls take 28 us). The tensors are kept alive."""

    def __init__(self, tensors) -> None:
        self.tensors = list(tensors)
        n = len(self.tensors)
        types, devices = [t.dtype for t in self.tensors], {t.get_device() for t in self.tensors}
        if not set(types) <= set(_FLOATS):
            raise ValueError("gradients must be float32 or bfloat16")
        if len(devices) > 1:
            raise ValueError("the gradients of a list are on one device")
        if not all([t.is_contiguous() for t in self.tensors]):
            raise ValueError("tensors passed to libpmpe must be contiguous")
        self.device = devices.pop() if n else -1
        self.ptrs = (ctypes.c_uint64 * n).from_buffer(array("Q", [t.data_ptr() for t in self.tensors]))
        self.sizes = (ctypes.c_uint64 * n).from_buffer(array("Q", [t.numel() for t in self.tensors]))
        self.dtypes = (_I32 * n).from_buffer(array("i", [_DTYPES[d] for d in types]))
        self.key = (bytes(self.sizes), bytes(self.dtypes))

    def __len__(self) -> int:
        return len(self.tensors)

    @classmethod
    def of(cls, grads) -> "GradList":
        return grads if isinstance(grads, cls) else cls(grads)


def pmpe_grad_norm_workspace_bytes(grads) -> int:
    g = GradList.of(grads)
    return int(_lib.pmpe_grad_norm_workspace_bytes(g.sizes, len(g)))


def _grad_args(grads, norm: torch.Tensor):
    """The list of gradients, the norm's pointer and their device."""
    g, dev = GradList.of(grads), _here(norm, "norm")
    if len(g) and g.device != dev:
        raise ValueError(f"the gradients are on {g.tensors[0].device}, not on device {dev}")
    return g, _arg(norm, "norm", (2,), _F32, dev), dev


def pmpe_grad_norm(grads, max_norm: float, norm: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """Global norm of the gradients (a GradList or tensors) and the factor that clips them to
    max_norm, into norm [2] fp32."""
    g, np, dev = _grad_args(grads, norm)
    _check(_lib.pmpe_grad_norm(g.ptrs, g.sizes, g.dtypes, len(g), max_norm, np, *_work(ws, dev), _stream(stream)),
           "pmpe_grad_norm")


def pmpe_clip_grads(grads, outs, norm: torch.Tensor, stream=None) -> None:
    """The gradients times the factor of pmpe_grad_norm, into `outs` (None: in place)."""
    g, np, dev = _grad_args(grads, norm)
    o = None
    if outs is not None:
        o = GradList.of(outs)
        if o.key != g.key or (len(o) and o.device != dev):
            raise ValueError("outs must be tensors of the gradients' sizes and types on their device")
    _check(_lib.pmpe_clip_grads(g.ptrs, None if o is None else o.ptrs, g.sizes, g.dtypes, len(g), np, _stream(stream)),
           "pmpe_clip_grads")


def pmpe_adamw_clipped(param: torch.Tensor, master: Optional[torch.Tensor], grad: torch.Tensor,
                       m: torch.Tensor, v: torch.Tensor, step: int, lr: float, beta1: float, beta2: float,
                       eps: float, weight_decay: float, norm: torch.Tensor, stream=None) -> None:
    """pmpe_adamw on the gradient times the factor that pmpe_grad_norm wrote to `norm`."""
    dev, n = _here(norm, "norm"), param.numel()
    _check(_lib.pmpe_adamw_clipped(
        _arg_n(param, "param", n, _FLOATS, dev), _DTYPES[param.dtype], _arg_n(master, "master", n, _F32, dev),
        _arg_n(grad, "grad", n, _F32, dev), _arg_n(m, "m", n, _F32, dev), _arg_n(v, "v", n, _F32, dev), n, step, lr, beta1,
        beta2, eps, weight_decay, _arg(norm, "norm", (2,), _F32, dev), _stream(stream)), "pmpe_adamw_clipped")


def pmpe_expert_ffn_mx_workspace_bytes(desc: LayerDesc, T: int) -> int:
    return int(_lib.pmpe_expert_ffn_mx_workspace_bytes(ctypes.byref(desc), T))


def pmpe_expert_ffn_mx(desc, T, xq, xs, expert_count, expert_offset, row_token, w13_pub, w2_pub, w13_priv, w2_priv,
                       w13s_pub, w2s_pub, w13s_priv, w2s_priv, y_perm, audit_token_rows, audit_priv_calls,
                       dev_status, ws, stream=None) -> None:
    """Expert FFN on 8-bit activations xq [T, H] with block scales xs [T, H / 32] (both uint8,
    as pmpe_rmsnorm writes them) and 8-bit weights with row scales."""
    dev, H, n = _here(xq, "xq"), desc.hidden, T * desc.top_k
    P, E = desc.n_priv, desc.n_pub + desc.n_priv
    wt = [_arg_n(t, name, cnt * rows * cols, _U8, dev) for t, name, cnt, rows, cols in (
        (w13_pub, "w13_pub", desc.n_pub, 2 * desc.inter, H), (w2_pub, "w2_pub", desc.n_pub, H, desc.inter),
        (w13_priv, "w13_priv", P, 2 * desc.inter, H), (w2_priv, "w2_priv", P, H, desc.inter))]
    ws_ = [_arg_n(t, name, cnt * rows, _F32, dev) for t, name, cnt, rows in (
        (w13s_pub, "w13s_pub", desc.n_pub, 2 * desc.inter), (w2s_pub, "w2s_pub", desc.n_pub, H),
        (w13s_priv, "w13s_priv", P, 2 * desc.inter), (w2s_priv, "w2s_priv", P, H))]
    _check(_lib.pmpe_expert_ffn_mx(
        ctypes.byref(desc), T, _arg(xq, "xq", (T, H), _U8, dev), _arg(xs, "xs", (T, H // 32), _U8, dev),
        _arg_n(expert_count, "expert_count", E, _I32T, dev), _arg_n(expert_offset, "expert_offset", E + 1, _I32T, dev),
        _arg_n(row_token, "row_token", n, _I32T, dev), *wt, *ws_, _arg_n(y_perm, "y_perm", n * H, _BF16, dev),
        _arg_n(audit_token_rows, "audit_token_rows", T, _WORDS, dev), _arg_n(audit_priv_calls, "audit_priv_calls", P, _WORDS, dev),
        _arg_n(dev_status, "dev_status", 1, _WORDS, dev), *_work(ws, dev), _stream(stream)), "pmpe_expert_ffn_mx")
