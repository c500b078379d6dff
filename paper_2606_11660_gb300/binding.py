"""Thin ctypes binding of the C ABI in include/bergson.h.

Each ``bergson_*`` function here has the name of the C entry point it calls
and only marshals arguments: torch tensors become device pointers and leading
dimensions, ``stream=None`` becomes torch's current stream.  All computation
happens in the CUDA library; if the library is missing, loading it raises.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os
import struct
from typing import Optional, Sequence

_PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG_DIR, "libbergson.so")

BERGSON_OK = 0
BERGSON_EINVAL = -1
BERGSON_EALIGN = -2
BERGSON_EUNSUPPORTED = -3
BERGSON_EWORKSPACE = -4
BERGSON_ECUDA = -5
BERGSON_EDEVICE_TIMEOUT = -6
BERGSON_EMOMENT = -7

BERGSON_PROJ_GAUSSIAN = 0
BERGSON_PROJ_IDENTITY = 1
BERGSON_PROJ_RADEMACHER = 2
BERGSON_PROJ_UNIFORM = 3

BERGSON_LAYER_BIAS = 1

BERGSON_AGG_SUM = 0
BERGSON_AGG_MEAN = 1

BERGSON_FISHER_INV_SQRT = 0
BERGSON_FISHER_INV = 1

BERGSON_F32 = 0
BERGSON_BF16 = 1
BERGSON_F16 = 2

BERGSON_POLICY_TOKEN_MEAN = 0
BERGSON_POLICY_SEQ_MEAN = 1
BERGSON_POLICY_SUM_NORM = 2

BERGSON_PREFERENCE_SIGMOID = 0
BERGSON_PREFERENCE_HINGE = 1
BERGSON_PREFERENCE_SQUARED = 2

BERGSON_STATE_F32 = 0
BERGSON_STATE_8BIT = 1
BERGSON_STATE_BLOCK = 256

BERGSON_NORM_LAYER = 0
BERGSON_NORM_RMS = 1

BERGSON_MOMENT_FIRST = 0
BERGSON_MOMENT_SECOND = 1

STATUS_NAMES = {
    0: "BERGSON_OK", -1: "BERGSON_EINVAL", -2: "BERGSON_EALIGN", -3: "BERGSON_EUNSUPPORTED",
    -4: "BERGSON_EWORKSPACE", -5: "BERGSON_ECUDA", -6: "BERGSON_EDEVICE_TIMEOUT",
    -7: "BERGSON_EMOMENT",
}

# Every symbol include/bergson.h declares.
EXPORTED = (
    "bergson_project_grads_workspace", "bergson_project_grads", "bergson_build_store",
    "bergson_score_topk_workspace", "bergson_score_topk", "bergson_score_bottomk",
    "bergson_projection_matrix",
    "bergson_module_seeds", "bergson_sync_status", "bergson_last_error", "bergson_version",
    "bergson_debug_wait_probe", "bergson_debug_inject_status", "bergson_debug_project_plan",
    "bergson_debug_score_plan", "bergson_debug_score_launches", "bergson_debug_xgemm_plan",
    "bergson_project_grads_noalloc",
    "bergson_score_grads_workspace", "bergson_score_grads", "bergson_token_scores_workspace",
    "bergson_token_scores", "bergson_aggregate_rows_workspace", "bergson_aggregate_rows",
    "bergson_fisher_fit_workspace", "bergson_fisher_fit", "bergson_fisher_preconditioner_workspace",
    "bergson_fisher_preconditioner", "bergson_precondition_rows", "bergson_store_save",
    "bergson_store_load", "bergson_fisher_preconditioner_tol", "bergson_debug_attr_once",
    "bergson_build_store_blocks", "bergson_score_topk_update_workspace",
    "bergson_score_topk_update", "bergson_score_bottomk_update",
    "bergson_score_topk_host_workspace", "bergson_score_topk_host",
    "bergson_token_logprobs", "bergson_token_logprobs_backward", "bergson_policy_loss_workspace",
    "bergson_policy_loss", "bergson_preference_loss", "bergson_adamw_step",
    "bergson_adamw_state_values", "bergson_factor_moments_workspace", "bergson_factor_moments",
    "bergson_norm", "bergson_norm_backward_workspace", "bergson_norm_backward",
    "bergson_embedding", "bergson_embedding_backward_workspace", "bergson_embedding_backward",
    "bergson_muon_step_workspace", "bergson_muon_step",
)


class BergsonError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class bergson_layer(ctypes.Structure):
    _fields_ = [
        ("A", ctypes.c_void_p), ("G", ctypes.c_void_p),
        ("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64),
        ("k_in", ctypes.c_int64), ("k_out", ctypes.c_int64),
        ("seed_in", ctypes.c_uint64), ("seed_out", ctypes.c_uint64),
        ("proj_kind", ctypes.c_int32), ("flags", ctypes.c_int32),
        ("r", ctypes.c_void_p), ("c", ctypes.c_void_p),
        ("out_col_offset", ctypes.c_int64), ("bias_col_offset", ctypes.c_int64),
    ]


class bergson_policy_args(ctypes.Structure):
    _fields_ = (
        [(n, ctypes.c_void_p) for n in ("logp", "old_logp", "ref_logp", "entropy", "advantages",
                                        "mask")]
        + [(n, ctypes.c_int64) for n in ("ld_logp", "ld_old", "ld_ref", "ld_entropy", "ld_adv",
                                         "ld_mask", "B", "T")]
        + [(n, ctypes.c_double) for n in ("clip_low", "clip_high", "kl_coef", "entropy_coef",
                                          "norm_tokens")]
        + [(n, ctypes.c_void_p) for n in ("loss", "seq_loss", "stats", "d_logp", "d_entropy")]
        + [("ld_d", ctypes.c_int64), ("ld_de", ctypes.c_int64), ("reduction", ctypes.c_int32),
           ("reserved", ctypes.c_int32)])


class bergson_preference_args(ctypes.Structure):
    _fields_ = (
        [(n, ctypes.c_void_p) for n in ("logp", "ref_logp", "mask")]
        + [(n, ctypes.c_int64) for n in ("ld_logp", "ld_ref", "ld_mask", "P", "T")]
        + [(n, ctypes.c_double) for n in ("beta", "margin", "label_smoothing")]
        + [(n, ctypes.c_void_p) for n in ("loss", "pair_loss", "rewards", "d_logp")]
        + [("ld_d", ctypes.c_int64), ("kind", ctypes.c_int32), ("mean_logp", ctypes.c_int32)])


# The records' fields, packed at once: as arguments of the ctypes classes they take twice the time.
_POLICY_RECORD = struct.Struct("=6Q8q5d5Q2q2i")
_PREFERENCE_RECORD = struct.Struct("=3Q5q3d4Qq2i")
_NORM_RECORD = struct.Struct("=6Q4qd4i")
_NORM_GRAD_RECORD = struct.Struct("=8Q5q4i")
_EMBEDDING_RECORD = struct.Struct("=3Q5qd2i")
_EMBEDDING_GRAD_RECORD = struct.Struct("=3Q5qd4i")


class bergson_adamw_tensor(ctypes.Structure):
    _fields_ = (
        [(n, ctypes.c_void_p) for n in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")]
        + [("n", ctypes.c_int64), ("lr_scale", ctypes.c_float), ("weight_decay", ctypes.c_float)]
        + [(n, ctypes.c_int32) for n in ("param_dtype", "grad_dtype", "state_kind", "reserved")])


class bergson_moment_matrix(ctypes.Structure):
    _fields_ = [
        ("v", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("d_out", ctypes.c_int64),
        ("d_in", ctypes.c_int64), ("r", ctypes.c_void_p), ("c", ctypes.c_void_p),
        ("state_kind", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class bergson_muon_tensor(ctypes.Structure):
    _fields_ = (
        [(n, ctypes.c_void_p) for n in ("param", "grad", "master", "m")]
        + [("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]
        + [(n, ctypes.c_float) for n in ("lr_scale", "ortho_scale", "weight_decay")]
        + [(n, ctypes.c_int32) for n in ("param_dtype", "grad_dtype", "reserved")])


_LIB = None


def lib() -> ctypes.CDLL:
    """The loaded library (raises if it was not built)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    i64, u64, vp, i32 = ctypes.c_int64, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_int
    f64 = ctypes.c_double
    szp = ctypes.POINTER(ctypes.c_size_t)
    i64p = ctypes.POINTER(ctypes.c_int64)
    lp = ctypes.POINTER(bergson_layer)
    sig = {
        "bergson_project_grads_workspace": (i32, [lp, i32, i64, i64, szp]),
        "bergson_project_grads": (i32, [lp, i32, i64, i64, vp, vp, i64, vp, ctypes.c_size_t, vp]),
        "bergson_build_store": (i32, [vp, i64, i64, i64, i32, vp, i64, i64, i64, vp, vp]),
        "bergson_build_store_blocks": (i32, [vp, i64, i64, i64, i64p, i32, vp, i64, i64, i64,
                                             vp, vp]),
        "bergson_score_topk_workspace": (i32, [i64, i64, i64, i64, szp]),
        "bergson_score_topk": (i32, [vp, i64, i64, i64, vp, i64, i64, i64, vp, vp, vp,
                                     ctypes.c_size_t, vp]),
        "bergson_score_bottomk": (i32, [vp, i64, i64, i64, vp, i64, i64, i64, vp, vp, vp,
                                        ctypes.c_size_t, vp]),
        "bergson_score_topk_update_workspace": (i32, [i64, i64, i64, szp]),
        "bergson_score_topk_update": (i32, [vp, i64, i64, i64, i64, vp, i64, i64, i64, i32, vp,
                                            vp, vp, ctypes.c_size_t, vp]),
        "bergson_score_bottomk_update": (i32, [vp, i64, i64, i64, i64, vp, i64, i64, i64, i32,
                                               vp, vp, vp, ctypes.c_size_t, vp]),
        "bergson_score_topk_host_workspace": (i32, [i64, i64, i64, i64, szp]),
        "bergson_score_topk_host": (i32, [vp, i64, i64, i64, vp, i64, i64, i64, i32, i64, vp,
                                          vp, vp, ctypes.c_size_t, vp, vp]),
        "bergson_projection_matrix": (i32, [u64, i64, i64, i32, vp, vp, vp]),
        "bergson_module_seeds": (None, [u64, i64, ctypes.POINTER(u64), ctypes.POINTER(u64)]),
        "bergson_sync_status": (i32, [vp]),
        "bergson_last_error": (ctypes.c_char_p, []),
        "bergson_version": (i32, []),
        "bergson_debug_wait_probe": (i32, [u64, vp]),
        "bergson_debug_inject_status": (None, [i32, i32]),
        "bergson_debug_project_plan": (i32, [lp, i32, i64, i64, i64p, i64p, i64p, i64p]),
        "bergson_debug_score_plan": (i32, [i64, i64, i64, i64, i32, i64p, i32,
                                           ctypes.POINTER(i32)]),
        "bergson_debug_score_launches": (i32, [i64, i64, i64, i64, i32, i64p, i32,
                                               ctypes.POINTER(i32)]),
        "bergson_debug_xgemm_plan": (i32, [i64, i64, i64, i64p, i32]),
        "bergson_debug_attr_once": (i32, [i32, i32, i32, i64p, ctypes.POINTER(i32)]),
        "bergson_project_grads_noalloc": (i32, [lp, i32, i64, i64, vp, vp, i64, vp]),
        "bergson_score_grads_workspace": (i32, [i64, i64, i64, szp]),
        "bergson_token_scores_workspace": (i32, [lp, i32, i64, i64, i64, szp]),
        "bergson_aggregate_rows_workspace": (i32, [i64, szp]),
        "bergson_store_save": (i32, [vp, i64, i64, i64, ctypes.c_char_p, i64, vp]),
        "bergson_store_load": (i32, [ctypes.c_char_p, i64, i64, i64, vp, i64, vp]),
        "bergson_fisher_fit_workspace": (i32, [i64, i64, szp]),
        "bergson_fisher_fit": (i32, [vp, i64, i64, i64, vp, i64, vp, ctypes.c_size_t, vp]),
        "bergson_fisher_preconditioner_workspace": (i32, [i64, szp]),
        "bergson_fisher_preconditioner": (i32, [vp, vp, i64, i64, ctypes.c_float, ctypes.c_float,
                                                i32, i32, vp, i64, vp, ctypes.c_size_t, vp]),
        "bergson_fisher_preconditioner_tol": (i32, [vp, vp, i64, i64, ctypes.c_float,
                                                    ctypes.c_float, i32, i32, ctypes.c_float, vp,
                                                    i64, vp, ctypes.c_size_t,
                                                    ctypes.POINTER(ctypes.c_float),
                                                    ctypes.POINTER(i32), vp]),
        "bergson_precondition_rows": (i32, [vp, i64, i64, i64, vp, i64, vp, i64, vp,
                                            ctypes.c_size_t, vp]),
        "bergson_aggregate_rows": (i32, [vp, i64, i64, i64, vp, i64, i32, i32, vp, i64, vp,
                                         ctypes.c_size_t, vp]),
        "bergson_token_scores": (i32, [lp, i32, i64, i64, vp, vp, i64, i64, vp, vp,
                                       ctypes.c_size_t, vp]),
        "bergson_score_grads": (i32, [vp, i64, i64, i64, vp, i64, i64, i32, vp, i64, vp,
                                      ctypes.c_size_t, vp]),
        "bergson_token_logprobs": (i32, [vp, i32, i64, i64, i64, vp, f64, vp, vp, vp, vp]),
        "bergson_token_logprobs_backward": (i32, [vp, i32, i64, i64, i64, vp, f64, vp, vp, vp, vp,
                                                  vp, i64, vp]),
        "bergson_policy_loss_workspace": (i32, [i64, i64, szp]),
        "bergson_policy_loss": (i32, [ctypes.POINTER(bergson_policy_args), vp, ctypes.c_size_t,
                                      vp]),
        "bergson_preference_loss": (i32, [ctypes.POINTER(bergson_preference_args), vp]),
        "bergson_adamw_step": (i32, [ctypes.POINTER(bergson_adamw_tensor), i32, f64, f64, f64, f64,
                                     i64, u64, vp, vp]),
        "bergson_adamw_state_values": (i32, [vp, vp, i64, i32, vp, vp]),
        "bergson_factor_moments_workspace": (i32, [ctypes.POINTER(bergson_moment_matrix), i32,
                                                   szp]),
        "bergson_factor_moments": (i32, [ctypes.POINTER(bergson_moment_matrix), i32, f64, f64, vp,
                                         ctypes.c_size_t, vp]),
        # records, as bytes
        "bergson_norm": (i32, [ctypes.c_char_p, vp]),
        "bergson_norm_backward_workspace": (i32, [i64, i64, szp]),
        "bergson_norm_backward": (i32, [ctypes.c_char_p, vp, ctypes.c_size_t, vp]),
        "bergson_embedding": (i32, [ctypes.c_char_p, vp]),
        "bergson_embedding_backward_workspace": (i32, [i64, i64, i64, szp]),
        "bergson_embedding_backward": (i32, [ctypes.c_char_p, vp, ctypes.c_size_t, vp]),
        "bergson_muon_step_workspace": (i32, [ctypes.POINTER(bergson_muon_tensor), i32, i32, szp]),
        "bergson_muon_step": (i32, [ctypes.POINTER(bergson_muon_tensor), i32, f64, f64, i32,
                                    ctypes.POINTER(f64), i32, i32, vp, vp, ctypes.c_size_t, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = L
    return L


def bergson_last_error() -> str:
    return lib().bergson_last_error().decode()


def _check(status: int) -> None:
    if status != BERGSON_OK:
        raise BergsonError(status, bergson_last_error())


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    return t.data_ptr() if hasattr(t, "data_ptr") else int(t)


_raw_stream = None


def _current_stream() -> int:
    """torch's current stream on the current device, without building the
    Stream object that torch.cuda.current_stream() returns (3 us a call)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()                       # initialises CUDA
        raw, dev = (getattr(torch._C, n, None)
                    for n in ("_cuda_getCurrentRawStream", "_cuda_getDevice"))
        _raw_stream = ((lambda: raw(dev())) if raw is not None and dev is not None
                       else (lambda: torch.cuda.current_stream().cuda_stream))
    return _raw_stream()


def _stream(stream) -> Optional[int]:
    if stream is None:
        return _current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


@dataclasses.dataclass
class Layer:
    """One nn.Linear's captured tensors: A [B,T,d_in] bf16, G [B,T,d_out] bf16."""
    A: object
    G: object
    k_in: int
    k_out: int
    seed_in: int
    seed_out: int
    r: object = None
    c: object = None
    out_col_offset: int = 0
    proj_kind: int = BERGSON_PROJ_GAUSSIAN
    bias_col_offset: Optional[int] = None     # set to also write the projected bias gradient

    def to_c(self) -> bergson_layer:
        bias = self.bias_col_offset
        # in the order of bergson_layer._fields_
        return bergson_layer(
            _ptr(self.A), _ptr(self.G), int(self.A.shape[-1]), int(self.G.shape[-1]),
            int(self.k_in), int(self.k_out), int(self.seed_in), int(self.seed_out),
            int(self.proj_kind), 0 if bias is None else BERGSON_LAYER_BIAS,
            None if self.r is None else _ptr(self.r), None if self.c is None else _ptr(self.c),
            int(self.out_col_offset), 0 if bias is None else int(bias))


def _layer_array(layers: Sequence) -> "ctypes.Array":
    arr = (bergson_layer * len(layers))()
    for i, ly in enumerate(layers):
        arr[i] = ly if isinstance(ly, bergson_layer) else ly.to_c()
    return arr


def bergson_module_seeds(base_seed: int, module_index: int) -> tuple[int, int]:
    a, b = ctypes.c_uint64(), ctypes.c_uint64()
    lib().bergson_module_seeds(int(base_seed), int(module_index), ctypes.byref(a), ctypes.byref(b))
    return a.value, b.value


def bergson_project_grads_workspace(layers: Sequence, B: int, T: int) -> int:
    arr = _layer_array(layers)
    n = ctypes.c_size_t()
    _check(lib().bergson_project_grads_workspace(arr, len(layers), int(B), int(T), ctypes.byref(n)))
    return n.value


def bergson_project_grads(layers: Sequence, B: int, T: int, mask, out, workspace,
                          stream=None, ld_out: Optional[int] = None) -> None:
    arr = _layer_array(layers)
    ld = int(out.stride(0)) if ld_out is None else int(ld_out)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().bergson_project_grads(arr, len(layers), int(B), int(T), _ptr(mask), _ptr(out), ld,
                                       _ptr(workspace), ws_bytes, _stream(stream)))


def bergson_project_grads_noalloc(layers: Sequence, B: int, T: int, mask, out, stream=None,
                                  ld_out: Optional[int] = None) -> None:
    """Like bergson_project_grads, but on the library's fixed static scratch (no workspace)."""
    arr = _layer_array(layers)
    ld = int(out.stride(0)) if ld_out is None else int(ld_out)
    _check(lib().bergson_project_grads_noalloc(arr, len(layers), int(B), int(T), _ptr(mask),
                                               _ptr(out), ld, _stream(stream)))


def bergson_build_store(proj, B: int, K: int, unit_normalize: bool, store, row_offset: int,
                        norms_out=None, stream=None) -> None:
    _check(lib().bergson_build_store(_ptr(proj), int(B), int(K), int(proj.stride(0)),
                                     1 if unit_normalize else 0, _ptr(store), int(store.stride(0)),
                                     int(row_offset), int(store.shape[0]), _ptr(norms_out),
                                     _stream(stream)))


def bergson_build_store_blocks(proj, B: int, K: int, block_offsets: Sequence[int], store,
                               row_offset: int, norms_out=None, stream=None) -> None:
    """Store rows with each column block [o_j, o_j+1) unit-normalised on its own."""
    n = len(block_offsets) - 1
    offs = (ctypes.c_int64 * max(1, n + 1))(*[int(v) for v in block_offsets])
    _check(lib().bergson_build_store_blocks(_ptr(proj), int(B), int(K), int(proj.stride(0)), offs,
                                            n, _ptr(store), int(store.stride(0)), int(row_offset),
                                            int(store.shape[0]), _ptr(norms_out), _stream(stream)))


def bergson_score_topk_workspace(N: int, K: int, Q: int, topk: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().bergson_score_topk_workspace(int(N), int(K), int(Q), int(topk), ctypes.byref(n)))
    return n.value


def bergson_score_topk(store, N: int, K: int, queries, topk: int, out_scores, out_idx, workspace,
                       stream=None) -> None:
    Q = int(queries.shape[0])
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().bergson_score_topk(_ptr(store), int(N), int(K), int(store.stride(0)),
                                    _ptr(queries), Q, int(queries.stride(0)), int(topk),
                                    _ptr(out_scores), _ptr(out_idx), _ptr(workspace), ws_bytes,
                                    _stream(stream)))


def bergson_score_bottomk(store, N: int, K: int, queries, bottomk: int, out_scores, out_idx,
                          workspace, stream=None) -> None:
    """The bottomk least similar store rows per query, lowest score first."""
    Q = int(queries.shape[0])
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().bergson_score_bottomk(_ptr(store), int(N), int(K), int(store.stride(0)),
                                       _ptr(queries), Q, int(queries.stride(0)), int(bottomk),
                                       _ptr(out_scores), _ptr(out_idx), _ptr(workspace), ws_bytes,
                                       _stream(stream)))


def bergson_score_topk_update_workspace(K: int, Q: int, topk: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().bergson_score_topk_update_workspace(int(K), int(Q), int(topk), ctypes.byref(n)))
    return n.value


def bergson_score_topk_update(store, N: int, K: int, row_base: int, queries, topk: int, init: bool,
                              scores, idx, workspace, stream=None, least: bool = False) -> None:
    """Merge the top-k (least: bottom-k) of store rows [row_base, row_base + N)
    (store[0:N] on the device) into the running result scores/idx [Q, topk]."""
    Q = int(queries.shape[0])
    fn = lib().bergson_score_bottomk_update if least else lib().bergson_score_topk_update
    _check(fn(_ptr(store), int(N), int(K), int(store.stride(0)), int(row_base), _ptr(queries), Q,
              int(queries.stride(0)), int(topk), 1 if init else 0, _ptr(scores), _ptr(idx),
              _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def bergson_score_topk_host_workspace(chunk_rows: int, K: int, Q: int, topk: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().bergson_score_topk_host_workspace(int(chunk_rows), int(K), int(Q), int(topk),
                                                   ctypes.byref(n)))
    return n.value


def bergson_score_topk_host(host_store, N: int, K: int, queries, topk: int, chunk_rows: int,
                            out_scores, out_idx, workspace, stream=None, copy_stream=None,
                            least: bool = False) -> None:
    """Exact top-k (least: bottom-k) of a store in host memory (a CPU tensor,
    ideally pinned), streamed to the device in chunks of chunk_rows rows."""
    Q = int(queries.shape[0])
    cs = None if copy_stream is None else _stream(copy_stream)
    _check(lib().bergson_score_topk_host(
        _ptr(host_store), int(N), int(K), int(host_store.stride(0)), _ptr(queries), Q,
        int(queries.stride(0)), int(topk), 1 if least else 0, int(chunk_rows), _ptr(out_scores),
        _ptr(out_idx), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream), cs))


def bergson_token_scores_workspace(layers: Sequence, B: int, T: int, n_queries: int) -> int:
    arr = _layer_array(layers)
    n = ctypes.c_size_t()
    _check(lib().bergson_token_scores_workspace(arr, len(layers), int(B), int(T), int(n_queries),
                                                ctypes.byref(n)))
    return n.value


def bergson_token_scores(layers: Sequence, B: int, T: int, mask, queries, out, workspace,
                         stream=None) -> None:
    """Per-token scores out[q, b, t] of every token against each query row."""
    arr = _layer_array(layers)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().bergson_token_scores(arr, len(layers), int(B), int(T), _ptr(mask), _ptr(queries),
                                      int(queries.shape[0]), int(queries.stride(0)), _ptr(out),
                                      _ptr(workspace), ws_bytes, _stream(stream)))


def bergson_aggregate_rows_workspace(n: int) -> int:
    m = ctypes.c_size_t()
    _check(lib().bergson_aggregate_rows_workspace(int(n), ctypes.byref(m)))
    return m.value


def bergson_aggregate_rows(rows, n: int, K: int, offsets, mode: int, normalize_each: bool, out,
                           workspace=None, stream=None) -> None:
    """out[g] = sum/mean of rows[offsets[g]:offsets[g+1]] (offsets: device int64 [G+1])."""
    G = int(offsets.shape[0]) - 1
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().bergson_aggregate_rows(_ptr(rows), int(n), int(K), int(rows.stride(0)),
                                        _ptr(offsets), G, int(mode), 1 if normalize_each else 0,
                                        _ptr(out), int(out.stride(0)), _ptr(workspace), ws_bytes,
                                        _stream(stream)))


def bergson_fisher_fit_workspace(n: int, K: int) -> int:
    m = ctypes.c_size_t()
    _check(lib().bergson_fisher_fit_workspace(int(n), int(K), ctypes.byref(m)))
    return m.value


def bergson_fisher_fit(rows, n: int, K: int, R, workspace, stream=None) -> None:
    """R = (1/n) sum_i rows[i] rows[i]^T (empirical Fisher of projected gradients)."""
    _check(lib().bergson_fisher_fit(_ptr(rows), int(n), int(K), int(rows.stride(0)), _ptr(R),
                                    int(R.stride(0)), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream(stream)))


def bergson_fisher_preconditioner_workspace(K: int) -> int:
    m = ctypes.c_size_t()
    _check(lib().bergson_fisher_preconditioner_workspace(int(K), ctypes.byref(m)))
    return m.value


def bergson_fisher_preconditioner(R1, R2, K: int, lam: float, damping: float, power: int,
                                  iterations: int, M, workspace, stream=None) -> None:
    """M = (lam R1 + (1-lam) R2 + damping tr/K I)^-1/2 (or ^-1)."""
    _check(lib().bergson_fisher_preconditioner(
        _ptr(R1), _ptr(R2), int(K), int(R1.stride(0)), float(lam), float(damping), int(power),
        int(iterations), _ptr(M), int(M.stride(0)), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def bergson_fisher_preconditioner_tol(R1, R2, K: int, lam: float, damping: float, power: int,
                                      max_iterations: int, tol: float, M, workspace,
                                      stream=None) -> tuple[int, list]:
    """As bergson_fisher_preconditioner, stopping at the first iterate whose
    residual ||I - Z Y||_F / sqrt(K) is <= tol.  Returns (updates applied,
    residuals of the iterates computed)."""
    res = (ctypes.c_float * (int(max_iterations) + 1))(*([float("nan")] * (int(max_iterations) + 1)))
    done = ctypes.c_int()
    _check(lib().bergson_fisher_preconditioner_tol(
        _ptr(R1), _ptr(R2), int(K), int(R1.stride(0)), float(lam), float(damping), int(power),
        int(max_iterations), float(tol), _ptr(M), int(M.stride(0)), _ptr(workspace),
        workspace.numel() * workspace.element_size(), res, ctypes.byref(done), _stream(stream)))
    vals = [float(v) for v in res]
    return done.value, [v for v in vals if v == v]


def bergson_precondition_rows(rows, B: int, K: int, M, out, workspace, stream=None) -> None:
    """out[b] = M rows[b] (M symmetric K x K)."""
    _check(lib().bergson_precondition_rows(_ptr(rows), int(B), int(K), int(rows.stride(0)),
                                           _ptr(M), int(M.stride(0)), _ptr(out),
                                           int(out.stride(0)), _ptr(workspace),
                                           workspace.numel() * workspace.element_size(),
                                           _stream(stream)))


def bergson_store_save(store, rows: int, K: int, path: str, file_row_offset: int = 0,
                       stream=None) -> None:
    """Write device store rows [0, rows) to the raw fp16 store file at path."""
    _check(lib().bergson_store_save(_ptr(store), int(rows), int(K), int(store.stride(0)),
                                    os.fsencode(path), int(file_row_offset), _stream(stream)))


def bergson_store_load(path: str, file_row_offset: int, rows: int, K: int, store,
                       stream=None) -> None:
    """Read file rows [file_row_offset, +rows) into device store rows [0, rows)."""
    _check(lib().bergson_store_load(os.fsencode(path), int(file_row_offset), int(rows), int(K),
                                    _ptr(store), int(store.stride(0)), _stream(stream)))


def bergson_score_grads_workspace(B: int, K: int, Q: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().bergson_score_grads_workspace(int(B), int(K), int(Q), ctypes.byref(n)))
    return n.value


def bergson_score_grads(proj, B: int, K: int, queries, unit_normalize: bool, scores, workspace,
                        stream=None) -> None:
    """On-the-fly scores of B projected rows against Q projected queries."""
    Q = int(queries.shape[0])
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib().bergson_score_grads(_ptr(proj), int(B), int(K), int(proj.stride(0)),
                                     _ptr(queries), Q, int(queries.stride(0)),
                                     1 if unit_normalize else 0, _ptr(scores),
                                     int(scores.stride(0)), _ptr(workspace), ws_bytes,
                                     _stream(stream)))


def bergson_projection_matrix(seed: int, d: int, k: int, proj_kind: int, moment, out,
                              stream=None) -> None:
    _check(lib().bergson_projection_matrix(int(seed), int(d), int(k), int(proj_kind), _ptr(moment),
                                           _ptr(out), _stream(stream)))


def bergson_sync_status(stream=None) -> int:
    """Returns the status code (does not raise)."""
    return lib().bergson_sync_status(_stream(stream))


def bergson_version() -> int:
    return lib().bergson_version()


def bergson_debug_wait_probe(timeout_ns: int, stream=None) -> None:
    _check(lib().bergson_debug_wait_probe(int(timeout_ns), _stream(stream)))


def bergson_debug_inject_status(status: int, count: int) -> None:
    lib().bergson_debug_inject_status(int(status), int(count))


def bergson_debug_attr_once(n_threads: int, n_devices: int, fail_device: int = -1):
    """(setting runs per simulated device, failed requests) of the per-device
    attribute record under n_threads concurrent first calls; host only."""
    calls = (ctypes.c_int64 * int(n_devices))()
    fails = ctypes.c_int()
    _check(lib().bergson_debug_attr_once(int(n_threads), int(n_devices), int(fail_device), calls,
                                         ctypes.byref(fails)))
    return list(calls), fails.value


def bergson_debug_project_plan(layers, B: int, T: int) -> tuple[int, int, int, int]:
    """(slots, work items, pieces, layers sharing their A) the projection planner
    chooses; host only."""
    arr = _layer_array(layers)
    n = [ctypes.c_int64() for _ in range(4)]
    _check(lib().bergson_debug_project_plan(arr, len(layers), int(B), int(T),
                                            *(ctypes.byref(x) for x in n)))
    return tuple(x.value for x in n)


SCORE_PLAN_COLUMNS = ("pass", "stage", "rows", "n_qg", "qg_base", "cpg", "grid", "n_tiles",
                      "q_begin", "q_end", "pair", "qt")


SCORE_LAUNCH_COLUMNS = ("rows", "n_qg", "bn", "n_tiles", "cpg", "grid", "bound_j", "bound_r")


def _score_rows(fn: str, columns, N: int, K: int, Q: int, topk: int, ctas: int) -> list[dict]:
    call = getattr(lib(), fn)
    args = (int(N), int(K), int(Q), int(topk), int(ctas))
    n, w = ctypes.c_int32(), len(columns)
    _check(call(*args, None, 0, ctypes.byref(n)))
    buf = (ctypes.c_int64 * (w * max(1, n.value)))()
    _check(call(*args, buf, n.value, ctypes.byref(n)))
    return [dict(zip(columns, buf[w * i:w * i + w])) for i in range(n.value)]


def bergson_debug_score_plan(N: int, K: int, Q: int, topk: int, ctas: int) -> list[dict]:
    """The score launches (one dict per launch, keys SCORE_PLAN_COLUMNS) the
    scorer's planner makes for `ctas` resident CTAs; host only."""
    return _score_rows("bergson_debug_score_plan", SCORE_PLAN_COLUMNS, N, K, Q, topk, ctas)


def bergson_debug_score_launches(N: int, K: int, Q: int, topk: int, ctas: int) -> list[dict]:
    """The same launches with their tiles, grid and bound (keys SCORE_LAUNCH_COLUMNS); host only."""
    return _score_rows("bergson_debug_score_launches", SCORE_LAUNCH_COLUMNS, N, K, Q, topk, ctas)


XGEMM_PLAN_FIELDS = ("n_pad", "n_ntiles", "n_mtiles", "steps", "S", "stages", "n_chunks",
                     "pair", "n_buf", "y_rows", "tmem_cols", "xnorm_off", "ynorm_off",
                     "partial_off", "xh_off", "xl_off", "total", "a_base", "a_slots")


def bergson_debug_xgemm_plan(B: int, Q: int, K: int) -> dict:
    """The skinny-product planner's choices for B x rows, Q y rows, length K; host only."""
    buf = (ctypes.c_int64 * 19)()
    _check(lib().bergson_debug_xgemm_plan(int(B), int(Q), int(K), buf, 19))
    return dict(zip(XGEMM_PLAN_FIELDS, buf))


# ------------------------------------------------------------------ training side

_DTYPES = {}
_F32 = _I64 = _U8 = None


def _load_dtypes() -> None:
    global _F32, _I64, _U8
    import torch
    _F32, _I64, _U8 = torch.float32, torch.int64, torch.uint8
    _DTYPES.update({torch.float32: BERGSON_F32, torch.bfloat16: BERGSON_BF16,
                    torch.float16: BERGSON_F16})


def _dtype(t) -> int:
    """The bergson_dtype of a torch tensor."""
    if not _DTYPES:
        _load_dtypes()
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"expected float32, bfloat16 or float16, got {t.dtype}")
    return code


def _host_tensor(t, what: str) -> None:
    """Refuses a tensor that is not on a device, but for pinned host memory, which one can read."""
    if t.numel() > 0 and not t.is_pinned():
        raise ValueError(f"{what} must be on a CUDA device, got one on {t.device}")


def _rows(t, what: str) -> tuple[int, int]:
    """(device pointer, leading dimension) of a matrix with consecutive columns."""
    ld, col = t.stride()
    if col != 1 and t.shape[1] > 1:
        raise ValueError(f"{what}: elements of a row must be consecutive")
    if not t.is_cuda:
        _host_tensor(t, what)
    return t.data_ptr(), ld if t.shape[0] > 1 else max(ld, t.shape[1])


def _rows_like(t, what: str, dtype, shape) -> tuple[Optional[int], int]:
    """_rows() of a matrix of this type and shape; None passes as NULL."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what} must be {dtype} of shape {tuple(shape)}, got {t.dtype} of "
                         f"shape {tuple(t.shape)}")
    if not t.is_cuda:
        _host_tensor(t, what)
    ld, col = t.stride()
    return (t.data_ptr(), ld) if col == 1 and ld >= shape[1] else _rows(t, what)


def _vector(t, what: str, dtype, n: int) -> Optional[int]:
    """The device pointer of n consecutive elements; None passes as NULL."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{what} must be {dtype}, contiguous and of {n} elements, got {t.dtype} "
                         f"of shape {tuple(t.shape)}")
    if not t.is_cuda:
        _host_tensor(t, what)
    return t.data_ptr()


def _scratch(t) -> tuple[int, int]:
    """(device pointer, bytes) of a workspace."""
    if not t.is_cuda:
        _host_tensor(t, "workspace")
    return t.data_ptr(), t.numel() * t.element_size()


def bergson_token_logprobs(logits, targets, tau: float, logp, lse, entropy=None,
                           stream=None) -> None:
    """logp[r] = logits[r, targets[r]] / tau - lse[r] (and entropies); a target < 0 leaves
    its row out."""
    rows, V = logits.shape
    dtype = _dtype(logits)
    x, ld = _rows(logits, "logits")
    _check(lib().bergson_token_logprobs(x, dtype, rows, V, ld,
                                        _vector(targets, "targets", _I64, rows), tau,
                                        _vector(logp, "logp", _F32, rows),
                                        _vector(lse, "lse", _F32, rows),
                                        _vector(entropy, "entropy", _F32, rows), _stream(stream)))


def bergson_token_logprobs_backward(logits, targets, tau: float, lse, entropy, d_logp, d_entropy,
                                    d_logits, stream=None) -> None:
    """d_logits from the gradients at logp and entropy (either may be None)."""
    rows, V = logits.shape
    dtype = _dtype(logits)
    x, ld = _rows(logits, "logits")
    d, ld_d = _rows_like(d_logits, "d_logits", logits.dtype, logits.shape)
    _check(lib().bergson_token_logprobs_backward(
        x, dtype, rows, V, ld, _vector(targets, "targets", _I64, rows), tau,
        _vector(lse, "lse", _F32, rows), _vector(entropy, "entropy", _F32, rows),
        _vector(d_logp, "d_logp", _F32, rows), _vector(d_entropy, "d_entropy", _F32, rows), d, ld_d,
        _stream(stream)))


def bergson_policy_loss_workspace(B: int, T: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().bergson_policy_loss_workspace(int(B), int(T), ctypes.byref(n)))
    return n.value


def bergson_policy_loss(logp, old_logp, ref_logp, entropy, advantages, mask, clip_low: float,
                        clip_high: float, kl_coef: float, entropy_coef: float, reduction: int,
                        norm_tokens: float, loss, seq_loss, stats, d_logp, d_entropy, workspace,
                        stream=None) -> None:
    """Clipped policy loss with a KL term and an entropy bonus: the loss, the
    sequences' shares, statistics and the gradients at logp and entropy.
    advantages: [B] (one a sequence) or [B, T]; ref_logp, entropy, mask,
    seq_loss, stats and d_entropy may be None."""
    if not _DTYPES:
        _load_dtypes()
    shape = logp.shape
    B, T = shape
    x, ld = _rows_like(logp, "logp", _F32, shape)
    old, ld_old = _rows_like(old_logp, "old_logp", _F32, shape)
    ref, ld_ref = _rows_like(ref_logp, "ref_logp", _F32, shape)
    ent, ld_ent = _rows_like(entropy, "entropy", _F32, shape)
    if advantages.dim() == 1:
        adv, ld_adv = _vector(advantages, "advantages", _F32, B), 0
    else:
        adv, ld_adv = _rows_like(advantages, "advantages", _F32, shape)
        if ld_adv == 0 and T > 0:             # to the C call: one a sequence, [B]
            raise ValueError("advantages [B, T]: rows must not share their memory")
    on, ld_mask = _rows_like(mask, "mask", _U8, shape)
    d, ld_d = _rows_like(d_logp, "d_logp", _F32, shape)
    de, ld_de = _rows_like(d_entropy, "d_entropy", _F32, shape)
    args = bergson_policy_args.from_buffer_copy(_POLICY_RECORD.pack(
        x, old or 0, ref or 0, ent or 0, adv, on or 0, ld, ld_old, ld_ref, ld_ent, ld_adv, ld_mask, B, T,
        clip_low, clip_high, kl_coef, entropy_coef, norm_tokens,
        _vector(loss, "loss", _F32, 1) or 0, _vector(seq_loss, "seq_loss", _F32, B) or 0,
        _vector(stats, "stats", _F32, 3) or 0, d or 0, de or 0, ld_d, ld_de, reduction, 0))
    _check(lib().bergson_policy_loss(args, *_scratch(workspace), _stream(stream)))


def bergson_preference_loss(logp, ref_logp, mask, kind: int, beta: float, margin: float,
                            label_smoothing: float, mean_logp: bool, loss, pair_loss, rewards,
                            d_logp, stream=None) -> None:
    """Preference loss over pairs (rows p and P + p of logp [2P, T]): the loss,
    the pairs' losses, rewards and the gradient at logp.  ref_logp, mask and
    rewards may be None."""
    if not _DTYPES:
        _load_dtypes()
    shape = logp.shape
    rows, T = shape
    if rows % 2:
        raise ValueError("logp must have an even number of rows")
    P = rows // 2
    x, ld = _rows_like(logp, "logp", _F32, shape)
    ref, ld_ref = _rows_like(ref_logp, "ref_logp", _F32, shape)
    on, ld_mask = _rows_like(mask, "mask", _U8, shape)
    d, ld_d = _rows_like(d_logp, "d_logp", _F32, shape)
    args = bergson_preference_args.from_buffer_copy(_PREFERENCE_RECORD.pack(
        x, ref or 0, on or 0, ld, ld_ref, ld_mask, P, T, beta, margin, label_smoothing,
        _vector(loss, "loss", _F32, 1) or 0, _vector(pair_loss, "pair_loss", _F32, P) or 0,
        _vector(rewards, "rewards", _F32, rows) or 0, d or 0, ld_d, kind, 1 if mean_logp else 0))
    _check(lib().bergson_preference_loss(args, _stream(stream)))


@dataclasses.dataclass
class AdamWTensor:
    """One tensor of an AdamW step (see bergson_adamw_tensor); 8-bit states come
    with their scales.  Contiguous tensors, which share no memory."""
    param: object
    grad: object
    m: object
    v: object
    master: object = None
    m_scale: object = None
    v_scale: object = None
    lr_scale: float = 1.0
    weight_decay: float = 0.0

    def to_c(self) -> bergson_adamw_tensor:
        if not _DTYPES:
            _load_dtypes()
        n = self.param.numel()
        eight = self.m_scale is not None
        if eight != (self.v_scale is not None):
            raise ValueError("m_scale and v_scale must both be given or both be None")
        blocks, state = -(-n // BERGSON_STATE_BLOCK), _U8 if eight else _F32
        param = _vector(self.param, "param", self.param.dtype, n)
        grad = _vector(self.grad, "grad", self.grad.dtype, n)
        master = _vector(self.master, "master", _F32, n)
        m, v = _vector(self.m, "m", state, n), _vector(self.v, "v", state, n)
        ms = _vector(self.m_scale, "m_scale", _F32, blocks)
        vs = _vector(self.v_scale, "v_scale", _F32, blocks)
        return bergson_adamw_tensor(
            param, grad, master, m, v, ms, vs, n, float(self.lr_scale), float(self.weight_decay),
            _dtype(self.param), _dtype(self.grad),
            BERGSON_STATE_8BIT if eight else BERGSON_STATE_F32, 0)


def _records(kind, items) -> "ctypes.Array":
    """The C array of a list of records; one that is an array already is returned."""
    if isinstance(items, ctypes.Array):
        return items
    return (kind * len(items))(*[x if isinstance(x, kind) else x.to_c() for x in items])


def bergson_adamw_tensors(tensors: Sequence) -> "ctypes.Array":
    """The record array of bergson_adamw_step, to be kept from step to step.  It
    holds addresses: keep the tensors alive and in place."""
    return _records(bergson_adamw_tensor, tensors)


def bergson_adamw_step(tensors, lr: float, beta1: float, beta2: float, eps: float, step: int,
                       seed: int = 0, grad_scale=None, stream=None) -> None:
    """One AdamW step over tensors (AdamWTensor list, or bergson_adamw_tensors' array)."""
    if not _DTYPES:
        _load_dtypes()
    arr = _records(bergson_adamw_tensor, tensors)
    scale = (_vector(grad_scale, "grad_scale", _F32, 1) if hasattr(grad_scale, "data_ptr")
             else _ptr(grad_scale))
    _check(lib().bergson_adamw_step(arr, len(arr), lr, beta1, beta2, eps, step, seed, scale,
                                    _stream(stream)))


def bergson_adamw_state_values(codes, scale, moment: int, out, stream=None) -> None:
    """out = the fp32 values of an 8-bit state (moment: BERGSON_MOMENT_FIRST or _SECOND)."""
    if not _DTYPES:
        _load_dtypes()
    n = codes.numel()
    _check(lib().bergson_adamw_state_values(
        _vector(codes, "codes", _U8, n),
        _vector(scale, "scale", _F32, -(-n // BERGSON_STATE_BLOCK)), n, moment, _vector(out, "out", _F32, n), _stream(stream)))


@dataclasses.dataclass
class MomentMatrix:
    """AdamW's v [d_out, d_in] (fp32, or u8 codes with their scales) and its factors."""
    v: object
    r: object
    c: object
    v_scale: object = None

    def to_c(self) -> bergson_moment_matrix:
        if not _DTYPES:
            _load_dtypes()
        d_out, d_in = self.v.shape
        n = d_out * d_in
        v = _vector(self.v, "v", _F32 if self.v_scale is None else _U8, n)
        vs = _vector(self.v_scale, "v_scale", _F32, -(-n // BERGSON_STATE_BLOCK))
        r, c = _vector(self.r, "r", _F32, d_out), _vector(self.c, "c", _F32, d_in)
        return bergson_moment_matrix(
            v, vs, d_out, d_in, r, c,
            BERGSON_STATE_F32 if self.v_scale is None else BERGSON_STATE_8BIT, 0)


def bergson_moment_matrices(mats: Sequence) -> "ctypes.Array":
    """The record array of bergson_factor_moments, to be kept (it holds addresses)."""
    return _records(bergson_moment_matrix, mats)


def bergson_factor_moments_workspace(mats) -> int:
    arr = _records(bergson_moment_matrix, mats)
    n = ctypes.c_size_t()
    _check(lib().bergson_factor_moments_workspace(arr, len(arr), ctypes.byref(n)))
    return n.value


def bergson_factor_moments(mats, correction: float, floor: float, workspace, stream=None) -> None:
    """r and c of every matrix (MomentMatrix list, or bergson_moment_matrices' array)."""
    arr = _records(bergson_moment_matrix, mats)
    _check(lib().bergson_factor_moments(arr, len(arr), correction, floor, *_scratch(workspace),
                                        _stream(stream)))


def _no_matrix(shape, what: str):
    raise ValueError(f"{what} must be a matrix [rows, columns], got a tensor of shape {tuple(shape)}")


def _matrix(t, what: str) -> tuple:
    """(device pointer, shape, leading dimension, torch's and the library's dtype) of a matrix."""
    shape, dtype = t.shape, t.dtype
    if len(shape) != 2:
        _no_matrix(shape, what)
    code = _DTYPES.get(dtype)
    if code is None:
        code = _dtype(t)
    ld, col = t.stride()
    if col == 1 and ld >= shape[1] and t.is_cuda:
        return t.data_ptr(), shape, ld, dtype, code
    x, ld = _rows(t, what)
    return x, shape, ld, dtype, code


def _array(t, what: str, dtype, n: int) -> int:
    """_vector() where None passes as 0."""
    if t is None:
        return 0
    if t.dtype is dtype and t.is_cuda and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    return _vector(t, what, dtype, n)


def bergson_norm(x, weight, bias, kind: int, eps: float, y, mean=None, rstd=None,
                 stream=None) -> None:
    """y = layer norm of the rows of x (kind: BERGSON_NORM_LAYER, or BERGSON_NORM_RMS without a
    mean), and the rows' mean and rstd; weight and bias may be None."""
    px, shape, ld, dtype, code = _matrix(x, "x")
    py, ld_y = _rows_like(y, "y", dtype, shape)
    rows, d = shape
    one = weight if weight is not None else bias
    wt, w_code = (_F32, BERGSON_F32) if one is None else (one.dtype, _dtype(one))
    status = (_LIB or lib()).bergson_norm(_NORM_RECORD.pack(
        px, _array(weight, "weight", wt, d), _array(bias, "bias", wt, d), py,
        _array(mean, "mean", _F32, rows), _array(rstd, "rstd", _F32, rows), rows, d, ld, ld_y, eps, code,
        w_code, kind, 0), _stream(stream))
    if status:
        _check(status)


def bergson_norm_backward_workspace(rows: int, d: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().bergson_norm_backward_workspace(int(rows), int(d), ctypes.byref(n)))
    return n.value


def bergson_norm_backward(x, weight, kind: int, mean, rstd, dy, dx, d_weight, d_bias, workspace,
                          stream=None) -> None:
    """dx, d_weight and d_bias (either may be None) from the gradient at y."""
    px, shape, ld, dtype, code = _matrix(x, "x")
    pdy, ld_dy = _rows_like(dy, "dy", dtype, shape)
    pdx, ld_dx = _rows_like(dx, "dx", dtype, shape)
    rows, d = shape
    wt, w_code = (_F32, BERGSON_F32) if weight is None else (weight.dtype, _dtype(weight))
    status = (_LIB or lib()).bergson_norm_backward(_NORM_GRAD_RECORD.pack(
        px, _array(weight, "weight", wt, d), _array(mean, "mean", _F32, rows),
        _array(rstd, "rstd", _F32, rows), pdy, pdx, _array(d_weight, "d_weight", _F32, d),
        _array(d_bias, "d_bias", _F32, d), rows, d, ld, ld_dy, ld_dx, code, w_code, kind, 0),
        *_scratch(workspace), _stream(stream))
    if status:
        _check(status)


def bergson_embedding(table, ids, scale: float, out, stream=None) -> None:
    """out[r] = scale table[ids[r]]; a negative id gives zeros."""
    t, (V, d), ld, dtype, code = _matrix(table, "table")
    rows = ids.numel()
    po, ld_o = _rows_like(out, "out", dtype, (rows, d))
    status = (_LIB or lib()).bergson_embedding(_EMBEDDING_RECORD.pack(
        t, _array(ids, "ids", _I64, rows), po, V, d, rows, ld, ld_o, scale, code, 0), _stream(stream))
    if status:
        _check(status)


def bergson_embedding_backward_workspace(rows: int, V: int, d: int) -> int:
    n = ctypes.c_size_t()
    _check(lib().bergson_embedding_backward_workspace(int(rows), int(V), int(d), ctypes.byref(n)))
    return n.value


def bergson_embedding_backward(dy, ids, scale: float, d_table, add: bool, workspace,
                               stream=None) -> None:
    """The table's gradient from the gradient at the lookups, in place of d_table's values or
    (add) on top of them."""
    g, (rows, d), ld, _, code = _matrix(dy, "dy")
    t, (V, d_t), ld_t, _, t_code = _matrix(d_table, "d_table")
    if d_t != d:
        raise ValueError(f"d_table must have {d} columns, got {d_t}")
    status = (_LIB or lib()).bergson_embedding_backward(_EMBEDDING_GRAD_RECORD.pack(
        g, _array(ids, "ids", _I64, rows), t, V, d, rows, ld, ld_t, scale, code, t_code, 1 if add else 0, 0),
        *_scratch(workspace), _stream(stream))
    if status:
        _check(status)


@dataclasses.dataclass
class MuonTensor:
    """One matrix of a Muon step (see bergson_muon_tensor).  Contiguous tensors [rows, cols], which
    share no memory."""
    param: object
    grad: object
    m: object
    master: object = None
    ortho_scale: float = 1.0
    weight_decay: float = 0.0
    lr_scale: float = 1.0

    def to_c(self) -> bergson_muon_tensor:
        if not _DTYPES:
            _load_dtypes()
        shape = self.param.shape
        if len(shape) != 2:
            _no_matrix(shape, "param")
        rows, cols = shape
        for what in ("grad", "m", "master"):
            t = getattr(self, what)
            if t is not None and t.shape != shape:
                raise ValueError(f"{what} must have param's shape {tuple(shape)}, got "
                                 f"{tuple(t.shape)}")
        n = rows * cols
        return bergson_muon_tensor(
            _vector(self.param, "param", self.param.dtype, n),
            _vector(self.grad, "grad", self.grad.dtype, n), _vector(self.master, "master", _F32, n),
            _vector(self.m, "m", _F32, n), rows, cols, float(self.lr_scale),
            float(self.ortho_scale), float(self.weight_decay), _dtype(self.param),
            _dtype(self.grad), 0)


def bergson_muon_tensors(tensors: Sequence) -> "ctypes.Array":
    """The record array of bergson_muon_step, to be kept from step to step.  It holds
    addresses: keep the tensors alive and in place."""
    return _records(bergson_muon_tensor, tensors)


def bergson_muon_step_workspace(tensors, products: int) -> int:
    arr = _records(bergson_muon_tensor, tensors)
    n = ctypes.c_size_t()
    _check(lib().bergson_muon_step_workspace(arr, len(arr), int(products), ctypes.byref(n)))
    return n.value


def bergson_muon_step(tensors, lr: float, beta: float, nesterov: bool, coefficients, products: int,
                      workspace, grad_scale=None, stream=None) -> None:
    """One Muon step over matrices (MuonTensor list, or bergson_muon_tensors' array); coefficients:
    (a, b, c) an iteration."""
    if not _DTYPES:
        _load_dtypes()
    arr = _records(bergson_muon_tensor, tensors)
    if any(len(abc) != 3 for abc in coefficients):
        raise ValueError("coefficients must be triples (a, b, c)")
    flat = [float(x) for abc in coefficients for x in abc]
    scale = (_vector(grad_scale, "grad_scale", _F32, 1) if hasattr(grad_scale, "data_ptr")
             else _ptr(grad_scale))
    _check(lib().bergson_muon_step(arr, len(arr), lr, beta, 1 if nesterov else 0,
                                   (ctypes.c_double * len(flat))(*flat), len(coefficients), products,
                                   scale, *_scratch(workspace), _stream(stream)))


# ------------------------------------------------------------------ helpers

def workspace_tensor(nbytes: int, device="cuda"):
    """A byte tensor usable as workspace (torch allocations are 512-byte aligned)."""
    import torch
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)
