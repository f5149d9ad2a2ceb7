"""ctypes binding of libtss.so: the C ABI declared in include/tss.h, with the same names.

Argument marshalling only: every step of verification runs in the library's CUDA kernels.  The
binding never falls back to another implementation; if the library is missing it raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Dict, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtss.so")

TSS_OK = 0
TSS_ERR_INVALID_ARG = 1
TSS_ERR_OUT_OF_MEMORY = 2
TSS_ERR_KV_CAPACITY = 3
TSS_ERR_CUDA = 4
TSS_ERR_UNSUPPORTED_ARCH = 5
TSS_ERR_TIMEOUT = 6
TSS_ERR_DEVICE_CHECK = 7
TSS_MODE_GREEDY = 0
TSS_MODE_SAMPLE = 1

EXPORTS = (
    "tss_create", "tss_set_skip_config", "tss_clear_skip_config", "tss_sparsity_ratio",
    "tss_active_layer_count", "tss_verify", "tss_verify_profiled", "tss_prefill", "tss_sync_status", "tss_destroy",
    "tss_linear", "tss_linear_static", "tss_read_trace", "tss_status_string", "tss_last_error",
    "tss_estimate_step_bytes", "tss_persistent_plan", "tss_inject_timeout", "tss_philox_uniforms",
    "tss_linear_static_status", "tss_verify_grouped", "tss_attention_kernel",
    "tss_qk_rope", "tss_rope_frequencies", "tss_rope_table",
    "tss_paged_page_bytes", "tss_paged_create", "tss_paged_destroy", "tss_paged_sync_status", "tss_paged_append",
    "tss_paged_append_rope", "tss_paged_read", "tss_paged_attention", "tss_paged_inject_timeout",
    "tss_paged_create_shared", "tss_paged_attention_shared",
    "tss_pages_create", "tss_pages_destroy", "tss_pages_sync_status", "tss_pages_reserve", "tss_pages_free",
    "tss_pages_fork", "tss_pages_reorder", "tss_pages_compact", "tss_pages_copy",
    "tss_beam_create", "tss_beam_destroy", "tss_beam_sync_status", "tss_beam_select",
)
TSS_DTYPE_BF16 = 0
TSS_DTYPE_F16 = 1
TSS_DTYPE_F32 = 2
PAGE_TOKENS = 64
ROPE_KINDS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}

_P = ctypes.c_void_p
_I32P = ctypes.POINTER(ctypes.c_int32)


class TssArch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_layers", "d_model", "n_heads", "head_dim", "d_mlp", "vocab")] + [
        ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float)] + [
        (n, ctypes.c_int) for n in ("max_batch", "max_rows", "max_nodes", "max_domains", "max_positions")]


class TssWeights(ctypes.Structure):
    _fields_ = [("embed", _P), ("lm_head", _P), ("final_norm", _P)] + [
        (n, ctypes.POINTER(_P)) for n in ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")]


class TssVerifyBatch(ctypes.Structure):
    _fields_ = [
        ("n_req", ctypes.c_int), ("n_nodes", _P), ("ctx_len", _P), ("domain_id", _P), ("kv_slot", _P),
        ("parent_idx", _P), ("positions", _P), ("tokens", _P), ("mode", ctypes.c_int),
        ("temperature", ctypes.c_float), ("draft_probs", _P), ("uniforms", _P), ("uniform_stride", ctypes.c_int),
        ("philox_seed", ctypes.c_uint64), ("philox_offset", ctypes.c_uint64), ("io_host", ctypes.c_int)]


class TssKvCache(ctypes.Structure):
    _fields_ = [("layer", ctypes.POINTER(_P)), ("n_slots", ctypes.c_int), ("cap", ctypes.c_int)]


KERNEL_KINDS = ("controller+embed+norms", "qkv_gemm", "attention", "o_gemm", "gate_up_gemm", "down_gemm",
                "lm_head_gemm", "accept+compact", "verify_persistent")


class TssKernelTimes(ctypes.Structure):
    _fields_ = [("ms", ctypes.c_float * 9), ("launches", ctypes.c_int * 9)]


class TssStepBytes(ctypes.Structure):
    _fields_ = [("weights", ctypes.c_uint64), ("kv_read", ctypes.c_uint64), ("kv_write", ctypes.c_uint64),
                ("total", ctypes.c_uint64), ("active_union", ctypes.c_int)]


class TssPersistentPlanInfo(ctypes.Structure):
    _fields_ = [("fits", ctypes.c_int), ("kps", ctypes.c_int), ("stages", ctypes.c_int), ("attn_splits", ctypes.c_int),
                ("smem_bytes", ctypes.c_uint64)]


class TssVerifyResult(ctypes.Structure):
    _fields_ = [("accept_len", _P), ("bonus", _P), ("path", _P), ("path_stride", ctypes.c_int),
                ("new_ctx_len", _P), ("logits", _P)]


class TssRopeArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_rows", "n_q_heads", "n_k_heads", "head_dim", "rot_dim", "interleaved", "dtype")] + [
        (n, _P) for n in ("q", "k", "q_out", "k_out")] + [
        (n, ctypes.c_int64) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride")] + [
        ("q_gain", _P), ("k_gain", _P), ("eps", ctypes.c_float), ("table", _P), ("max_positions", ctypes.c_int),
        ("positions", _P), ("status", _P)]


class TssPagedCache(ctypes.Structure):
    _fields_ = [("layer", ctypes.POINTER(_P)), ("n_layers", ctypes.c_int), ("n_pages", ctypes.c_int), ("table", _P),
                ("n_seqs", ctypes.c_int), ("max_pages", ctypes.c_int)]


class TssPagedBatch(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int), ("seq", _P), ("first", _P), ("n_tokens", _P)]


class TssPagedAttn(ctypes.Structure):
    _fields_ = [("q", _P), ("q_stride", ctypes.c_int64), ("out", _P), ("out_stride", ctypes.c_int64), ("lse", _P),
                ("dtype", ctypes.c_int), ("scale", ctypes.c_float), ("window", ctypes.c_int), ("n_sinks", ctypes.c_int),
                ("mask", _P), ("positions", _P)]


class TssPagedGroups(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_int), ("n_req", _P), ("shared", _P)]


class TssPageTables(ctypes.Structure):
    _fields_ = [("table", _P), ("held", _P), ("refs", _P)]


class TssBeamArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_groups", "n_beams", "n_keep", "dtype")] + [
        ("logits", _P), ("stride", ctypes.c_int64), ("score", _P), ("done", _P), ("end_token", ctypes.c_int), ("score_out", _P),
        ("parent", _P), ("token", _P)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load libtss.so (built by __graft_entry__.build() or paper_2609_26100_gb300/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it first (python -c 'import __graft_entry__ as g; g.build()')")
        L = ctypes.CDLL(LIB_PATH)
        L.tss_create.argtypes = [ctypes.POINTER(TssWeights), ctypes.POINTER(TssArch), ctypes.POINTER(_P)]
        L.tss_set_skip_config.argtypes = [_P, ctypes.c_int, ctypes.c_uint64]
        L.tss_clear_skip_config.argtypes = [_P, ctypes.c_int]
        L.tss_sparsity_ratio.argtypes = [_P, ctypes.c_int, ctypes.POINTER(ctypes.c_double)]
        L.tss_active_layer_count.argtypes = [_P, ctypes.POINTER(TssVerifyBatch), ctypes.POINTER(ctypes.c_int)]
        L.tss_verify.argtypes = [_P, ctypes.POINTER(TssVerifyBatch), ctypes.POINTER(TssKvCache),
                                 ctypes.POINTER(TssVerifyResult), _P]
        L.tss_verify_profiled.argtypes = [_P, ctypes.POINTER(TssVerifyBatch), ctypes.POINTER(TssKvCache),
                                          ctypes.POINTER(TssVerifyResult), _P, ctypes.POINTER(TssKernelTimes)]
        L.tss_prefill.argtypes = [_P, ctypes.c_int, _I32P, _I32P, _I32P, _I32P, _P, ctypes.c_int,
                                  ctypes.POINTER(TssKvCache), _P]
        L.tss_sync_status.argtypes = [_P, _P]
        L.tss_destroy.argtypes = [_P]
        L.tss_destroy.restype = None
        L.tss_linear.argtypes = [_P, _P, _P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_int, _P]
        L.tss_linear_static.argtypes = [_P, _P, _P, ctypes.c_int, ctypes.c_int, ctypes.c_int, _P]
        L.tss_read_trace.argtypes = [_P, _P, ctypes.c_size_t, ctypes.POINTER(ctypes.c_size_t)]
        L.tss_status_string.argtypes = [ctypes.c_int]
        L.tss_status_string.restype = ctypes.c_char_p
        L.tss_last_error.argtypes = []
        L.tss_last_error.restype = ctypes.c_char_p
        L.tss_estimate_step_bytes.argtypes = [ctypes.POINTER(TssArch), ctypes.c_int, ctypes.POINTER(ctypes.c_uint64),
                                              _I32P, _I32P, ctypes.POINTER(TssStepBytes)]
        L.tss_persistent_plan.argtypes = [ctypes.POINTER(TssArch), ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                          ctypes.c_int, ctypes.POINTER(TssPersistentPlanInfo)]
        L.tss_inject_timeout.argtypes = [_P, ctypes.c_int]
        L.tss_philox_uniforms.argtypes = [ctypes.c_uint64, ctypes.c_uint64, ctypes.c_int, ctypes.c_int, _P, _P, _P]
        L.tss_linear_static_status.argtypes = [_P]
        L.tss_verify_grouped.argtypes = [_P, ctypes.POINTER(TssVerifyBatch), ctypes.POINTER(TssKvCache),
                                         ctypes.POINTER(TssVerifyResult), _P, ctypes.POINTER(ctypes.c_int),
                                         ctypes.POINTER(_P)]
        L.tss_attention_kernel.argtypes = [_P]
        L.tss_attention_kernel.restype = ctypes.c_int
        I, L64, PP = ctypes.c_int, ctypes.c_int64, ctypes.POINTER(_P)
        D = ctypes.POINTER(ctypes.c_double)
        cache, batch, tables = ctypes.POINTER(TssPagedCache), ctypes.POINTER(TssPagedBatch), ctypes.POINTER(TssPageTables)
        L.tss_qk_rope.argtypes = [ctypes.POINTER(TssRopeArgs), _P]
        L.tss_rope_frequencies.argtypes = [I, I, ctypes.c_double, ctypes.c_double, ctypes.c_double, D, D]
        L.tss_rope_table.argtypes = [D, I, ctypes.c_double, I, _P, _P]
        L.tss_paged_page_bytes.argtypes = [I, I]
        L.tss_paged_page_bytes.restype = ctypes.c_size_t
        L.tss_paged_create.argtypes = [I, I, I, PP]
        L.tss_paged_sync_status.argtypes = [_P, _P]
        L.tss_paged_append.argtypes = [_P, cache, I, batch, _P, _P, L64, L64, I, _P]
        L.tss_paged_append_rope.argtypes = [_P, cache, I, batch, ctypes.POINTER(TssRopeArgs), _P, L64, _P]
        L.tss_paged_read.argtypes = L.tss_paged_append.argtypes
        L.tss_paged_attention.argtypes = [_P, cache, I, batch, ctypes.POINTER(TssPagedAttn), _P]
        L.tss_paged_create_shared.argtypes = [I, I, I, I, PP]
        L.tss_paged_attention_shared.argtypes = [_P, cache, I, batch, ctypes.POINTER(TssPagedGroups), ctypes.POINTER(TssPagedAttn), _P]
        L.tss_paged_inject_timeout.argtypes = [_P, I]
        L.tss_paged_inject_timeout.restype = I
        L.tss_pages_create.argtypes = [I, I, I, PP]
        L.tss_pages_sync_status.argtypes = [_P, _P]
        L.tss_pages_reserve.argtypes = [_P, tables, I, _P, _P, _P]
        L.tss_pages_free.argtypes = [_P, tables, I, _P, _P, _P]
        L.tss_pages_fork.argtypes = [_P, tables, PP, I, ctypes.c_size_t, I, _P, _P, _P, _P, _P]
        L.tss_pages_reorder.argtypes = L.tss_pages_fork.argtypes
        L.tss_pages_compact.argtypes = [_P, tables, _P, _P, PP, I, ctypes.c_size_t, _P]
        L.tss_pages_copy.argtypes = [_P, PP, I, ctypes.c_size_t, I, _P, _P, _P]
        L.tss_beam_create.argtypes = [I, I, I, PP]
        L.tss_beam_sync_status.argtypes = [_P, _P]
        L.tss_beam_select.argtypes = [_P, ctypes.POINTER(TssBeamArgs), _P]
        for name in ("tss_paged_destroy", "tss_pages_destroy", "tss_beam_destroy"):
            getattr(L, name).argtypes = [_P]
            getattr(L, name).restype = None
        for name in ("tss_qk_rope", "tss_rope_frequencies", "tss_rope_table", "tss_paged_create", "tss_paged_sync_status",
                     "tss_paged_append", "tss_paged_append_rope", "tss_paged_read", "tss_paged_attention", "tss_pages_create",
                     "tss_paged_create_shared", "tss_paged_attention_shared",
                     "tss_pages_sync_status", "tss_pages_reserve", "tss_pages_free", "tss_pages_fork", "tss_pages_reorder",
                     "tss_pages_compact", "tss_pages_copy", "tss_beam_create", "tss_beam_sync_status", "tss_beam_select"):
            getattr(L, name).restype = ctypes.c_int
        for name in ("tss_create", "tss_set_skip_config", "tss_clear_skip_config", "tss_sparsity_ratio",
                     "tss_active_layer_count", "tss_verify", "tss_verify_profiled", "tss_prefill", "tss_sync_status",
                     "tss_linear", "tss_linear_static", "tss_read_trace", "tss_estimate_step_bytes",
                     "tss_persistent_plan", "tss_inject_timeout", "tss_philox_uniforms", "tss_linear_static_status",
                     "tss_verify_grouped"):
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def linear_static(x, w, y, stream=None) -> None:
    """y = x @ w^T through tss_linear_static (no context, no device allocation)."""
    m, k = x.shape
    check(lib().tss_linear_static(x.data_ptr(), w.data_ptr(), y.data_ptr(), m, k, w.shape[0], stream),
          "tss_linear_static")


def linear_static_status(stream=None) -> int:
    """tss_linear_static_status: synchronise, return and clear the static linear layer's status."""
    return lib().tss_linear_static_status(stream)


def philox_uniforms(seed: int, offset: int, words=None, uniforms=None, stream=None) -> None:
    """tss_philox_uniforms into device tensors words [n_req][n_slots][4] (int32 or uint32 bits)
    and/or uniforms [n_req][n_slots] (float32)."""
    t = words if words is not None else uniforms
    n_req, n_slots = int(t.shape[0]), int(t.shape[1])
    check(lib().tss_philox_uniforms(int(seed), int(offset), n_req, n_slots, _ptr(words), _ptr(uniforms), stream),
          "tss_philox_uniforms")


def persistent_plan(arch, n_req: int, n_rows: int, max_keys: int, num_sms: int) -> Dict[str, int]:
    """tss_persistent_plan: the persistent kernel's shared-memory plan for a step (host only)."""
    a = TssArch(arch.n_layers, arch.d_model, arch.n_heads, arch.head_dim, arch.d_mlp, arch.vocab,
                arch.rms_eps, arch.rope_theta, 1, 1, 1, 1, 1)
    out = TssPersistentPlanInfo()
    check(lib().tss_persistent_plan(ctypes.byref(a), n_req, n_rows, max_keys, num_sms, ctypes.byref(out)),
          "tss_persistent_plan")
    return {"fits": bool(out.fits), "kps": out.kps, "stages": out.stages, "attn_splits": out.attn_splits,
            "smem_bytes": out.smem_bytes}


def estimate_step_bytes(arch, masks: Sequence[int], ctx_len: Sequence[int], n_nodes: Sequence[int]) -> Dict[str, int]:
    """tss_estimate_step_bytes: HBM bytes of a verification step (host arithmetic, no GPU)."""
    a = TssArch(arch.n_layers, arch.d_model, arch.n_heads, arch.head_dim, arch.d_mlp, arch.vocab,
                arch.rms_eps, arch.rope_theta, 1, 1, 1, 1, 1)
    n = len(masks)
    m = (ctypes.c_uint64 * n)(*[int(x) for x in masks])
    out = TssStepBytes()
    check(lib().tss_estimate_step_bytes(ctypes.byref(a), n, m, ctypes.cast(_i32(ctx_len), _I32P),
                                        ctypes.cast(_i32(n_nodes), _I32P), ctypes.byref(out)), "tss_estimate_step_bytes")
    return {"weights": out.weights, "kv_read": out.kv_read, "kv_write": out.kv_write, "total": out.total,
            "active_union": out.active_union}


def dtype_code(t) -> int:
    """TSS_DTYPE_* of a torch tensor."""
    name = str(t.dtype)
    codes = {"torch.bfloat16": TSS_DTYPE_BF16, "torch.float16": TSS_DTYPE_F16, "torch.float32": TSS_DTYPE_F32}
    if name not in codes:
        raise TypeError(f"bfloat16, float16 or float32 is wanted, not {name}")
    return codes[name]


def _rows(t, what: str):
    """(rows, heads, head_dim, row stride) of a GPU tensor [rows][heads][head_dim] whose heads are contiguous."""
    if t.dim() != 3 or not t.is_cuda:
        raise ValueError(f"{what}: [rows][heads][head_dim] on the GPU is wanted")
    n, h, d = t.shape
    if n and h and (t.stride(2) != 1 or (h > 1 and t.stride(1) != d)):
        raise ValueError(f"{what}: the heads of a row must be contiguous")
    return n, h, d, t.stride(0) if n > 1 else h * d  # (nothing steps from a single row)


def _same(a, b, what: str) -> None:
    if b is None or a.shape != b.shape or a.dtype != b.dtype or a.device != b.device:
        raise ValueError(f"{what}: the output's shape, type and device must be the input's")


def rope_frequencies(rot_dim: int, theta: float = 10000.0, kind: str = "none", factor: float = 1.0, original: float = 0.0):
    """tss_rope_frequencies: (list of rot_dim / 2 frequencies, attention factor); kind one of ROPE_KINDS."""
    n = max(int(rot_dim) // 2, 1)
    f, a = (ctypes.c_double * n)(), ctypes.c_double()
    check(lib().tss_rope_frequencies(ROPE_KINDS[kind], rot_dim, theta, factor, original, f, ctypes.byref(a)),
          "tss_rope_frequencies")
    return list(f), a.value


def rope_table(inv_freq: Sequence[float], table, attention_factor: float = 1.0, stream=None) -> None:
    """tss_rope_table into the float32 device tensor table [positions][len(inv_freq)][2], on the given stream (None:
    torch's current one)."""
    import torch
    n = len(inv_freq)
    if tuple(table.shape[1:]) != (n, 2) or dtype_code(table) != TSS_DTYPE_F32 or not table.is_contiguous() or not table.is_cuda:
        raise ValueError("table: contiguous float32 [positions][pairs][2] on the GPU is wanted")
    if table.get_device() != torch.cuda.current_device():
        raise ValueError("the table's device is not the current one")
    check(lib().tss_rope_table((ctypes.c_double * n)(*inv_freq), n, attention_factor, table.shape[0], table.data_ptr(),
                               current_stream() if stream is None else stream), "tss_rope_table")


def rope_args(q, k, q_out, k_out, positions, table, q_gain=None, k_gain=None, eps: float = 1e-6, interleaved: bool = False,
              status=None, to_pages: bool = False) -> TssRopeArgs:
    """Arguments of tss_qk_rope from tensors of one GPU: q, k [rows][heads][head_dim] (either may be None) and their
    outputs (q_out may be q), positions int32 [rows], table [positions][pairs][2] float32 (None: no rotation),
    gains [head_dim] (None: no norm).  to_pages: for Kv4Cache.append_rope, where k_out may be None.  The structure keeps
    the tensors alive."""
    one = q if q is not None else k
    if one is None:
        raise ValueError("q or k is wanted")
    a = TssRopeArgs()
    a.n_rows, _, a.head_dim, _ = _rows(one, "q")
    a._device = one.get_device()
    for x in (k, table, positions, status):
        if x is not None and x.get_device() != a._device:
            raise ValueError("q, k, table, positions and status on one GPU are wanted")
    a.dtype, a.interleaved, a.eps = dtype_code(one), int(interleaved), eps
    for name, x, y, gain in (("q", q, q_out, q_gain), ("k", k, k_out, k_gain)):
        if x is None:
            continue
        n, h, d, stride = _rows(x, name)
        if y is not None or name == "q" or not to_pages:
            _same(x, y, name)
        if (n, d, dtype_code(x)) != (a.n_rows, a.head_dim, a.dtype):
            raise ValueError("q and k must agree in rows, head_dim and type")
        setattr(a, f"n_{name}_heads", h)
        setattr(a, name, x.data_ptr())
        setattr(a, name + "_stride", stride)
        if y is not None:
            setattr(a, name + "_out", y.data_ptr())
            setattr(a, name + "_out_stride", _rows(y, name + "_out")[3])
        if gain is not None:
            if tuple(gain.shape) != (d,) or gain.dtype != x.dtype or gain.device != x.device or not gain.is_contiguous():
                raise ValueError(f"{name}_gain: contiguous [head_dim] of the same type and device is wanted")
            setattr(a, name + "_gain", gain.data_ptr())
    if table is not None:
        if (table.dim() != 3 or table.shape[2] != 2 or dtype_code(table) != TSS_DTYPE_F32 or not table.is_contiguous()
                or not table.is_cuda):
            raise ValueError("table: contiguous float32 [positions][pairs][2] on the GPU is wanted")
        if (positions is None or str(positions.dtype) != "torch.int32" or positions.numel() != a.n_rows or not positions.is_contiguous()
                or not positions.is_cuda):
            raise ValueError("positions: contiguous int32 [rows] on the GPU is wanted")
        a.table, a.max_positions, a.rot_dim = table.data_ptr(), table.shape[0], 2 * table.shape[1]
        a.positions = positions.data_ptr()
    if status is not None and (str(status.dtype) != "torch.int32" or not status.is_cuda):
        raise ValueError("status: an int32 tensor on the GPU is wanted")
    a.status = _ptr(status)
    a._to_pages = to_pages
    a._keep = (q, k, q_out, k_out, positions, table, q_gain, k_gain, status)
    return a


def current_stream() -> int:
    """torch's current stream on the current device."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def qk_rope(args: TssRopeArgs, stream=None) -> None:
    """tss_qk_rope on the given stream (None: torch's current one) of the tensors' device, which has to be the current one."""
    import torch
    device = torch.cuda.current_device()
    if getattr(args, "_device", device) != device:
        raise ValueError("the tensors' device is not the current one")
    s = lib().tss_qk_rope(ctypes.byref(args), torch._C._cuda_getCurrentRawStream(device) if stream is None else stream)
    if s:
        check(s, "tss_qk_rope")


class TssError(RuntimeError):
    def __init__(self, status: int, where: str):
        L = lib()
        self.status = status
        msg = L.tss_last_error().decode()
        super().__init__(f"{where}: {L.tss_status_string(status).decode()} ({status}): {msg}")


def check(status: int, where: str) -> None:
    if status != TSS_OK:
        raise TssError(status, where)


def _ptr(t) -> Optional[int]:
    """Address of a tensor / numpy array (None -> NULL)."""
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        return t.data_ptr()
    return t.ctypes.data


def _i32(values) -> "ctypes.Array":
    arr = (ctypes.c_int32 * len(values))(*map(int, values))
    return arr


class Verifier:
    """Owns one tss_ctx.  Weights: dict as produced by synth.make_weights (bf16 CUDA tensors)."""

    def __init__(self, weights: Dict, arch, max_batch: int = 16, max_rows: int = 256, max_nodes: int = 64,
                 max_domains: int = 64, max_positions: int = 20480):
        L = lib()
        self.arch = arch
        a = TssArch(arch.n_layers, arch.d_model, arch.n_heads, arch.head_dim, arch.d_mlp, arch.vocab,
                    arch.rms_eps, arch.rope_theta, max_batch, max_rows, max_nodes, max_domains, max_positions)
        self._arch = a
        n = arch.n_layers
        arrs = {}
        for key in ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down"):
            arrs[key] = (_P * n)(*[weights["layers"][l][key].data_ptr() for l in range(n)])
        w = TssWeights(weights["embed"].data_ptr(), weights["lm_head"].data_ptr(), weights["final_norm"].data_ptr(),
                       *[ctypes.cast(arrs[k], ctypes.POINTER(_P)) for k in
                         ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")])
        h = _P()
        check(L.tss_create(ctypes.byref(w), ctypes.byref(a), ctypes.byref(h)), "tss_create")
        self.ctx = h

    def close(self):
        if getattr(self, "ctx", None):
            lib().tss_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_skip_config(self, domain: int, mask: int) -> None:
        check(lib().tss_set_skip_config(self.ctx, domain, mask), "tss_set_skip_config")

    def clear_skip_config(self, domain: int) -> None:
        check(lib().tss_clear_skip_config(self.ctx, domain), "tss_clear_skip_config")

    def sparsity_ratio(self, domain: int) -> float:
        out = ctypes.c_double()
        check(lib().tss_sparsity_ratio(self.ctx, domain, ctypes.byref(out)), "tss_sparsity_ratio")
        return out.value

    def sync_status(self, stream=None) -> int:
        return lib().tss_sync_status(self.ctx, stream)

    def attention_kernel(self) -> int:
        """tss_attention_kernel: the attention kernel of the last step (0 split-KV warp-MMA kernel,
        1 tcgen05 kernel, 2 its wide variant, 3 inside the persistent kernel, -1 none yet)."""
        return int(lib().tss_attention_kernel(self.ctx))

    def inject_timeout(self, n_steps: int) -> None:
        check(lib().tss_inject_timeout(self.ctx, n_steps), "tss_inject_timeout")

    def linear(self, x, w, y, stream=None) -> None:
        m, k = x.shape
        n = w.shape[0]
        check(lib().tss_linear(self.ctx, x.data_ptr(), w.data_ptr(), y.data_ptr(), m, k, n, stream), "tss_linear")

    @staticmethod
    def make_batch(n_nodes: Sequence[int], ctx_len: Sequence[int], domain_id: Sequence[int], parent_idx: Sequence[int],
                   tokens, kv_slot=None, positions=None, mode: int = TSS_MODE_GREEDY, temperature: float = 1.0,
                   draft_probs=None, uniforms=None, uniform_stride: int = 0, philox_seed: int = 0,
                   philox_offset: int = 0, io_host: bool = False):
        """Build a TssVerifyBatch; host metadata arrays are kept alive on the returned object."""
        keep = {"n_nodes": _i32(n_nodes), "ctx_len": _i32(ctx_len), "domain_id": _i32(domain_id),
                "parent_idx": _i32(parent_idx)}
        if kv_slot is not None:
            keep["kv_slot"] = _i32(kv_slot)
        if positions is not None:
            keep["positions"] = _i32(positions)
        addr = {k: ctypes.cast(v, _P) for k, v in keep.items()}
        b = TssVerifyBatch(
            len(n_nodes), addr["n_nodes"], addr["ctx_len"], addr["domain_id"], addr.get("kv_slot"),
            addr["parent_idx"], addr.get("positions"), _ptr(tokens), mode, temperature, _ptr(draft_probs),
            _ptr(uniforms), uniform_stride, philox_seed, philox_offset, 1 if io_host else 0)
        b._keep = (keep, tokens, draft_probs, uniforms)
        return b

    def make_kv(self, layer_ptrs: Sequence[Optional[int]], n_slots: int, cap: int):
        arr = (_P * len(layer_ptrs))(*[p if p else None for p in layer_ptrs])
        kv = TssKvCache(ctypes.cast(arr, ctypes.POINTER(_P)), n_slots, cap)
        kv._keep = arr
        return kv

    @staticmethod
    def make_result(accept_len, bonus, path, path_stride: int, new_ctx_len, logits=None):
        r = TssVerifyResult(_ptr(accept_len), _ptr(bonus), _ptr(path), path_stride, _ptr(new_ctx_len), _ptr(logits))
        r._keep = (accept_len, bonus, path, new_ctx_len, logits)
        return r

    def verify(self, batch, kv, result, stream=None) -> None:
        check(lib().tss_verify(self.ctx, ctypes.byref(batch), ctypes.byref(kv), ctypes.byref(result), stream),
              "tss_verify")

    def verify_grouped(self, batch, kv, result, stream=None, events=None) -> int:
        """tss_verify_grouped; events: optional list of torch.cuda.Event (one per request, the first
        n_groups are recorded).  Returns the number of groups."""
        n = ctypes.c_int()
        ev = None
        if events is not None:
            for e in events:  # torch creates an event at its first record
                if e is not None and not e.cuda_event:
                    e.record()
            ev = (_P * len(events))(*[e.cuda_event if e is not None else None for e in events])
        check(lib().tss_verify_grouped(self.ctx, ctypes.byref(batch), ctypes.byref(kv), ctypes.byref(result), stream,
                                       ctypes.byref(n), ev), "tss_verify_grouped")
        return n.value

    def prefill(self, n_tokens: Sequence[int], ctx_len: Sequence[int], domain_id: Sequence[int], tokens, kv,
                kv_slot=None, io_host: bool = False, stream=None) -> None:
        """tss_prefill: tokens (int32, the requests' tokens concatenated) appended to the caches."""
        keep = [_i32(n_tokens), _i32(ctx_len), _i32(domain_id), _i32(kv_slot) if kv_slot is not None else None]
        cast = [ctypes.cast(a, _I32P) if a is not None else None for a in keep]
        check(lib().tss_prefill(self.ctx, len(n_tokens), cast[0], cast[1], cast[2], cast[3], _ptr(tokens),
                                1 if io_host else 0, ctypes.byref(kv), stream), "tss_prefill")

    def verify_profiled(self, batch, kv, result, times: "TssKernelTimes", stream=None) -> None:
        check(lib().tss_verify_profiled(self.ctx, ctypes.byref(batch), ctypes.byref(kv), ctypes.byref(result), stream,
                                        ctypes.byref(times)), "tss_verify_profiled")

    def read_trace(self):
        """Persistent-kernel timeline of the last step (see tss_read_trace), as a numpy array
        [n_sms, slots] of globaltimer ns, or None when tracing is off."""
        import numpy as np
        n = ctypes.c_size_t()
        check(lib().tss_read_trace(self.ctx, None, 0, ctypes.byref(n)), "tss_read_trace")
        if n.value == 0:
            return None
        buf = np.zeros(n.value, dtype=np.uint64)
        check(lib().tss_read_trace(self.ctx, buf.ctypes.data, n.value, ctypes.byref(n)), "tss_read_trace")
        return buf

    def active_layer_count(self, batch) -> int:
        out = ctypes.c_int()
        check(lib().tss_active_layer_count(self.ctx, ctypes.byref(batch), ctypes.byref(out)), "tss_active_layer_count")
        return out.value
