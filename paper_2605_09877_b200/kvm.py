"""Thin ctypes binding over the C ABI of libkvm.so (include/kvm.h).

Argument marshalling only: every step of the layer runs inside the CUDA library.  torch is
used for device memory and streams.  Importing this module raises if the library has not
been built (python -m paper_2605_09877_b200.build) -- there is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from dataclasses import dataclass

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvm.so")

KVM_OK = 0
STATUS = {0: "KVM_OK", 1: "KVM_ERR_INVALID_ARG", 2: "KVM_ERR_UNSUPPORTED", 3: "KVM_ERR_OOM",
          4: "KVM_ERR_CUDA", 5: "KVM_ERR_STATE_MISMATCH", 6: "KVM_ERR_CAPACITY", 7: "KVM_ERR_TIMEOUT"}
GROWTH_FIXED, GROWTH_SQRT, GROWTH_UNBOUNDED, GROWTH_POWER, GROWTH_SATURATING = 0, 1, 2, 3, 4
FLAG_NO_RADIUS, FLAG_RECORD_ASSIGN, FLAG_SIMT_ATTENTION, FLAG_SIMT_ROUTING, FLAG_MIN_KEY_SLOTS, FLAG_SERIAL_FOLDS, FLAG_FUSED_QK_LN = 1, 2, 4, 8, 16, 32, 64

EXPORTS = ["kvm_plan_capacity", "kvm_state_create", "kvm_prefill", "kvm_decode_step", "kvm_prefill_host",
           "kvm_decode_step_host", "kvm_state_free", "kvm_state_info", "kvm_state_check", "kvm_state_export",
           "kvm_debug_assignments", "kvm_launch_count", "kvm_status_string", "kvm_state_reset",
           "kvm_profile_enable", "kvm_profile_read", "kvm_debug_counters", "kvm_attend_rows_noalloc", "kvm_merge_gate", "kvm_head_layernorm",
           "kvm_state_snapshot_info", "kvm_state_export_window", "kvm_state_import", "kvm_debug_expire_wait",
           "kvm_debug_decode_plan", "kvm_debug_decode_ahead", "kvm_debug_apply_plan", "kvm_debug_attention_plan",
           "kvm_debug_drop_exchange",
           "kvm_rope_frequencies", "kvm_qk_norm_rope", "kvm_cache_ingest", "kvm_cache_read",
           "kvm_cache_attend_shared", "kvm_cache_shared_workspace", "kvm_pages_shared",
           "kvm_cache_append", "kvm_cache_attend", "kvm_cache_workspace", "kvm_cache_copy_pages",
           "kvm_pages_create", "kvm_pages_destroy", "kvm_pages_open", "kvm_pages_fork", "kvm_pages_close", "kvm_pages_extend",
           "kvm_pages_trim", "kvm_pages_compact", "kvm_pages_table", "kvm_pages_info"]


class KVMError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {STATUS.get(code, code)}")


class Growth(C.Structure):
    _fields_ = [("kind", C.c_int32), ("sqrt_coeff", C.c_int32), ("fixed_slots", C.c_int64),
                ("pow_num", C.c_int32), ("pow_den", C.c_int32), ("sat_half", C.c_int64)]


class Strides(C.Structure):
    _fields_ = [("q", C.c_int64 * 4), ("k", C.c_int64 * 4), ("v", C.c_int64 * 4), ("out", C.c_int64 * 4)]


class SnapshotInfo(C.Structure):
    _fields_ = [("block", C.c_int32), ("rope_dims", C.c_int32), ("growth", Growth), ("n_slots", C.c_int64),
                ("position", C.c_int64), ("n_folds", C.c_int64), ("window_begin", C.c_int64), ("window_len", C.c_int64)]


class Config(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("n_bswa_chunks", C.c_int32), ("sink_len", C.c_int32),
        ("rope_base", C.c_float), ("ln_eps", C.c_float), ("norm_eps", C.c_float),
        ("ln_weight", C.POINTER(C.c_float)), ("ln_bias", C.POINTER(C.c_float)),
        ("tau_state", C.POINTER(C.c_float)), ("tau_bswa", C.POINTER(C.c_float)),
        ("max_block", C.c_int32), ("max_state_slots", C.c_int64), ("max_call_tokens", C.c_int64),
        ("max_seq_len", C.c_int64), ("device", C.c_int32), ("flags", C.c_uint32),
        ("qk_ln_eps", C.c_float),
        ("ln_q_weight", C.POINTER(C.c_float)), ("ln_q_bias", C.POINTER(C.c_float)),
        ("ln_k_weight", C.POINTER(C.c_float)), ("ln_k_bias", C.POINTER(C.c_float)),
    ]


class CacheDesc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("n_pages", C.c_int64),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32)]


class CacheCall(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("start", C.c_void_p), ("count", C.c_void_p), ("batch", C.c_int32), ("max_pages", C.c_int32),
                ("n_tokens", C.c_int64)]


class FrontDesc(C.Structure):
    _fields_ = [("norm", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32), ("rope_dims", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double), ("magnitude", C.c_double),
                ("original_len", C.c_int64), ("eps", C.c_float), ("frequencies", C.POINTER(C.c_double)),
                ("q_weight", C.c_void_p), ("q_bias", C.c_void_p), ("k_weight", C.c_void_p), ("k_bias", C.c_void_p)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_09877_b200.build` "
                          "(the KVM layer has no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp = C.c_void_p
    L.kvm_plan_capacity.restype = C.c_int64
    L.kvm_plan_capacity.argtypes = [C.c_int32, C.c_int32, Growth, C.c_int64]
    L.kvm_state_create.restype = C.c_int
    L.kvm_state_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
    L.kvm_prefill.restype = C.c_int
    L.kvm_prefill.argtypes = [vp, vp, vp, vp, C.c_int32, Growth, C.c_int32, C.c_int64, vp, vp, C.POINTER(Strides), vp]
    L.kvm_decode_step.restype = C.c_int
    L.kvm_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.kvm_prefill_host.restype = C.c_int
    L.kvm_prefill_host.argtypes = [vp, vp, vp, vp, C.c_int32, Growth, C.c_int32, C.c_int64, vp, vp, vp]
    L.kvm_decode_step_host.restype = C.c_int
    L.kvm_decode_step_host.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.kvm_state_free.restype = C.c_int
    L.kvm_state_free.argtypes = [vp]
    L.kvm_state_info.restype = C.c_int
    L.kvm_state_info.argtypes = [vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
    L.kvm_state_check.restype = C.c_int
    L.kvm_state_check.argtypes = [vp, vp]
    L.kvm_state_export.restype = C.c_int
    L.kvm_state_export.argtypes = [vp] * 9
    L.kvm_debug_assignments.restype = C.c_int
    L.kvm_debug_assignments.argtypes = [vp, C.c_int64, vp, vp, vp]
    L.kvm_state_reset.restype = C.c_int
    L.kvm_state_reset.argtypes = [vp]
    L.kvm_profile_enable.restype = C.c_int
    L.kvm_profile_enable.argtypes = [vp, C.c_int32]
    L.kvm_profile_read.restype = C.c_int
    L.kvm_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
    L.kvm_debug_counters.restype = C.c_int
    L.kvm_debug_counters.argtypes = [vp, C.POINTER(C.c_int64), vp]
    L.kvm_launch_count.restype = C.c_int64
    L.kvm_launch_count.argtypes = [vp]
    L.kvm_attend_rows_noalloc.restype = C.c_int
    L.kvm_attend_rows_noalloc.argtypes = [vp, vp, vp, C.c_int32, C.c_int64, C.c_int32, C.c_float, vp, vp]
    L.kvm_merge_gate.restype = C.c_int
    L.kvm_merge_gate.argtypes = [vp, vp, C.c_int32, C.c_int64, C.c_int32, C.c_int32, vp, vp, vp]
    L.kvm_debug_drop_exchange.restype = C.c_int
    L.kvm_debug_drop_exchange.argtypes = [vp, C.c_int32]
    L.kvm_debug_decode_plan.restype = C.c_int
    L.kvm_debug_decode_plan.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.POINTER(C.c_int32)]
    L.kvm_debug_decode_ahead.restype = C.c_int
    L.kvm_debug_decode_ahead.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.POINTER(C.c_int32)]
    L.kvm_debug_apply_plan.restype = C.c_int
    L.kvm_debug_apply_plan.argtypes = [C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]
    L.kvm_debug_attention_plan.restype = C.c_int
    L.kvm_debug_attention_plan.argtypes = [C.c_int32] * 5 + [C.c_int64, C.c_int32, C.POINTER(C.c_int32)]
    L.kvm_debug_expire_wait.restype = C.c_int
    L.kvm_debug_expire_wait.argtypes = [vp, C.c_int32, vp]
    L.kvm_head_layernorm.restype = C.c_int
    L.kvm_head_layernorm.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, C.c_int64, C.c_int32, C.c_float, vp]
    L.kvm_state_snapshot_info.restype = C.c_int
    L.kvm_state_snapshot_info.argtypes = [vp, C.POINTER(SnapshotInfo)]
    L.kvm_state_export_window.restype = C.c_int
    L.kvm_state_export_window.argtypes = [vp, vp, vp, vp, vp]
    L.kvm_state_import.restype = C.c_int
    L.kvm_state_import.argtypes = [vp, C.POINTER(SnapshotInfo)] + [vp] * 9
    cd, cc, i32p, i64p = C.POINTER(CacheDesc), C.POINTER(CacheCall), C.POINTER(C.c_int32), C.POINTER(C.c_int64)
    fd = C.POINTER(FrontDesc)
    L.kvm_rope_frequencies.restype = C.c_int
    L.kvm_rope_frequencies.argtypes = [fd, C.c_int32, vp]
    L.kvm_qk_norm_rope.restype = C.c_int
    L.kvm_qk_norm_rope.argtypes = [fd, vp, vp, vp, vp, C.c_int32, C.c_int32, C.c_int32, C.c_int64, C.c_int32, vp, vp, i64p, i64p, i64p, i64p, vp, vp]
    L.kvm_cache_ingest.restype = C.c_int
    L.kvm_cache_ingest.argtypes = [cd, cc, fd, vp, C.c_int32, vp, vp, vp, i64p, i64p, i64p, i64p, vp, vp]
    L.kvm_cache_read.restype = C.c_int
    L.kvm_cache_read.argtypes = [cd, cc, vp, vp, i64p, i64p, vp, vp]
    L.kvm_cache_append.restype = C.c_int
    L.kvm_cache_append.argtypes = [cd, cc, vp, vp, i64p, i64p, vp, vp]
    L.kvm_cache_attend.restype = C.c_int
    L.kvm_cache_attend.argtypes = [cd, cc, vp, C.c_int32, C.c_float, C.c_int32, C.c_int32, vp, i64p, i64p, vp, C.c_int64, vp, vp]
    L.kvm_cache_workspace.restype = C.c_int64
    L.kvm_cache_workspace.argtypes = [cd, cc, C.c_int32]
    L.kvm_cache_attend_shared.restype = C.c_int
    L.kvm_cache_attend_shared.argtypes = [cd, cc, vp, vp, C.c_int32, vp, C.c_int32, C.c_float, vp, i64p, i64p, vp, C.c_int64, vp, vp]
    L.kvm_cache_shared_workspace.restype = C.c_int64
    L.kvm_cache_shared_workspace.argtypes = [cd, cc, C.c_int32, C.c_int32]
    L.kvm_pages_shared.restype = C.c_int
    L.kvm_pages_shared.argtypes = [vp, i32p, C.c_int64, C.c_int64, i32p]
    L.kvm_cache_copy_pages.restype = C.c_int
    L.kvm_cache_copy_pages.argtypes = [cd, vp, vp, C.c_int64, vp]
    L.kvm_pages_create.restype = C.c_int
    L.kvm_pages_create.argtypes = [C.c_int64, C.c_int32, C.POINTER(vp)]
    L.kvm_pages_destroy.restype = C.c_int
    L.kvm_pages_destroy.argtypes = [vp]
    L.kvm_pages_open.restype = C.c_int
    L.kvm_pages_open.argtypes = [vp, i32p]
    L.kvm_pages_fork.restype = C.c_int
    L.kvm_pages_fork.argtypes = [vp, C.c_int32, i32p]
    L.kvm_pages_close.restype = C.c_int
    L.kvm_pages_close.argtypes = [vp, C.c_int32]
    L.kvm_pages_extend.restype = C.c_int
    L.kvm_pages_extend.argtypes = [vp, C.c_int32, C.c_int64, i32p, i32p]
    L.kvm_pages_trim.restype = C.c_int
    L.kvm_pages_trim.argtypes = [vp, C.c_int32, C.c_int32, C.c_int32]
    L.kvm_pages_compact.restype = C.c_int
    L.kvm_pages_compact.argtypes = [vp, vp, vp, C.c_int64, i64p]
    L.kvm_pages_table.restype = C.c_int
    L.kvm_pages_table.argtypes = [vp, C.c_int32, vp, C.c_int64, i64p, i64p]
    L.kvm_pages_info.restype = C.c_int
    L.kvm_pages_info.argtypes = [vp, i64p, i64p]
    L.kvm_status_string.restype = C.c_char_p
    L.kvm_status_string.argtypes = [C.c_int]
    return L


lib = _load()


def growth(kind: str, fixed_slots: int = 0, sqrt_coeff: int = 16, pow_num: int = 1, pow_den: int = 2,
           sat_half: int = 0) -> Growth:
    """fixed: B = fixed_slots; sqrt: floor(sqrt_coeff sqrt(e)); power: floor(sqrt_coeff e^(pow_num/pow_den));
    saturating: floor(fixed_slots e / (e + sat_half)); unbounded: no budget."""
    k = {"fixed": GROWTH_FIXED, "sqrt": GROWTH_SQRT, "unbounded": GROWTH_UNBOUNDED, "power": GROWTH_POWER,
         "saturating": GROWTH_SATURATING}[kind]
    return Growth(k, sqrt_coeff, fixed_slots, pow_num, pow_den, sat_half)


def merge_gate(x: "torch.Tensor", w_gate: "torch.Tensor", out=None, stream=None, status=None) -> "torch.Tensor":
    """g = 1 + ELU(x W_g): x bf16 [B, T, d_model], w_gate fp32 [Hkv, d_model] -> fp32 [B, Hkv, T]
    (argument marshalling only; the product runs in kvm_merge_gate).  `status`: optional int32 CUDA tensor
    of one element that receives KVM_ERR_TIMEOUT should a bounded device-side wait run out."""
    assert x.is_cuda and w_gate.is_cuda and x.dtype == torch.bfloat16 and w_gate.dtype == torch.float32
    assert x.is_contiguous() and w_gate.is_contiguous() and x.dim() == 3 and w_gate.dim() == 2
    B, T, dm = x.shape
    H = w_gate.shape[0]
    assert w_gate.shape[1] == dm
    if out is None:
        out = torch.empty((B, H, T), dtype=torch.float32, device=x.device)
    rc = lib.kvm_merge_gate(C.c_void_p(x.data_ptr()), C.c_void_p(w_gate.data_ptr()), B, T, dm, H,
                            C.c_void_p(out.data_ptr()), C.c_void_p(status.data_ptr()) if status is not None else None,
                            _stream_ptr(stream))
    if rc != 0:
        raise KVMError(rc, "kvm_merge_gate")
    return out


def head_layernorm(x: "torch.Tensor", weight=None, bias=None, eps: float = 1e-5, stream=None) -> "torch.Tensor":
    """LN_q / LN_k in place: x bf16 [B, H, T, d] contiguous; weight, bias fp32 [H, d] on the device or None."""
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.is_contiguous() and x.dim() == 4
    B, H, T, d = x.shape
    for t in (weight, bias):
        assert t is None or (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and tuple(t.shape) == (H, d))
    rc = lib.kvm_head_layernorm(C.c_void_p(x.data_ptr()), C.c_void_p(weight.data_ptr() if weight is not None else 0),
                                C.c_void_p(bias.data_ptr() if bias is not None else 0), B, H, T, d, eps, _stream_ptr(stream))
    if rc != 0:
        raise KVMError(rc, "kvm_head_layernorm")
    return x


def _plan(fn, n, *args):
    out = (C.c_int32 * n)()
    rc = getattr(lib, fn)(*args, out)
    if rc != KVM_OK:
        raise KVMError(rc, fn)
    return tuple(out)


def decode_plan(batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, n_rows: int):
    """(query heads per CTA, CTAs per cluster, clusters per group of heads) of a decode step over n_rows rows in the kernel that
    loops over them (decode_ahead says whether the step runs that one)."""
    return _plan("kvm_debug_decode_plan", 3, batch, n_q_heads, n_kv_heads, head_dim, n_rows)


def decode_ahead(batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, n_rows: int):
    """(CTAs per group of query heads, query heads per CTA, rows per warp) of a decode step over n_rows rows in the kernel that
    fetches its rows ahead; (0, 0, 0): the step runs the kernel that loops over them."""
    return _plan("kvm_debug_decode_ahead", 3, batch, n_q_heads, n_kv_heads, head_dim, n_rows)


def apply_plan(n_units: int, head_dim: int, block: int, serial: bool = False, group: int = 1):
    """(rows per warp, CTAs per unit) of the kernel that writes the rows a fold touches; group: query heads per unit."""
    return _plan("kvm_debug_apply_plan", 2, n_units, group, head_dim, block, 1 if serial else 0)


def attention_plan(batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, n_queries: int, n_slots: int, decides: bool = True):
    """(CTAs that run whole, key splits of each of the others) of the attention of n_queries tokens of a block over n_slots rows;
    decides: a fold that compares its tokens with the state runs beside it."""
    return _plan("kvm_debug_attention_plan", 2, batch, n_q_heads, n_kv_heads, head_dim, n_queries, n_slots, 1 if decides else 0)


def kvm_plan_capacity(block: int, n_bswa_chunks: int, g: Growth, seq_len: int) -> int:
    return lib.kvm_plan_capacity(block, n_bswa_chunks, g, seq_len)


def _fp(a):
    if a is None:
        return None, None
    arr = np.ascontiguousarray(np.asarray(a, dtype=np.float32))
    return arr, arr.ctypes.data_as(C.POINTER(C.c_float))


def _stream_ptr(stream):
    if stream is not None:
        return stream.cuda_stream
    if not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream
    # the current stream of the current device, without the Stream object around it
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def attend_rows_noalloc(q, keys, values, scale: float, out=None, stream=None):
    """kvm_attend_rows_noalloc: out[h] = softmax(scale * q[h] . keys[h]^T) . values[h] for callers that may not
    allocate device memory inside the call (the split partials live in a fixed array of the library).
    q [H,d] fp16, keys/values [H,n,d] fp16 contiguous CUDA tensors; `out` [H,d] bf16 should be passed by such
    callers (it is only created here for convenience when omitted)."""
    assert q.dtype == torch.float16 and keys.dtype == torch.float16 and values.dtype == torch.float16
    assert q.is_contiguous() and keys.is_contiguous() and values.is_contiguous()
    H, n, d = keys.shape
    if out is None:
        out = torch.empty((H, d), dtype=torch.bfloat16, device=q.device)
    rc = lib.kvm_attend_rows_noalloc(C.c_void_p(q.data_ptr()), C.c_void_p(keys.data_ptr()), C.c_void_p(values.data_ptr()),
                                     H, n, d, scale, C.c_void_p(out.data_ptr()), _stream_ptr(stream))
    if rc != KVM_OK:
        raise KVMError(rc, "kvm_attend_rows_noalloc")
    return out


@dataclass
class LayerConfig:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    max_block: int
    max_state_slots: int
    max_call_tokens: int
    n_bswa_chunks: int = 2
    sink_len: int = 1
    rope_base: float = 10000.0
    ln_eps: float = 1e-5
    norm_eps: float = 1e-12
    max_seq_len: int = 0
    device: int = 0
    flags: int = 0


class KVMState:
    """Owns one kvm_state_t.  Methods map 1:1 to the C entry points of the same name."""

    def __init__(self, cfg: LayerConfig, ln_weight=None, ln_bias=None, tau_state=None, tau_bswa=None, qk_ln=None):
        """qk_ln: dict(eps, q_weight, q_bias, k_weight, k_bias) turns the fused front end on (KVM_FLAG_FUSED_QK_LN)."""
        self.cfg = cfg
        keep = [_fp(ln_weight), _fp(ln_bias), _fp(tau_state), _fp(tau_bswa)]
        flags, eps = cfg.flags, 0.0
        ln4 = [(None, None)] * 4
        if qk_ln is not None:
            flags |= FLAG_FUSED_QK_LN
            eps = float(qk_ln.get("eps", 1e-5))
            ln4 = [_fp(qk_ln.get(n)) for n in ("q_weight", "q_bias", "k_weight", "k_bias")]
        c = Config(cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.n_bswa_chunks, cfg.sink_len,
                   cfg.rope_base, cfg.ln_eps, cfg.norm_eps, keep[0][1], keep[1][1], keep[2][1], keep[3][1],
                   cfg.max_block, cfg.max_state_slots, cfg.max_call_tokens, cfg.max_seq_len, cfg.device, flags,
                   eps, ln4[0][1], ln4[1][1], ln4[2][1], ln4[3][1])
        h = C.c_void_p()
        rc = lib.kvm_state_create(C.byref(c), C.byref(h))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_state_create")
        self._h = h
        self.U = cfg.batch * cfg.n_kv_heads

    def free(self):
        if getattr(self, "_h", None):
            lib.kvm_state_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    # -- kvm_prefill ---------------------------------------------------------------------
    def prefill(self, q, k, v, block: int, g: Growth, rope_dims: int, out=None, gate=None, stream=None):
        """q [B,Hq,n,d], k,v [B,Hkv,n,d] bf16 CUDA tensors (last dim contiguous)."""
        assert q.is_cuda and q.dtype == torch.bfloat16 and k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16
        n = q.shape[2]
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        st = Strides()
        for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
            arr = getattr(st, name)
            for i in range(4):
                arr[i] = t.stride(i)
        gp = None
        if gate is not None:
            assert gate.dtype == torch.float32 and gate.is_contiguous() and gate.is_cuda
            gp = C.c_void_p(gate.data_ptr())
        rc = lib.kvm_prefill(C.c_void_p(q.data_ptr()), C.c_void_p(k.data_ptr()), C.c_void_p(v.data_ptr()), self._h,
                             block, g, rope_dims, n, gp, C.c_void_p(out.data_ptr()), C.byref(st), _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_prefill")
        return out

    # -- kvm_decode_step -----------------------------------------------------------------
    def decode_step(self, q, k, v, out=None, gate=None, stream=None):
        """q [B,Hq,d], k,v [B,Hkv,d] contiguous bf16 CUDA tensors."""
        assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        # (plain integers: ctypes converts them by the argument types, and a step is short enough for the
        # objects around a pointer to show)
        rc = lib.kvm_decode_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), self._h,
                                 gate.data_ptr() if gate is not None else None, out.data_ptr(), _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_decode_step")
        return out

    # -- host-buffer variants ------------------------------------------------------------
    def prefill_host(self, q, k, v, block: int, g: Growth, rope_dims: int, out, gate=None, stream=None):
        """Contiguous bf16 CPU tensors (pinned for speed); `out` is a CPU tensor that is filled."""
        for t in (q, k, v, out):
            assert (not t.is_cuda) and t.is_contiguous() and t.dtype == torch.bfloat16
        gp = C.c_void_p(gate.data_ptr()) if gate is not None else None
        rc = lib.kvm_prefill_host(C.c_void_p(q.data_ptr()), C.c_void_p(k.data_ptr()), C.c_void_p(v.data_ptr()),
                                  self._h, block, g, rope_dims, q.shape[2], gp, C.c_void_p(out.data_ptr()),
                                  _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_prefill_host")
        return out

    def decode_step_host(self, q, k, v, out, gate=None, stream=None):
        for t in (q, k, v, out):
            assert (not t.is_cuda) and t.is_contiguous() and t.dtype == torch.bfloat16
        gp = C.c_void_p(gate.data_ptr()) if gate is not None else None
        rc = lib.kvm_decode_step_host(C.c_void_p(q.data_ptr()), C.c_void_p(k.data_ptr()), C.c_void_p(v.data_ptr()),
                                      self._h, gp, C.c_void_p(out.data_ptr()), _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_decode_step_host")
        return out

    # -- inspection ----------------------------------------------------------------------
    def info(self):
        a, b, c = C.c_int64(), C.c_int64(), C.c_int64()
        rc = lib.kvm_state_info(self._h, C.byref(a), C.byref(b), C.byref(c))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_state_info")
        return dict(n_slots=a.value, position=b.value, n_folds=c.value)

    def check(self, stream=None):
        return lib.kvm_state_check(self._h, _stream_ptr(stream))

    def reset(self):
        rc = lib.kvm_state_reset(self._h)
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_state_reset")

    def profile_enable(self, on=True):
        lib.kvm_profile_enable(self._h, 1 if on else 0)

    def profile_read(self):
        """Returns {phase: (milliseconds, bracket count)} accumulated since the last read."""
        ms = (C.c_double * 8)(); n = (C.c_int64 * 8)()
        rc = lib.kvm_profile_read(self._h, ms, n)
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_profile_read")
        names = ("ingest", "attention", "kbar", "route_filter", "fold_decide", "fold_apply", "decode")
        return {names[i]: (ms[i], n[i]) for i in range(7)}

    def debug_counters(self, stream=None):
        out = (C.c_int64 * 4)()
        rc = lib.kvm_debug_counters(self._h, out, _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_debug_counters")
        return dict(exhaustive_tokens=out[0], candidate_pairs=out[1], tokens=out[2], clamped_inputs=out[3])

    def debug_expire_wait(self, spins: int = 10000, stream=None):
        rc = lib.kvm_debug_expire_wait(self._h, spins, _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_debug_expire_wait")

    def debug_drop_exchange(self, unit: int):
        rc = lib.kvm_debug_drop_exchange(self._h, unit)
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_debug_drop_exchange")

    def launch_count(self):
        return lib.kvm_launch_count(self._h)

    def export(self, readout=True, stream=None):
        m, d, U = self.info()["n_slots"], self.cfg.head_dim, self.U
        sk = np.zeros((U, m, d), np.float64); sv = np.zeros((U, m, d), np.float32)
        rho = np.zeros((U, m), np.float32); w = np.zeros((U, m), np.float64); cnt = np.zeros((U, m), np.int32)
        kr = torch.zeros((U, m, d), dtype=torch.float16) if readout else None
        vr = torch.zeros((U, m, d), dtype=torch.float16) if readout else None
        p = lambda a: C.c_void_p(a.ctypes.data)
        rc = lib.kvm_state_export(self._h, p(sk), p(sv), p(rho), p(w), p(cnt),
                                  C.c_void_p(kr.data_ptr()) if readout else None,
                                  C.c_void_p(vr.data_ptr()) if readout else None, _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_state_export")
        return dict(sum_k=sk, sum_v=sv, radius=rho, weight=w, count=cnt, k_read=kr, v_read=vr)

    def snapshot(self, stream=None):
        """kvm_state_snapshot_info + kvm_state_export + kvm_state_export_window: everything kvm_state_import needs."""
        info = SnapshotInfo()
        rc = lib.kvm_state_snapshot_info(self._h, C.byref(info))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_state_snapshot_info")
        snap = self.export(readout=False, stream=stream)
        n, d = info.window_len, self.cfg.head_dim
        wk = torch.zeros((self.U, n, d), dtype=torch.float16); wv = torch.zeros((self.U, n, d), dtype=torch.float16)
        wg = np.zeros((self.U, n), np.float32)
        if info.block > 0:
            rc = lib.kvm_state_export_window(self._h, C.c_void_p(wk.data_ptr()), C.c_void_p(wv.data_ptr()),
                                             C.c_void_p(wg.ctypes.data), _stream_ptr(stream))
            if rc != KVM_OK:
                raise KVMError(rc, "kvm_state_export_window")
        snap.update(info=info, win_k=wk, win_v=wv, win_gate=wg)
        return snap

    def restore(self, snap, stream=None):
        """kvm_state_import of a snapshot() (possibly taken from another state of the same shape)."""
        p = lambda a: C.c_void_p(a.ctypes.data) if a is not None and a.size else None
        t = lambda a: C.c_void_p(a.data_ptr()) if a is not None and a.numel() else None
        rc = lib.kvm_state_import(self._h, C.byref(snap["info"]), p(snap["sum_k"]), p(snap["sum_v"]), p(snap["radius"]),
                                  p(snap["weight"]), p(snap["count"]), t(snap["win_k"]), t(snap["win_v"]),
                                  p(snap.get("win_gate")), _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_state_import")

    def assignments(self, n=None, stream=None):
        n = self.info()["position"] if n is None else n
        slot = np.zeros((self.U, n), np.int32); app = np.zeros((self.U, n), np.uint8)
        rc = lib.kvm_debug_assignments(self._h, n, C.c_void_p(slot.ctypes.data), C.c_void_p(app.ctypes.data),
                                       _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_debug_assignments")
        return slot, app


_THREE = C.c_int64 * 3
_INT32, _BF16 = torch.int32, torch.bfloat16


def _strides3(t):
    """Element strides of the first three dims; None where the tensor is contiguous."""
    if t.is_contiguous():
        return None
    b, h, n, c = t.stride()
    if c != 1 and t.shape[3] > 1:
        raise ValueError("the channels of a row must be contiguous")
    return _THREE(b, h, n)


def _int(x, bits=32):
    """x as a number that a C integer of so many bits holds (ctypes would cut off the rest)."""
    x = operator.index(x)
    if not -(1 << bits - 1) <= x < 1 << bits - 1:
        raise ValueError(f"{x} does not fit into {bits} bits")
    return x


def _page_list(x):
    """Page numbers on the host as contiguous int32."""
    if not isinstance(x, torch.Tensor):
        x = torch.as_tensor(x)
    if x.is_cuda or x.dim() != 1:
        raise ValueError("src and dst are lists of page numbers on the host")
    if x.dtype == torch.int32:
        return x.contiguous()
    if x.numel():
        if x.dtype == torch.bool or x.is_floating_point() or x.is_complex():
            raise ValueError("page numbers are whole numbers")
        x = x.to(torch.int64)
        if x.min() < -(1 << 31) or x.max() >= 1 << 31:
            raise ValueError("page numbers are of 32 bits")
    return x.to(torch.int32)


class Front:
    """What an exact layer does to q and k before its attention (kvm_front_t): norm "layer", "rms" or "none" of every head's row, then rotary positions
    in its first `rope_dims` channels, layout "half" (pairs i, i + r/2) or "interleaved" (2i, 2i + 1), scaling "none", "linear" or "parts" (factor, original_len,
    low, high), cos and sin times `magnitude`.  Weights and biases: contiguous fp32 CUDA tensors [heads, head_dim] or None; they are kept."""

    def __init__(self, norm="layer", eps: float = 1e-5, rope_dims: int = 0, layout="half", base: float = 10000.0, scaling="none", factor: float = 1.0,
                 original_len: int = 0, low: float = 1.0, high: float = 32.0, magnitude: float = 1.0, q_weight=None, q_bias=None, k_weight=None, k_bias=None):
        kinds = []
        for x, names in ((norm, ("none", "layer", "rms")), (layout, ("half", "interleaved")), (scaling, ("none", "linear", "parts"))):
            if x not in names:
                raise ValueError(f"{x!r} is none of {names}")
            kinds.append(names.index(x))
        self._affine = (q_weight, q_bias, k_weight, k_bias)
        self._device = -1
        for t in self._affine:
            if t is not None:
                if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.dim() != 2 or self._device not in (-1, t.get_device()):
                    raise ValueError("weights and biases are contiguous float32 [heads, head_dim] on one CUDA device")
                self._device = t.get_device()
        self._shapes = []
        for pair in (self._affine[:2], self._affine[2:]):
            shapes = [tuple(t.shape) for t in pair if t is not None]
            if len(set(shapes)) > 1:
                raise ValueError("a bias has its weight's shape")
            self._shapes.append(shapes[0] if shapes else None)
        self.rope_dims = _int(rope_dims)
        self._desc = FrontDesc(*kinds, self.rope_dims, base, factor, low, high, magnitude, _int(original_len, 64), eps, None,
                               *(t.data_ptr() if t is not None else None for t in self._affine))
        self._ref = C.byref(self._desc)
        if self.rope_dims > 0:
            # computed once (for one of the two widths of heads that there are: they do not depend on it)
            self._frequencies = (C.c_double * 64)()
            if lib.kvm_rope_frequencies(self._ref, 128, self._frequencies) == KVM_OK:   # (what is wrong with the rest, a call says)
                self._desc.frequencies = C.cast(self._frequencies, C.POINTER(C.c_double))

    def frequencies(self, head_dim: int):
        """Radians per position of each pair (kvm_rope_frequencies), a list of rope_dims / 2."""
        out = (C.c_double * max(1, self.rope_dims // 2))()
        rc = lib.kvm_rope_frequencies(self._ref, _int(head_dim), out)
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_rope_frequencies")
        return list(out[:self.rope_dims // 2])


def _front_rows(x, out, device, front, which, batch, tokens, head_dim):
    """Checks rows of q (which 0), k (1) or v (2) and their out, or None, for a front-end call; their number of heads."""
    if x.dtype is not _BF16 or x.get_device() != device or x.dim() != 4:
        raise ValueError("rows are bfloat16 [batch, heads, tokens, head_dim] on one CUDA device")
    B, H, T, d = shape = x.shape
    if B != batch or T != tokens or d != head_dim:
        raise ValueError("q, k and v have the same batch, tokens and head_dim")
    if out is not None and (out.shape != shape or out.dtype is not _BF16 or out.get_device() != device):
        raise ValueError("an out has its input's shape, type and device")
    if which < 2 and front._shapes[which] is not None and (front._shapes[which] != (H, d) or front._device != device):
        raise ValueError("weights and biases [heads, head_dim] on the rows' device")
    return H


def _other_stream(stream):
    """Whether a stream is given that is not the current one."""
    return stream is not None and stream != torch.cuda.current_stream()


def qk_norm_rope(q, k, front: Front, start=None, count=None, q_out=None, k_out=None, status=None, stream=None):
    """kvm_qk_norm_rope: q bf16 [B, n_q_heads, T, head_dim] and k bf16 [B, n_kv_heads, T, head_dim] (channels contiguous; either may be None) through
    `front`, at positions start[b] + t (start None: t).  Returns (q_out, k_out), made here unless given; an out may be its input.  Rows behind a sequence's
    count are left as they were (unset where the out is made here).  `status` as in Cache."""
    x = q if q is not None else k
    if x is None:
        raise ValueError("q or k")
    device = x.get_device()
    if device < 0 or x.dim() != 4:
        raise ValueError("rows are bfloat16 [batch, heads, tokens, head_dim] on one CUDA device")
    B, _, T, d = x.shape
    Hq = _front_rows(q, q_out, device, front, 0, B, T, d) if q is not None else 0
    Hk = _front_rows(k, k_out, device, front, 1, B, T, d) if k is not None else 0
    for t in (start, count, status):
        if t is not None and (t.dtype is not _INT32 or not t.is_contiguous() or t.get_device() != device or (t is not status and t.numel() != B)):
            raise ValueError("start [batch], count [batch] and status are contiguous int32 tensors on the rows' device")
    if torch._C._cuda_getDevice() != device or _other_stream(stream):
        with torch.cuda.device(device), torch.cuda.stream(stream):   # (memory made here comes from the stream's own)
            return qk_norm_rope(q, k, front, start, count, q_out, k_out, status)
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    if k is not None and k_out is None:
        k_out = torch.empty(k.shape, dtype=torch.bfloat16, device=k.device)
    rc = lib.kvm_qk_norm_rope(front._ref, q.data_ptr() if Hq else None, k.data_ptr() if Hk else None, start.data_ptr() if start is not None else None,
                              count.data_ptr() if count is not None else None, B, Hq, Hk, T, d, q_out.data_ptr() if Hq else None, k_out.data_ptr() if Hk else None,
                              _strides3(q) if Hq else None, _strides3(k) if Hk else None, _strides3(q_out) if Hq else None, _strides3(k_out) if Hk else None,
                              status.data_ptr() if status is not None else None, _stream_ptr(None))
    if rc != KVM_OK:
        raise KVMError(rc, "kvm_qk_norm_rope")
    return q_out, k_out


class Cache:
    """A pool of pages for exact keys and values in 8 bits (kvm_cache_t): codes k8, v8 float8_e4m3fn [n_pages, n_kv_heads, page_tokens,
    head_dim], scales fp32 [n_pages, n_kv_heads] (powers of two; a row stands for code * scale).  The tensors are the caller's;
    Cache.empty makes them.  Which page holds what is the caller's too (Pages keeps book of it).

    pages int32 [B, max_pages], start int32 [B] (tokens in the cache before the call) and count int32 [B] (tokens of the call; None: all of
    them) are CUDA tensors.  `status`: optional int32 CUDA tensor of one element that receives KVM_ERR_INVALID_ARG where the kernels
    meet lengths or pages that the call does not allow, KVM_ERR_TIMEOUT should a bounded device-side wait run out.  Arguments that the
    binding can see to be wrong, numbers beyond 32 bits among them, raise ValueError."""

    def __init__(self, k8, v8, k_scale, v_scale):
        if k8.dim() != 4 or v8.shape != k8.shape or k_scale.shape != k8.shape[:2] or v_scale.shape != k8.shape[:2]:
            raise ValueError("k8, v8 [n_pages, n_kv_heads, page_tokens, head_dim], k_scale, v_scale [n_pages, n_kv_heads]")
        for t, dt in ((k8, torch.float8_e4m3fn), (v8, torch.float8_e4m3fn), (k_scale, torch.float32), (v_scale, torch.float32)):
            if t.dtype != dt or not t.is_cuda or not t.is_contiguous() or t.device != k8.device:
                raise ValueError("codes are contiguous float8_e4m3fn, scales contiguous float32, on one CUDA device")
        self.k8, self.v8, self.k_scale, self.v_scale = k8, v8, k_scale, v_scale
        self.n_pages, self.n_kv_heads, self.page_tokens, self.head_dim = k8.shape
        self._device = k8.device
        self._desc = CacheDesc(k8.data_ptr(), v8.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), self.n_pages, self.n_kv_heads,
                               self.head_dim, self.page_tokens)
        self._ref = C.byref(self._desc)

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, head_dim: int, page_tokens: int = 64, device="cuda"):
        codes = [torch.zeros((n_pages, n_kv_heads, page_tokens, head_dim), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)
                 for _ in range(2)]
        return cls(*codes, *(torch.ones((n_pages, n_kv_heads), dtype=torch.float32, device=device) for _ in range(2)))

    def _call(self, pages, start, count, rows, status):
        B, _, T, _ = rows[0].shape
        dev = self._device.index
        for t in (pages, start, count, status):
            if t is not None and (t.dtype is not _INT32 or t.get_device() != dev or not t.is_contiguous()):
                raise ValueError("pages, start, count and status are contiguous int32 tensors on the cache's device")
        for t in rows:
            if t.dtype is not _BF16 or t.get_device() != dev:
                raise ValueError("rows are bfloat16 on the cache's device")
        if pages.dim() != 2 or pages.shape[0] != B or start.numel() != B or (count is not None and count.numel() != B):
            raise ValueError("pages [batch, max_pages], start [batch], count [batch]")
        return C.byref(CacheCall(pages.data_ptr(), start.data_ptr(), count.data_ptr() if count is not None else None, B, pages.shape[1], T))

    def _elsewhere(self):
        """Whether another device than the cache's is the current one."""
        return torch._C._cuda_getDevice() != self._device.index

    def append(self, k, v, pages, start, count=None, status=None, stream=None):
        """kvm_cache_append: k, v bf16 [B, n_kv_heads, T, head_dim] (channels contiguous) behind the tokens that the sequences hold."""
        if k.dim() != 4 or v.shape != k.shape or k.shape[1] != self.n_kv_heads or k.shape[3] != self.head_dim:
            raise ValueError("k, v [batch, n_kv_heads, tokens, head_dim]")
        if self._elsewhere():
            with torch.cuda.device(self._device):
                return self.append(k, v, pages, start, count, status, stream)
        call = self._call(pages, start, count, (k, v), status)
        rc = lib.kvm_cache_append(self._ref, call, k.data_ptr(), v.data_ptr(), _strides3(k), _strides3(v),
                                  status.data_ptr() if status is not None else None, _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_cache_append")

    def ingest(self, q, k, v, front: Front, pages, start, count=None, q_out=None, status=None, stream=None):
        """kvm_cache_ingest: q and k bf16 [B, heads, T, head_dim] through `front` at positions start[b] + t, k and v into the cache behind the tokens that the
        sequences hold.  Returns q_out, made here unless given; it may be q.  q may be None: k and v only."""
        if k.dim() != 4 or k.shape[1] != self.n_kv_heads or k.shape[3] != self.head_dim or v.shape != k.shape:
            raise ValueError("k, v [batch, n_kv_heads, tokens, head_dim]")
        device = self._device.index
        B, _, T, d = k.shape
        _front_rows(k, None, device, front, 1, B, T, d)
        _front_rows(v, None, device, front, 2, B, T, d)
        if q is None:
            if q_out is not None:
                raise ValueError("q_out without q")
            Hq = 0
        else:
            Hq = _front_rows(q, q_out, device, front, 0, B, T, d)
        if torch._C._cuda_getDevice() != device or _other_stream(stream):
            with torch.cuda.device(self._device), torch.cuda.stream(stream):   # (memory made here comes from the stream's own)
                return self.ingest(q, k, v, front, pages, start, count, q_out, status)
        if Hq and q_out is None:
            q_out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        call = self._call(pages, start, count, (k,), status)
        rc = lib.kvm_cache_ingest(self._ref, call, front._ref, q.data_ptr() if Hq else None, Hq, k.data_ptr(), v.data_ptr(), q_out.data_ptr() if Hq else None,
                                  _strides3(q) if Hq else None, _strides3(k), _strides3(v), _strides3(q_out) if Hq else None,
                                  status.data_ptr() if status is not None else None, _stream_ptr(None))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_cache_ingest")
        return q_out

    def read(self, pages, start, n_tokens: int, count=None, k_out=None, v_out=None, status=None, stream=None):
        """kvm_cache_read: positions start[b] .. start[b] + count[b] - 1 as bf16 [B, n_kv_heads, n_tokens, head_dim], (k_out, v_out), made here unless given.  Rows behind a
        sequence's count are left as they were (unset where made here)."""
        shape = (pages.shape[0], self.n_kv_heads, _int(n_tokens), self.head_dim)
        for t in (k_out, v_out):
            if t is not None and tuple(t.shape) != shape:
                raise ValueError("k_out, v_out [batch, n_kv_heads, n_tokens, head_dim]")
        if self._elsewhere() or _other_stream(stream):
            with torch.cuda.device(self._device), torch.cuda.stream(stream):   # (memory made here comes from the stream's own)
                return self.read(pages, start, n_tokens, count, k_out, v_out, status)
        k_out, v_out = (torch.empty(shape, dtype=torch.bfloat16, device=self._device) if t is None else t for t in (k_out, v_out))
        call = self._call(pages, start, count, (k_out, v_out), status)
        rc = lib.kvm_cache_read(self._ref, call, k_out.data_ptr(), v_out.data_ptr(), _strides3(k_out), _strides3(v_out),
                                status.data_ptr() if status is not None else None, _stream_ptr(None))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_cache_read")
        return k_out, v_out

    def attend(self, q, pages, start, count=None, window: int = 0, sinks: int = 0, scale=None, out=None, status=None, stream=None):
        """kvm_cache_attend: q bf16 [B, n_q_heads, T, head_dim] over the cache, which holds the T tokens' own keys already; a token sees
        the last `window` positions up to its own (0: all) and the first `sinks`.  scale: 1 / sqrt(head_dim) unless given.  Rows of `out`
        behind a sequence's count are left as they were (unset where `out` is made here)."""
        window, sinks = _int(window), _int(sinks)
        if q.dim() != 4 or q.shape[3] != self.head_dim or (out is not None and out.shape != q.shape):
            raise ValueError("q, out [batch, n_q_heads, tokens, head_dim]")
        if self._elsewhere() or (stream is not None and stream != torch.cuda.current_stream()):
            # (memory made here comes from the stream's own: neither a call on another stream nor another captured graph gets the same bytes)
            with torch.cuda.device(self._device), torch.cuda.stream(stream):
                return self.attend(q, pages, start, count, window, sinks, scale, out, status)
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        call = self._call(pages, start, count, (q, out), status)
        Hq = q.shape[1]
        n = lib.kvm_cache_workspace(self._ref, call, Hq)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n > 0 else None
        rc = lib.kvm_cache_attend(self._ref, call, q.data_ptr(), Hq, self.head_dim ** -0.5 if scale is None else scale, window, sinks,
                                  out.data_ptr(), _strides3(q), _strides3(out), ws.data_ptr() if n > 0 else None, max(n, 0),
                                  status.data_ptr() if status is not None else None, _stream_ptr(None))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_cache_attend")
        return out

    def attend_shared(self, q, pages, start, groups, shared, count=None, scale=None, out=None, status=None, stream=None):
        """kvm_cache_attend_shared: attend (window 0) where sequences groups[g] .. groups[g + 1] - 1 have their first shared[g] blocks in common, which are read
        for the group together.  groups int32 [n_groups + 1], shared int32 [n_groups]: CUDA tensors (Pages.shared counts the blocks).  For decode steps whose sequences share a lot
        (8 samples of 4096 tokens, 64 of 512, with 8 kv heads of 128); below that, and for prompts, attend is faster."""
        if q.dim() != 4 or q.shape[3] != self.head_dim or (out is not None and out.shape != q.shape):
            raise ValueError("q, out [batch, n_q_heads, tokens, head_dim]")
        for t in (groups, shared):
            if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous() or t.device != self._device:
                raise ValueError("groups and shared are contiguous int32 tensors on the cache's device")
        if groups.numel() != shared.numel() + 1:
            raise ValueError("groups [n_groups + 1], shared [n_groups]")
        if self._elsewhere() or _other_stream(stream):
            with torch.cuda.device(self._device), torch.cuda.stream(stream):   # (memory made here comes from the stream's own)
                return self.attend_shared(q, pages, start, groups, shared, count, scale, out, status)
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
        call = self._call(pages, start, count, (q, out), status)
        Hq, n_groups = q.shape[1], shared.numel()
        n = lib.kvm_cache_shared_workspace(self._ref, call, n_groups, Hq)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n > 0 else None
        rc = lib.kvm_cache_attend_shared(self._ref, call, groups.data_ptr(), shared.data_ptr(), n_groups, q.data_ptr(), Hq, self.head_dim ** -0.5 if scale is None else scale,
                                         out.data_ptr(), _strides3(q), _strides3(out), ws.data_ptr() if n > 0 else None, max(n, 0),
                                         status.data_ptr() if status is not None else None, _stream_ptr(None))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_cache_attend_shared")
        return out

    def copy_pages(self, src, dst, stream=None):
        """kvm_cache_copy_pages: page src[i] to page dst[i]; lists or CPU int32 tensors."""
        src, dst = _page_list(src), _page_list(dst)
        if src.shape != dst.shape:
            raise ValueError("src and dst are lists of the same length")
        if self._elsewhere():
            with torch.cuda.device(self._device):
                return self.copy_pages(src, dst, stream)
        rc = lib.kvm_cache_copy_pages(self._ref, src.data_ptr(), dst.data_ptr(), src.numel(), _stream_ptr(stream))
        if rc != KVM_OK:
            raise KVMError(rc, "kvm_cache_copy_pages")


class Pages:
    """Which page of a pool holds which block of which sequence (kvm_pages_t): host bookkeeping, pages shared by forks until written."""

    def __init__(self, n_pages: int, page_tokens: int = 64):
        self._h = None
        h = C.c_void_p()
        self._do("kvm_pages_create", _int(n_pages, 64), _int(page_tokens), C.byref(h))
        self._h = h
        self.n_pages = n_pages

    def __del__(self):
        if getattr(self, "_h", None) and lib is not None:   # (None: the interpreter is ending, and the memory goes with it)
            lib.kvm_pages_destroy(self._h)
            self._h = None

    def _do(self, fn, *args):
        rc = getattr(lib, fn)(*args)
        if rc != KVM_OK:
            raise KVMError(rc, fn)

    def open(self) -> int:
        seq = C.c_int32()
        self._do("kvm_pages_open", self._h, C.byref(seq))
        return seq.value

    def fork(self, seq: int) -> int:
        child = C.c_int32()
        self._do("kvm_pages_fork", self._h, _int(seq), C.byref(child))
        return child.value

    def close(self, seq: int):
        self._do("kvm_pages_close", self._h, _int(seq))

    def extend(self, seq: int, n_tokens: int):
        """Room for n_tokens more tokens; (src, dst) of the page to copy before the append, or None."""
        src, dst = C.c_int32(), C.c_int32()
        self._do("kvm_pages_extend", self._h, _int(seq), _int(n_tokens, 64), C.byref(src), C.byref(dst))
        return (src.value, dst.value) if src.value >= 0 else None

    def trim(self, seq: int, window: int, sinks: int = 0):
        self._do("kvm_pages_trim", self._h, _int(seq), _int(window), _int(sinks))

    def compact(self):
        """(src, dst): the copies to make before the next call over the cache, as CPU int32 tensors."""
        src, dst = torch.empty(self.n_pages, dtype=torch.int32), torch.empty(self.n_pages, dtype=torch.int32)
        n = C.c_int64()
        self._do("kvm_pages_compact", self._h, src.data_ptr(), dst.data_ptr(), self.n_pages, C.byref(n))
        return src[:n.value].clone(), dst[:n.value].clone()

    def table(self, seq: int):
        seq, n = _int(seq), C.c_int64()
        self._do("kvm_pages_table", self._h, seq, None, 0, C.byref(n), None)
        out = (C.c_int32 * max(1, n.value))()
        self._do("kvm_pages_table", self._h, seq, out, n.value, None, None)
        return list(out[:n.value])

    def length(self, seq: int) -> int:
        n = C.c_int64()
        self._do("kvm_pages_table", self._h, _int(seq), None, 0, None, C.byref(n))
        return n.value

    def shared(self, seqs, n_tokens: int = 1) -> int:
        """The number of leading blocks that the sequences have in common in front of the last n_tokens tokens of each: full ones, on the same pages (what
        Cache.attend_shared takes for a group, in a call of n_tokens tokens)."""
        ids = [_int(s) for s in seqs]
        n = C.c_int32()
        self._do("kvm_pages_shared", self._h, (C.c_int32 * max(1, len(ids)))(*ids), len(ids), _int(n_tokens, 64), C.byref(n))
        return n.value

    def tables(self, seqs, max_pages: int = 0, device="cuda"):
        """pages [len(seqs), max_pages] and lengths [len(seqs)], int32 on `device`: what Cache.append and Cache.attend take."""
        rows = [self.table(s) for s in seqs]
        width = max([max_pages, 1] + [len(r) for r in rows])
        t = torch.full((len(rows), width), -1, dtype=torch.int32)
        for i, r in enumerate(rows):
            t[i, :len(r)] = torch.tensor(r, dtype=torch.int32)
        return t.to(device), torch.tensor([self.length(s) for s in seqs], dtype=torch.int32).to(device)

    def info(self):
        free, high = C.c_int64(), C.c_int64()
        self._do("kvm_pages_info", self._h, C.byref(free), C.byref(high))
        return dict(n_free=free.value, high=high.value)
