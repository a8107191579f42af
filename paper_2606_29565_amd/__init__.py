"""Speculative pre-positioning on one MI355X: thin Python binding of libspp.so.

Every call marshals arguments into the C ABI declared in ``include/spp.h``; all
device work runs in the library's HIP kernels.  PyTorch only provides device
memory (tensors whose data pointers are handed to the library) and streams.
There is no fallback: if ``libspp.so`` is missing or no GPU is present, the calls
raise.
"""
from __future__ import annotations

import ctypes
import dataclasses
import math
import operator
import os
from typing import Dict, List, Optional, Sequence, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libspp.so")

# spp_status
SPP_OK, SPP_SKIPPED_BUDGET, SPP_YIELDED = 0, 1, 2
SPP_E_INVALID_ARG, SPP_E_CAPACITY, SPP_E_HIP, SPP_E_STATE, SPP_E_NOMEM = -1, -2, -3, -4, -5
# spp_gate_outcome
SPP_SERVED, SPP_FALL_INVALID, SPP_FALL_INELIGIBLE, SPP_FALL_GAP, SPP_FALL_NOT_IN_SET, \
    SPP_FALL_NONFINITE = range(6)
OUTCOME_NAMES = ["SERVED", "FALL_INVALID", "FALL_INELIGIBLE", "FALL_GAP", "FALL_NOT_IN_SET",
                 "FALL_NONFINITE"]
# spp_mutation
SPP_MUT_SHIFT, SPP_MUT_ROLLBACK, SPP_MUT_UPDATE = 0, 1, 2
SPP_DTYPE_F32, SPP_DTYPE_BF16 = 0, 1
SPP_W_Q, SPP_W_K, SPP_W_V, SPP_W_O, SPP_W_GATE, SPP_W_UP, SPP_W_DOWN = range(7)
SPP_WFMT_DTYPE, SPP_WFMT_MXFP4 = 0, 1
# largest session capacity in cells per layer (spp.h)
SPP_MAX_CAPACITY = 16777216 - 64


class spp_model_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("ffn_dim", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_base", ctypes.c_double), ("dtype", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("max_sessions", ctypes.c_int32),
                ("weights_packed", ctypes.c_int32), ("weight_format", ctypes.c_int32)]


_PP = ctypes.POINTER(ctypes.c_void_p)


class spp_weights(ctypes.Structure):
    _fields_ = [("embed", ctypes.c_void_p), ("final_norm", ctypes.c_void_p),
                ("lm_head", ctypes.c_void_p), ("lm_bias", ctypes.c_void_p),
                ("attn_norm", _PP), ("wq", _PP), ("wk", _PP), ("wv", _PP), ("wo", _PP),
                ("mlp_norm", _PP), ("w_gate", _PP), ("w_up", _PP), ("w_down", _PP),
                ("scales", _PP * 7)]


class spp_session_config(ctypes.Structure):
    _fields_ = [("capacity", ctypes.c_int32), ("budget", ctypes.c_int32)]


class spp_kv_layout(ctypes.Structure):
    _fields_ = [("k_offset", ctypes.c_int64), ("v_offset", ctypes.c_int64),
                ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
                ("elem_bytes", ctypes.c_int32)]


class spp_ready_t(ctypes.Structure):
    _fields_ = [("session_id", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("epoch", ctypes.c_uint64)]


class spp_summary(ctypes.Structure):
    _fields_ = [("argmax", ctypes.c_int32), ("top1", ctypes.c_float), ("top2", ctypes.c_float),
                ("gap", ctypes.c_float), ("lse", ctypes.c_float), ("position", ctypes.c_int32),
                ("flags", ctypes.c_uint32)]


class spp_session_info(ctypes.Structure):
    _fields_ = [("n_committed", ctypes.c_int32), ("used_cells", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("position", ctypes.c_int32), ("valid", ctypes.c_int32),
                ("decoded", ctypes.c_int32), ("entry_len", ctypes.c_int32),
                ("epoch", ctypes.c_uint64)]


class spp_gate_point(ctypes.Structure):
    _fields_ = [("tau", ctypes.c_float), ("served", ctypes.c_int32), ("wrong", ctypes.c_int32),
                ("coverage", ctypes.c_double), ("coverage_lo", ctypes.c_double),
                ("coverage_hi", ctypes.c_double), ("risk", ctypes.c_double),
                ("risk_lo", ctypes.c_double), ("risk_hi", ctypes.c_double)]


class spp_pool_config(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("page_cells", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("max_seqs", ctypes.c_int32)]


class spp_page_layout(ctypes.Structure):
    _fields_ = [("page_stride", ctypes.c_int64), ("layer_stride", ctypes.c_int64),
                ("v_offset", ctypes.c_int64), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("elem_bytes", ctypes.c_int32)]


class spp_pool_info(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("used_pages", ctypes.c_int32),
                ("shared_pages", ctypes.c_int32), ("n_seqs", ctypes.c_int32),
                ("max_seqs", ctypes.c_int32)]


class spp_seq_info(ctypes.Structure):
    _fields_ = [("n_cells", ctypes.c_int32), ("n_pages", ctypes.c_int32),
                ("decoded", ctypes.c_int32)]


class spp_paged_attn(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("layer", ctypes.c_int32), ("n_seqs", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("table", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("max_pages", ctypes.c_int32),
                ("lengths", ctypes.c_void_p), ("scale", ctypes.c_float), ("out", ctypes.c_void_p),
                ("out_stride", ctypes.c_int64)]


class spp_adjust(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p), ("tokens", ctypes.c_void_p),
                ("bias_tokens", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("allowed", ctypes.c_void_p), ("n_tokens", ctypes.c_int32),
                ("n_prompt", ctypes.c_int32), ("n_bias", ctypes.c_int32),
                ("repetition", ctypes.c_float), ("frequency", ctypes.c_float),
                ("presence", ctypes.c_float), ("fill", ctypes.c_float)]


EXPORTS = ["spp_model_create", "spp_model_destroy", "spp_session_kv_bytes", "spp_session_kv_layout",
           "spp_session_create", "spp_session_destroy", "spp_session_id", "spp_session_restore",
           "spp_kv_append_delta", "spp_preposition", "spp_ready_summary", "spp_gate",
           "spp_invalidate_on_mutation", "spp_session_info", "spp_session_info_get",
           "spp_preposition_batch",
           "spp_gate_batch", "spp_last_error", "spp_profile_preposition", "spp_kernel_class_name",
           "spp_copy_reference", "spp_pack_weight", "spp_pack_weight_mxfp4", "spp_resume",
           "spp_shift", "spp_gate_calibrate", "spp_preposition_idle", "spp_gate_batch_noalloc",
           "spp_profile_preposition_batch", "spp_pool_bytes", "spp_pool_page_layout",
           "spp_pool_create", "spp_pool_destroy", "spp_pool_info", "spp_pool_compact",
           "spp_seq_create", "spp_seq_free", "spp_seq_info", "spp_seq_table", "spp_seq_fork",
           "spp_seq_reserve", "spp_seq_commit", "spp_seq_truncate", "spp_seq_import",
           "spp_seq_export", "spp_seq_summaries", "spp_decode_batch",
           "spp_paged_attention_work_bytes", "spp_paged_attention",
           "spp_adjust_logits_work_bytes", "spp_adjust_logits"]

_lib = None


def lib() -> ctypes.CDLL:
    """The loaded libspp.so (raises if it was not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
    L = ctypes.CDLL(LIB_PATH)
    P, i32, u32, f32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_float, ctypes.c_size_t
    st = ctypes.c_int
    sig = {
        "spp_model_create": (st, [ctypes.POINTER(spp_model_config), ctypes.POINTER(spp_weights), ctypes.POINTER(P)]),
        "spp_model_destroy": (st, [P]),
        "spp_session_kv_bytes": (sz, [P, i32]),
        "spp_session_kv_layout": (st, [P, i32, i32, ctypes.POINTER(spp_kv_layout)]),
        "spp_session_create": (st, [P, ctypes.POINTER(spp_session_config), P, sz, ctypes.POINTER(P)]),
        "spp_session_destroy": (st, [P]),
        "spp_session_id": (i32, [P]),
        "spp_session_restore": (st, [P, i32]),
        "spp_kv_append_delta": (st, [P, P, i32, P]),
        "spp_preposition": (st, [P, P, i32, P, P, P, ctypes.POINTER(spp_ready_t)]),
        "spp_preposition_idle": (st, [P, P, i32, P, P, P, i32, P, ctypes.POINTER(spp_ready_t)]),
        "spp_resume": (st, [P, P, i32, P, P, P, ctypes.POINTER(spp_ready_t)]),
        "spp_ready_summary": (st, [spp_ready_t, ctypes.POINTER(spp_summary)]),
        "spp_gate": (st, [spp_ready_t, f32, P, P, i32, P, ctypes.POINTER(i32), ctypes.POINTER(st),
                          ctypes.POINTER(spp_summary)]),
        "spp_invalidate_on_mutation": (st, [P, st, i32]),
        "spp_shift": (st, [P, i32, P]),
        "spp_gate_calibrate": (st, [i32, P, P, P, ctypes.c_double, ctypes.c_double, i32, P,
                                    ctypes.POINTER(spp_gate_point), i32, ctypes.POINTER(i32),
                                    ctypes.POINTER(f32)]),
        "spp_session_info": (st, [P, ctypes.POINTER(spp_session_info)]),
        "spp_session_info_get": (st, [P, ctypes.POINTER(spp_session_info)]),
        "spp_preposition_batch": (st, [i32, P, P, P, P, P, P, P]),
        "spp_gate_batch": (st, [i32, P, P, P, P, P, P]),
        "spp_gate_batch_noalloc": (st, [i32, P, P, P, P, P, P]),
        "spp_last_error": (ctypes.c_char_p, []),
        "spp_profile_preposition": (i32, [P, P, i32, P, P, i32, P, P]),
        "spp_profile_preposition_batch": (i32, [i32, P, P, P, P, P, P, P, i32, P, P]),
        "spp_kernel_class_name": (ctypes.c_char_p, [i32]),
        "spp_copy_reference": (st, [P, P, sz, P]),
        "spp_pack_weight": (st, [ctypes.POINTER(spp_model_config), i32, P, P, P]),
        "spp_pack_weight_mxfp4": (st, [ctypes.POINTER(spp_model_config), i32, P, P, P, P, P]),
        "spp_pool_bytes": (sz, [ctypes.POINTER(spp_pool_config)]),
        "spp_pool_page_layout": (st, [ctypes.POINTER(spp_pool_config), ctypes.POINTER(spp_page_layout)]),
        "spp_pool_create": (st, [ctypes.POINTER(spp_pool_config), P, sz, ctypes.POINTER(P)]),
        "spp_pool_destroy": (st, [P]),
        "spp_pool_info": (st, [P, ctypes.POINTER(spp_pool_info)]),
        "spp_pool_compact": (st, [P, P, ctypes.POINTER(i32)]),
        "spp_seq_create": (st, [P, i32, ctypes.POINTER(i32)]),
        "spp_seq_free": (st, [P, i32]),
        "spp_seq_info": (st, [P, i32, ctypes.POINTER(spp_seq_info)]),
        "spp_seq_table": (st, [P, i32, P, i32, ctypes.POINTER(i32)]),
        "spp_seq_fork": (st, [P, i32, i32, P]),
        "spp_seq_reserve": (st, [P, i32, P, i32, P]),
        "spp_seq_commit": (st, [P, i32, i32]),
        "spp_seq_truncate": (st, [P, i32, i32]),
        "spp_seq_import": (st, [P, i32, P, P]),
        "spp_seq_export": (st, [P, i32, P, P]),
        "spp_seq_summaries": (st, [P, i32, P, ctypes.POINTER(spp_summary)]),
        "spp_decode_batch": (st, [P, P, i32, P, P, P, P]),
        "spp_paged_attention_work_bytes": (sz, [ctypes.POINTER(spp_paged_attn)]),
        "spp_paged_attention": (st, [ctypes.POINTER(spp_paged_attn), P, sz, P]),
        "spp_adjust_logits_work_bytes": (sz, [i32, i32]),
        "spp_adjust_logits": (st, [i32, i32, ctypes.POINTER(spp_adjust), P, P, sz, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


class SppError(RuntimeError):
    def __init__(self, rc: int, where: str):
        super().__init__(f"{where} -> {rc}: {lib().spp_last_error().decode()}")
        self.rc = rc


class YieldFlag:
    """The host word an idle-window pre-position watches: set() when a request arrives."""

    def __init__(self):
        self._word = ctypes.c_uint32(0)

    @property
    def address(self) -> int:
        return ctypes.addressof(self._word)

    def set(self) -> None:
        self._word.value = 1

    def clear(self) -> None:
        self._word.value = 0

    def is_set(self) -> bool:
        return self._word.value != 0


def _unconverted(name: str):
    """The function as called with ctypes objects of its types (and int32 as int): without the
    conversion of every argument, 0.07 us each, for calls made in numbers."""
    return lib()[name]


def check(rc: int, where: str) -> int:
    if rc < 0:
        raise SppError(rc, where)
    return rc


def _ptr(t) -> int:
    """Device pointer of a tensor (or an int that already is one)."""
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _stream_of(stream, device: int) -> Optional[int]:
    """As _stream, with the current stream of that device for None."""
    if stream is None:
        import torch
        # (the handle without a Stream object around it: 0.1 us instead of 1.0)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return raw(device) if raw else torch.cuda.current_stream(device).cuda_stream
    return _stream(stream)


def _host_i32(tokens) -> Tuple[ctypes.Array, int]:
    vals = [int(t) for t in tokens]
    arr = (ctypes.c_int32 * max(1, len(vals)))(*vals)
    return arr, len(vals)


LAYER_KEYS = ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")
# projection keys in spp_weight_kind order (the MXFP4 scales are listed the same way)
PROJ_KEYS = ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down")


def model_config(n_layers: int, d_model: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                 ffn_dim: int, vocab: int, rope_base: float, bf16: bool, rms_eps: float = 1e-5,
                 max_tokens: int = 128, max_sessions: int = 1,
                 weights_packed: bool = False, mxfp4: bool = False) -> spp_model_config:
    return spp_model_config(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab,
                            rms_eps, rope_base, SPP_DTYPE_BF16 if bf16 else SPP_DTYPE_F32,
                            max_tokens, max_sessions, 1 if weights_packed else 0,
                            SPP_WFMT_MXFP4 if mxfp4 else SPP_WFMT_DTYPE)


def pack_weight_mxfp4(cfg: spp_model_config, which: int, codes_src, scales_src, codes_dst,
                      scales_dst, stream=None) -> None:
    """spp_pack_weight_mxfp4: row-major MXFP4 codes and scales into the tiled layout."""
    check(lib().spp_pack_weight_mxfp4(ctypes.byref(cfg), which, ctypes.c_void_p(_ptr(codes_src)),
                                      ctypes.c_void_p(_ptr(scales_src)),
                                      ctypes.c_void_p(_ptr(codes_dst)),
                                      ctypes.c_void_p(_ptr(scales_dst)),
                                      ctypes.c_void_p(_stream(stream))), "spp_pack_weight_mxfp4")


class Model:
    """A decoder whose weights live in caller-owned device memory.

    weights: dict with "embed", "final_norm", "lm_head", optional "lm_bias" (fp32), and
    per-layer lists under LAYER_KEYS, each entry a tensor or a device pointer.  With
    mxfp4=True the projection lists hold the 4-bit codes and "scales" maps each key of
    PROJ_KEYS to the per-layer e8m0 scales."""

    def __init__(self, n_layers: int, d_model: int, n_q_heads: int, n_kv_heads: int, head_dim: int,
                 ffn_dim: int, vocab: int, rope_base: float, bf16: bool, weights: Dict,
                 rms_eps: float = 1e-5, max_tokens: int = 128, max_sessions: int = 1,
                 weights_packed: bool = False, mxfp4: bool = False):
        self.cfg = model_config(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, ffn_dim, vocab,
                                rope_base, bf16, rms_eps, max_tokens, max_sessions, weights_packed,
                                mxfp4)
        self.vocab = vocab
        self._keep = weights  # the library stores non-owning pointers
        arrays = {}
        for k in LAYER_KEYS:
            ptrs = [_ptr(t) for t in weights[k]]
            if len(ptrs) != n_layers:
                raise ValueError(f"{k}: {len(ptrs)} layers, expected {n_layers}")
            arrays[k] = (ctypes.c_void_p * n_layers)(*ptrs)
        scale_arrays = (_PP * 7)()
        if mxfp4:
            for i, k in enumerate(PROJ_KEYS):
                ptrs = [_ptr(t) for t in weights["scales"][k]]
                if len(ptrs) != n_layers:
                    raise ValueError(f"scales {k}: {len(ptrs)} layers, expected {n_layers}")
                arrays["scales_" + k] = (ctypes.c_void_p * n_layers)(*ptrs)
                scale_arrays[i] = ctypes.cast(arrays["scales_" + k], _PP)
        self._arrays = arrays
        w = spp_weights(_ptr(weights["embed"]), _ptr(weights["final_norm"]),
                        _ptr(weights["lm_head"]), _ptr(weights.get("lm_bias")),
                        *[ctypes.cast(arrays[k], _PP) for k in LAYER_KEYS], scale_arrays)
        h = ctypes.c_void_p()
        check(lib().spp_model_create(ctypes.byref(self.cfg), ctypes.byref(w), ctypes.byref(h)),
              "spp_model_create")
        self.handle = h

    def close(self) -> None:
        if self.handle:
            lib().spp_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def kv_bytes(self, capacity: int) -> int:
        return lib().spp_session_kv_bytes(self.handle, capacity)

    def kv_layout(self, capacity: int, layer: int) -> spp_kv_layout:
        out = spp_kv_layout()
        check(lib().spp_session_kv_layout(self.handle, capacity, layer, ctypes.byref(out)),
              "spp_session_kv_layout")
        return out

    def profile_preposition(self, session: "Session", entry: Sequence[int], dist, stream=None):
        """Per-kernel-class device time (us) and launch counts of one pre-position."""
        n = 32
        times = (ctypes.c_float * n)()
        counts = (ctypes.c_int32 * n)()
        arr, L = _host_i32(entry)
        k = lib().spp_profile_preposition(session.handle, arr, L, ctypes.c_void_p(_ptr(dist)),
                                          ctypes.c_void_p(_stream(stream)), n, times, counts)
        check(k, "spp_profile_preposition")
        return {lib().spp_kernel_class_name(i).decode(): (times[i], counts[i]) for i in range(k)}


@dataclasses.dataclass
class Ready:
    handle: spp_ready_t
    status: int


class Session:
    """A session over a caller-owned KV buffer (a uint8 torch tensor unless given)."""

    def __init__(self, model: Model, capacity: int, budget: int = 0, kv=None, device="cuda"):
        self.model = model
        nbytes = model.kv_bytes(capacity)
        if kv is None:
            import torch
            kv = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.kv = kv
        cfg = spp_session_config(capacity, budget)
        h = ctypes.c_void_p()
        check(lib().spp_session_create(model.handle, ctypes.byref(cfg), ctypes.c_void_p(_ptr(kv)),
                                       nbytes, ctypes.byref(h)), "spp_session_create")
        self.handle = h
        self.capacity = capacity

    def close(self) -> None:
        if self.handle:
            lib().spp_session_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def id(self) -> int:
        return lib().spp_session_id(self.handle)

    def restore(self, n_tokens: int) -> None:
        check(lib().spp_session_restore(self.handle, n_tokens), "spp_session_restore")

    def append_delta(self, tokens: Sequence[int], stream=None) -> int:
        arr, n = _host_i32(tokens)
        return check(lib().spp_kv_append_delta(self.handle, arr, n, ctypes.c_void_p(_stream(stream))),
                     "spp_kv_append_delta")

    def preposition(self, entry: Sequence[int], dist, default_bitmap=None, stream=None) -> Ready:
        arr, L = _host_i32(entry)
        r = spp_ready_t()
        rc = check(lib().spp_preposition(self.handle, arr, L, ctypes.c_void_p(_ptr(dist)),
                                         ctypes.c_void_p(_ptr(default_bitmap)),
                                         ctypes.c_void_p(_stream(stream)), ctypes.byref(r)),
                   "spp_preposition")
        return Ready(r, rc)

    def preposition_idle(self, entry: Sequence[int], dist, flag: "YieldFlag", chunk_layers: int = 1,
                         default_bitmap=None, stream=None) -> Ready:
        """Idle-window pre-position (spp_preposition_idle): blocks until done, or returns
        with status SPP_YIELDED soon after `flag` is set from another thread."""
        arr, L = _host_i32(entry)
        r = spp_ready_t()
        rc = check(lib().spp_preposition_idle(self.handle, arr, L, ctypes.c_void_p(_ptr(dist)),
                                              ctypes.c_void_p(_ptr(default_bitmap)),
                                              ctypes.c_void_p(flag.address), chunk_layers,
                                              ctypes.c_void_p(_stream(stream)), ctypes.byref(r)),
                   "spp_preposition_idle")
        return Ready(r, rc)

    def resume(self, delta: Sequence[int], dist, default_bitmap=None, stream=None) -> Ready:
        """Fall-through resume (spp_resume): keep the entry cells, process the delta only."""
        arr, n = _host_i32(delta)
        r = spp_ready_t()
        rc = check(lib().spp_resume(self.handle, arr, n, ctypes.c_void_p(_ptr(dist)),
                                    ctypes.c_void_p(_ptr(default_bitmap)),
                                    ctypes.c_void_p(_stream(stream)), ctypes.byref(r)),
                   "spp_resume")
        return Ready(r, rc)

    def invalidate(self, kind: int, arg: int = 0) -> None:
        check(lib().spp_invalidate_on_mutation(self.handle, kind, arg), "spp_invalidate_on_mutation")

    def shift(self, delta: int, stream=None) -> None:
        """Sliding-window shift by `delta` cells (spp_shift)."""
        check(lib().spp_shift(self.handle, delta, ctypes.c_void_p(_stream(stream))), "spp_shift")

    def info(self) -> spp_session_info:
        out = spp_session_info()
        check(lib().spp_session_info(self.handle, ctypes.byref(out)), "spp_session_info")
        return out


def ready_summary(ready: Ready) -> spp_summary:
    out = spp_summary()
    check(lib().spp_ready_summary(ready.handle, ctypes.byref(out)), "spp_ready_summary")
    return out


def gate(ready: Ready, tau: float, bitmap=None, realized: Optional[Sequence[int]] = None,
         stream=None) -> Tuple[int, int, spp_summary]:
    """Alg. 2: returns (outcome, token or -1, scan summary)."""
    tok = ctypes.c_int32(-1)
    outc = ctypes.c_int(0)
    summ = spp_summary()
    if realized is None:
        arr, n = None, 0
    else:
        arr, n = _host_i32(realized)
    check(lib().spp_gate(ready.handle, tau, ctypes.c_void_p(_ptr(bitmap)), arr, n,
                         ctypes.c_void_p(_stream(stream)), ctypes.byref(tok), ctypes.byref(outc),
                         ctypes.byref(summ)), "spp_gate")
    return outc.value, tok.value, summ


class GateCall:
    """spp_gate (or, with n > 1 handles, spp_gate_batch) with its arguments marshalled
    once, as a serving loop keeps them: each call() is the C call alone.  outcomes() and
    tokens() read the last call's results."""

    def __init__(self, readies: Sequence[Ready], taus: Sequence[float], bitmaps, stream=None,
                 noalloc: bool = False):
        n = len(readies)
        self.n = n
        self._st = ctypes.c_void_p(_stream(stream))
        if n == 1 and not noalloc:
            self._args = (readies[0].handle, ctypes.c_float(float(taus[0])),
                          ctypes.c_void_p(_ptr(bitmaps[0])), None, 0, self._st)
            self._tok = ctypes.c_int32(-1)
            self._out = ctypes.c_int(0)
            self._fn = lib().spp_gate
            self._tail = (ctypes.byref(self._tok), ctypes.byref(self._out), None)
        else:
            self._rs = (spp_ready_t * n)(*[r.handle for r in readies])
            self._ts = (ctypes.c_float * n)(*[float(t) for t in taus])
            self._bms = (ctypes.c_void_p * n)(*[_ptr(b) for b in bitmaps])
            self._toks = (ctypes.c_int32 * n)()
            self._outs = (ctypes.c_int * n)()
            self._fn = lib().spp_gate_batch_noalloc if noalloc else lib().spp_gate_batch
            self._args = (n, self._rs, self._ts, self._bms, self._st, self._toks, self._outs)
            self._tail = ()

    def __call__(self) -> int:
        rc = self._fn(*self._args, *self._tail)
        if rc < 0:
            raise SppError(rc, "gate")
        return rc

    def outcomes(self) -> List[Tuple[int, int]]:
        if self._tail:
            return [(self._out.value, self._tok.value)]
        return [(self._outs[i], self._toks[i]) for i in range(self.n)]


def _batch_args(sessions, entries, dists):
    n = len(sessions)
    hs = (ctypes.c_void_p * n)(*[s.handle.value for s in sessions])
    arrs = [_host_i32(e)[0] for e in entries]
    eps = (ctypes.c_void_p * n)(*[ctypes.cast(a, ctypes.c_void_p).value for a in arrs])
    lens = (ctypes.c_int32 * n)(*[len(e) for e in entries])
    dps = (ctypes.c_void_p * n)(*[_ptr(d) for d in dists])
    return n, hs, eps, lens, dps, arrs


def preposition_batch(sessions: Sequence[Session], entries: Sequence[Sequence[int]], dists,
                      stream=None) -> List[Ready]:
    n, hs, eps, lens, dps, _keep = _batch_args(sessions, entries, dists)
    readies = (spp_ready_t * n)()
    stats = (ctypes.c_int * n)()
    check(lib().spp_preposition_batch(n, hs, eps, lens, dps, ctypes.c_void_p(_stream(stream)),
                                      readies, stats), "spp_preposition_batch")
    return [Ready(readies[i], stats[i]) for i in range(n)]


def profile_preposition_batch(sessions: Sequence[Session], entries: Sequence[Sequence[int]],
                              dists, stream=None):
    """Per-kernel-class device time (us) and launch counts of one batched pre-position."""
    n, hs, eps, lens, dps, _keep = _batch_args(sessions, entries, dists)
    readies = (spp_ready_t * n)()
    stats = (ctypes.c_int * n)()
    nc = 32
    times = (ctypes.c_float * nc)()
    counts = (ctypes.c_int32 * nc)()
    k = lib().spp_profile_preposition_batch(n, hs, eps, lens, dps, ctypes.c_void_p(_stream(stream)),
                                            readies, stats, nc, times, counts)
    check(k, "spp_profile_preposition_batch")
    return {lib().spp_kernel_class_name(i).decode(): (times[i], counts[i]) for i in range(k)}


def gate_batch(readies: Sequence[Ready], taus: Sequence[float], bitmaps, stream=None,
               noalloc: bool = False):
    """spp_gate_batch (or, with noalloc, spp_gate_batch_noalloc): [(outcome, token)]."""
    n = len(readies)
    rs = (spp_ready_t * n)(*[r.handle for r in readies])
    ts = (ctypes.c_float * n)(*[float(t) for t in taus])
    bms = (ctypes.c_void_p * n)(*[_ptr(b) for b in bitmaps])
    toks = (ctypes.c_int32 * n)()
    outs = (ctypes.c_int * n)()
    name = "spp_gate_batch_noalloc" if noalloc else "spp_gate_batch"
    check(getattr(lib(), name)(n, rs, ts, bms, ctypes.c_void_p(_stream(stream)), toks, outs), name)
    return [(outs[i], toks[i]) for i in range(n)]


_ShortTable = ctypes.c_int32 * 65  # 64 pages and their number


class PagePool:
    """Pages of a paged cache (spp_pool_*): sequences are numbers, the pages a device buffer
    (`pages`: a contiguous tensor of at least the pool's bytes; else allocated here)."""

    def __init__(self, n_layers: int, n_kv_heads: int, head_dim: int, bf16: bool, page_cells: int,
                 n_pages: int, max_seqs: int = 64, pages=None, device="cuda"):
        self.cfg = spp_pool_config(n_layers, n_kv_heads, head_dim,
                                   SPP_DTYPE_BF16 if bf16 else SPP_DTYPE_F32, page_cells, n_pages,
                                   max_seqs)
        self.handle = None
        self._free, self._table = _unconverted("spp_seq_free"), _unconverted("spp_seq_table")
        import torch
        if pages is None:
            nbytes = lib().spp_pool_bytes(ctypes.byref(self.cfg))
            pages = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
        self.pages = pages
        if not pages.is_contiguous() or not pages.is_cuda:
            raise ValueError("pages must be a contiguous device tensor")
        self.device = pages.get_device()
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):  # (the pool is the current device's)
            check(lib().spp_pool_create(ctypes.byref(self.cfg), ctypes.c_void_p(_ptr(pages)),
                                        pages.numel() * pages.element_size(), ctypes.byref(h)),
                  "spp_pool_create")
        self.handle = h

    def close(self) -> None:
        if self.handle:
            lib().spp_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def page_layout(self) -> spp_page_layout:
        out = spp_page_layout()
        check(lib().spp_pool_page_layout(ctypes.byref(self.cfg), ctypes.byref(out)),
              "spp_pool_page_layout")
        return out

    def info(self) -> spp_pool_info:
        out = spp_pool_info()
        check(lib().spp_pool_info(self.handle, ctypes.byref(out)), "spp_pool_info")
        return out

    def create(self, n_cells: int = 0) -> int:
        """A sequence of n_cells cells whose contents the caller has written or will write."""
        q = ctypes.c_int32()
        check(lib().spp_seq_create(self.handle, n_cells, ctypes.byref(q)), "spp_seq_create")
        return q.value

    def free(self, seq: int) -> None:
        rc = self._free(self.handle, operator.index(seq))
        if rc < 0:
            raise SppError(rc, "spp_seq_free")

    def seq_info(self, seq: int) -> spp_seq_info:
        out = spp_seq_info()
        check(lib().spp_seq_info(self.handle, seq, ctypes.byref(out)), "spp_seq_info")
        return out

    def table(self, seq: int) -> List[int]:
        """The sequence's page numbers."""
        t, seq = _ShortTable(), operator.index(seq)
        if self._table(self.handle, seq, t, 64, ctypes.byref(t, 256)) < 0:  # a longer one?
            n = ctypes.c_int32()
            check(self._table(self.handle, seq, None, 0, ctypes.byref(n)), "spp_seq_table")
            t = (ctypes.c_int32 * max(1, n.value))()
            check(self._table(self.handle, seq, t, len(t), ctypes.byref(n)), "spp_seq_table")
            return t[:n.value]
        return t[:t[64]]

    def fork(self, seq: int, n: int = 1) -> List[int]:
        """n sequences that share the pages of `seq` until they are written (spp_seq_fork)."""
        out = (ctypes.c_int32 * max(1, n))()
        check(lib().spp_seq_fork(self.handle, seq, n, out), "spp_seq_fork")
        return out[:n]

    def reserve(self, seqs: Sequence[int], cells: int = 1, stream=None) -> None:
        """Makes the next `cells` cells of the sequences writable (spp_seq_reserve)."""
        arr, n = _host_i32(seqs)
        check(lib().spp_seq_reserve(self.handle, n, arr, cells,
                                    ctypes.c_void_p(_stream_of(stream, self.device))), "spp_seq_reserve")

    def commit(self, seq: int, cells: int) -> None:
        check(lib().spp_seq_commit(self.handle, seq, cells), "spp_seq_commit")

    def truncate(self, seq: int, n: int) -> None:
        check(lib().spp_seq_truncate(self.handle, seq, n), "spp_seq_truncate")

    def import_session(self, seq: int, session: Session, stream=None) -> None:
        """The sequence becomes a copy of the session's committed cells (spp_seq_import)."""
        check(lib().spp_seq_import(self.handle, seq, session.handle,
                                   ctypes.c_void_p(_stream_of(stream, self.device))), "spp_seq_import")

    def export_session(self, seq: int, session: Session, stream=None) -> None:
        """The session's committed state becomes a copy of the sequence (spp_seq_export)."""
        check(lib().spp_seq_export(self.handle, seq, session.handle,
                                   ctypes.c_void_p(_stream_of(stream, self.device))), "spp_seq_export")

    def compact(self, stream=None) -> int:
        """Moves the used pages to the buffer's start (spp_pool_compact); how many moved."""
        n = ctypes.c_int32()
        check(lib().spp_pool_compact(self.handle, ctypes.c_void_p(_stream_of(stream, self.device)),
                                     ctypes.byref(n)), "spp_pool_compact")
        return n.value

    def summaries(self, seqs: Sequence[int]) -> List[spp_summary]:
        """The reductions over the logits of the sequences' last decode step."""
        arr, n = _host_i32(seqs)
        out = (spp_summary * max(1, n))()
        check(lib().spp_seq_summaries(self.handle, n, arr, out), "spp_seq_summaries")
        return list(out[:n])


def decode_batch(pool: PagePool, model: Model, seqs: Sequence[int], tokens: Sequence[int], dists,
                 stream=None) -> None:
    """One decode step: tokens[i] appended to seqs[i], its logits to dists[i] (spp_decode_batch):
    contiguous fp32 tensors of at least the vocabulary on the pool's device, or their pointers."""
    arr, n = _host_i32(seqs)
    toks, nt = _host_i32(tokens)
    if nt != n or len(dists) != n:
        raise ValueError("sequences, tokens and dists differ in number")
    import torch
    for i, d in enumerate(dists):
        if isinstance(d, torch.Tensor) and (d.dtype != torch.float32 or not d.is_contiguous() or
                                            d.numel() < model.vocab or d.get_device() != pool.device):
            raise ValueError(f"dist {i} is a contiguous float32 tensor of at least {model.vocab} "
                             f"elements on the pool's device")
    ptrs = (ctypes.c_void_p * max(1, n))(*[_ptr(d) for d in dists])
    check(lib().spp_decode_batch(pool.handle, model.handle, n, arr, toks, ptrs,
                                 ctypes.c_void_p(_stream_of(stream, pool.device))), "spp_decode_batch")


def _row_stride(t, what: str) -> int:
    """Elements between the rows of a [n][heads][head_dim] tensor whose rows are contiguous."""
    if t.dim() != 3 or t.stride(2) != 1 or t.stride(1) != t.shape[2]:
        raise ValueError(f"{what}: [n][heads][head_dim] with contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


class PagedAttention:
    """spp_paged_attention over fixed tables: table [n][max_pages] and lengths [n] are int32
    device tensors (their values may change between calls), the workspace is held here: one
    call at a time, and the object lives until its calls have finished.  Each call(q, out) is
    attention of one new token per sequence, rows of [n_q_heads][head_dim]."""

    def __init__(self, pool: PagePool, layer: int, n_q_heads: int, table, lengths,
                 io_bf16: bool = True, scale: float = 0.0):
        import torch
        self._dev = dev = pool.device
        if not pool.handle:
            raise ValueError("the pool is closed")
        if table.get_device() != dev or lengths.get_device() != dev:
            raise ValueError("table and lengths are on the pool's device")
        if table.dtype != torch.int32 or lengths.dtype != torch.int32 or table.dim() != 2 or \
                lengths.shape != table.shape[:1] or not lengths.is_contiguous() or \
                (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("table [n][max_pages] and lengths [n]: int32, contiguous rows")
        n, width = table.shape
        self._keep = (pool, table, lengths)
        self._dtype = torch.bfloat16 if io_bf16 else torch.float32
        self._shape = torch.Size((n, n_q_heads, pool.cfg.head_dim))
        self._row = row = n_q_heads * pool.cfg.head_dim
        dummy = pool.pages.data_ptr()
        self._a = spp_paged_attn(pool.handle.value, layer, n, n_q_heads,
                                 SPP_DTYPE_BF16 if io_bf16 else SPP_DTYPE_F32, dummy, row,
                                 table.data_ptr(), table.stride(0) if n > 1 else width, width,
                                 lengths.data_ptr(), scale, dummy, row)
        nbytes = lib().spp_paged_attention_work_bytes(ctypes.byref(self._a))
        self._work = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=table.device)
        self._call = _unconverted("spp_paged_attention")
        self._args = (ctypes.byref(self._a), ctypes.c_void_p(self._work.data_ptr()),
                      ctypes.c_size_t(self._work.numel()))

    def __call__(self, q, out, stream=None):
        if q.dtype != self._dtype or out.dtype != self._dtype or q.shape != self._shape or \
                out.shape != self._shape:
            raise ValueError(f"q and out: {self._dtype} of shape {tuple(self._shape)}")
        if q.get_device() != self._dev or out.get_device() != self._dev or not self._keep[0].handle:
            raise ValueError("q and out are on the pool's device, the pool is open")
        a = self._a
        a.q, a.q_stride = q.data_ptr(), self._row if q.is_contiguous() else _row_stride(q, "q")
        a.out, a.out_stride = out.data_ptr(), self._row if out.is_contiguous() else _row_stride(out, "out")
        rc = self._call(*self._args, ctypes.c_void_p(_stream_of(stream, self._dev)))
        if rc < 0:
            raise SppError(rc, "spp_paged_attention")
        return out


@dataclasses.dataclass
class AdjustRow:
    """One row of adjusted logits (spp_adjust): src and dst fp32 device tensors of the
    vocabulary, tokens / bias_tokens int32, bias fp32, allowed a bitmap of int32 words.  Entries
    of tokens outside the vocabulary are skipped."""
    src: object
    dst: object
    tokens: object = None
    n_tokens: Optional[int] = None  # default: all of tokens
    n_prompt: int = 0
    repetition: float = 1.0
    frequency: float = 0.0
    presence: float = 0.0
    bias_tokens: object = None
    bias: object = None
    allowed: object = None
    fill: float = -math.inf


class AdjustSummaries:
    """The reductions of adjusted rows, device tensors [n]."""

    def __init__(self, words):
        import torch
        f = words.view(torch.float32)
        self.argmax, self.flags = words[:, 0], words[:, 6]
        self.top1, self.top2, self.gap, self.lse = f[:, 1], f[:, 2], f[:, 3], f[:, 4]


def _vector(t, dtype, least: int, dev: int, row: int, what: str) -> Optional[int]:
    """The pointer of a contiguous tensor of at least `least` elements on device dev (None: none)."""
    if t is None:
        return None
    if t.dtype != dtype or not t.is_contiguous() or t.numel() < least or t.get_device() != dev or dev < 0:
        raise ValueError(f"row {row}: {what} is a contiguous {dtype} tensor of at least {least} "
                         f"elements on the device of the first row")
    return t.data_ptr()


class LogitsAdjust:
    """spp_adjust_logits with its rows marshalled once: each call() adjusts them and returns
    their AdjustSummaries (None with summaries=False), which the next call overwrites.  The
    workspace is held here: one call at a time, and the object lives until its calls have
    finished.

    A decode keeps one object over its steps: the rows' tensors are fixed, what they hold is read
    at each call.  A history that grows is a tensor with room for it, -1 behind its tokens; an
    object made anew takes the host some 10 us a row."""

    def __init__(self, vocab: int, rows: Sequence[AdjustRow], summaries: bool = True):
        import torch
        n = len(rows)
        self.n, self._keep, self._current_device = n, list(rows), torch.cuda.current_device
        if any(r.src is None or r.dst is None for r in rows):
            raise ValueError("a row has a src and a dst")
        self._dev = dev = rows[0].src.get_device() if n else -1
        words = (vocab + 31) // 32
        self._rows = (spp_adjust * max(1, n))()
        for i, r in enumerate(rows):
            nt = (0 if r.tokens is None else r.tokens.numel()) if r.n_tokens is None else r.n_tokens
            if nt and r.tokens is None:
                raise ValueError(f"row {i}: n_tokens without tokens")
            nb = 0 if r.bias_tokens is None else r.bias_tokens.numel()
            if nb != (0 if r.bias is None else r.bias.numel()):
                raise ValueError(f"row {i}: bias and bias_tokens differ in length")
            self._rows[i] = spp_adjust(
                _vector(r.src, torch.float32, vocab, dev, i, "src"),
                _vector(r.dst, torch.float32, vocab, dev, i, "dst"),
                _vector(r.tokens, torch.int32, nt, dev, i, "tokens"),
                _vector(r.bias_tokens, torch.int32, nb, dev, i, "bias_tokens"),
                _vector(r.bias, torch.float32, nb, dev, i, "bias"),
                _vector(r.allowed, torch.int32, words, dev, i, "allowed"), nt, r.n_prompt, nb,
                r.repetition, r.frequency, r.presence, r.fill)
        self._out, self._summ, nbytes = None, None, 0
        if summaries and n:
            self._out = torch.empty(n, 7, dtype=torch.int32, device=rows[0].src.device)
            self._summ = AdjustSummaries(self._out)
            nbytes = lib().spp_adjust_logits_work_bytes(n, vocab)
            self._work = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=self._out.device)
        self._args = (n, vocab, self._rows, ctypes.c_void_p(_ptr(self._out)),
                      ctypes.c_void_p(_ptr(self._work) if nbytes else 0), ctypes.c_size_t(nbytes))
        self._call = _unconverted("spp_adjust_logits")

    def __call__(self, stream=None):
        if not self.n:
            return None
        if self._current_device() != self._dev:
            raise ValueError(f"the rows are on device {self._dev}, which is not the current one")
        rc = self._call(*self._args, ctypes.c_void_p(_stream_of(stream, self._dev)))
        if rc < 0:
            raise SppError(rc, "spp_adjust_logits")
        return self._summ


def pack_weight(cfg: spp_model_config, which: int, src, dst, stream=None) -> None:
    """Row-major projection weight `which` (SPP_W_*) of a model with configuration cfg ->
    the tiled layout spp_model_create expects with weights_packed (spp_pack_weight)."""
    check(lib().spp_pack_weight(ctypes.byref(cfg), which, ctypes.c_void_p(_ptr(src)),
                                ctypes.c_void_p(_ptr(dst)), ctypes.c_void_p(_stream(stream))),
          "spp_pack_weight")


def copy_reference(dst, src, nbytes: int, stream=None) -> None:
    check(lib().spp_copy_reference(ctypes.c_void_p(_ptr(dst)), ctypes.c_void_p(_ptr(src)), nbytes,
                                   ctypes.c_void_p(_stream(stream))), "spp_copy_reference")


def gate_calibrate(gaps, in_set, correct, r_max: float, taus=None, z: float = 1.959964):
    """spp_gate_calibrate: (tau_star, [spp_gate_point]) for the decision points' gaps,
    set membership and correctness (host arrays); tau_star is inf when no threshold keeps
    the risk within r_max."""
    import numpy as np
    g = np.ascontiguousarray(gaps, dtype=np.float32)
    a = np.ascontiguousarray(in_set, dtype=np.uint8)
    c = np.ascontiguousarray(correct, dtype=np.uint8)
    n = len(g)
    if len(a) != n or len(c) != n:
        raise ValueError("gaps, in_set and correct differ in length")
    t = None if taus is None else np.ascontiguousarray(taus, dtype=np.float32)
    cap = (len(t) if t is not None else n + 1)
    pts = (spp_gate_point * max(cap, 1))()
    npts, tau_star = ctypes.c_int32(), ctypes.c_float()
    check(lib().spp_gate_calibrate(n, ctypes.c_void_p(g.ctypes.data), ctypes.c_void_p(a.ctypes.data),
                                   ctypes.c_void_p(c.ctypes.data), float(r_max), float(z),
                                   0 if t is None else len(t),
                                   None if t is None else ctypes.c_void_p(t.ctypes.data), pts, cap,
                                   ctypes.byref(npts), ctypes.byref(tau_star)),
          "spp_gate_calibrate")
    return float(tau_star.value), [pts[i] for i in range(npts.value)]
