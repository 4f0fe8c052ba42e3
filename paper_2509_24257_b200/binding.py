"""Thin ctypes binding over the C ABI of libverillm.so (include/verillm.h).

Argument marshalling only: torch supplies device memory and the stream, every step of the path
runs in the library's kernels.  There is no CPU fallback: a missing library raises on first use.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libverillm.so")

NSTAT = 16
STAT_NAMES = (
    "rel_l2", "max_abs", "mae", "mean_signed", "p_e", "p_m", "p_w", "q_small", "z_large",
    "n_exp_mismatch", "n_mant_large", "n_mant_small", "n_exact", "n_nonfinite", "l2_delta", "l2_ref",
)
BF16, F32 = 0, 1
TOL_BIT_AWARE = 1
E_INVAL, E_SHAPE, E_RANGE, E_NOMEM, E_CUDA, E_ARCH = -1, -2, -3, -4, -5, -6
DEV_TOKEN_RANGE, DEV_WAIT_TIMEOUT, DEV_PAGE_RANGE, DEV_ROWS_RANGE, DEV_LOGITS, DEV_NO_PAGES = 1, 2, 3, 4, 5, 6
KV_BF16, KV_E4M3, KV_INT8 = 0, 1, 2

EXPORTS = (
    "verillm_default_tol", "verillm_load_weights", "verillm_load_layer", "verillm_load_globals",
    "verillm_verify_prefill", "verillm_decode_commit", "verillm_compare", "verillm_compare_noalloc", "verillm_op_gemm",
    "verillm_op_rmsnorm", "verillm_op_attention", "verillm_free", "verillm_strerror",
    "verillm_last_launch_count", "verillm_profile_enable", "verillm_profile_read",
    "verillm_load_lm_head", "verillm_token_match", "verillm_verify_segment", "verillm_spot_check", "verillm_merkle_roots",
    "verillm_threshold_sweep", "verillm_selftest_wait_timeout", "verillm_kv_write", "verillm_kv_read",
    "verillm_op_attention_paged", "verillm_op_attention_paged_workspace", "verillm_decode_commit_paged",
    "verillm_quantise_w4", "verillm_decode_commit_w4", "verillm_w4_quantise", "verillm_w4_dequantise", "verillm_op_w4_matvec", "verillm_verify_drafts", "verillm_verify_drafts_workspace",
    "verillm_kv_pages_workspace", "verillm_kv_reserve", "verillm_kv_free", "verillm_kv_fork", "verillm_kv_compact", "verillm_kv_copy",
)
PROF_CLASSES = ("setup", "rmsnorm", "gemm_qkv_rope", "attention", "gemm_o_resid", "gemm_gate_up_swiglu",
                "gemm_down_resid_compare", "verdict")


class VerillmError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: error {code} ({strerror(code)})")
        self.code = code


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim", "d_ffn", "vocab")] + [
        ("rope_base", C.c_float), ("rms_eps", C.c_float),
        ("max_tokens", C.c_int32), ("max_checks", C.c_int32), ("max_batch", C.c_int32),
    ]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")]


class Weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("final_norm", C.c_void_p), ("layers", C.POINTER(LayerWeights)), ("on_device", C.c_int32)]


class Tol(C.Structure):
    _fields_ = [
        ("rel_l2", C.c_float), ("max_abs", C.c_float), ("mae", C.c_float),
        ("pe_max", C.c_float), ("pm_min", C.c_float), ("pw_min", C.c_float), ("e_abs_max", C.c_float),
        ("e_w", C.c_float), ("e_m", C.c_int32),
        ("tau_large", C.c_float), ("z_large_max", C.c_float), ("q_small_min", C.c_float),
        ("flags", C.c_uint32),
    ]


class ReportC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("stats", "pos_ok", "first_bad_layer", "seq_ok", "seq_score", "hidden_out", "status")]


class KVCacheC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "k_scale", "v_scale")] + [
        (n, C.c_int32) for n in ("n_pages", "page_size", "n_kv_heads", "head_dim", "dtype")]


class KVRowsC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("page_table", "cu_rows", "kv_len")] + [
        (n, C.c_int32) for n in ("table_width", "batch", "n_rows", "max_rows")]


class W4C(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("codes", "scales")] + [(n, C.c_int32) for n in ("n", "k", "group")]


class DraftsC(C.Structure):
    _fields_ = [("target", C.c_void_p), ("draft", C.c_void_p), ("target_stride", C.c_int64), ("draft_stride", C.c_int64)] + [
        (n, C.c_int32) for n in ("dtype", "vocab", "batch", "n_rows", "max_rows")] + [
        (n, C.c_void_p) for n in ("cu_rows", "tokens", "kv_len", "temperature", "accept_u", "sample_u")]


class DraftReportC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("tokens", "n_emitted", "logp", "new_len")]


class KVPagesC(C.Structure):
    _fields_ = [("layers", C.POINTER(KVCacheC)), ("n_layers", C.c_int32), ("page_table", C.c_void_p), ("kv_len", C.c_void_p),
                ("refs", C.c_void_p), ("batch", C.c_int32), ("table_width", C.c_int32)]


_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    """Loads libverillm.so (built in-tree by paper_2509_24257_b200.build); raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2509_24257_b200.build` "
                "(there is no fallback implementation)"
            )
        L = C.CDLL(LIB_PATH)
        L.verillm_strerror.restype = C.c_char_p
        L.verillm_strerror.argtypes = [C.c_int]
        L.verillm_default_tol.restype = None
        L.verillm_default_tol.argtypes = [C.POINTER(Tol)]
        L.verillm_free.restype = None
        L.verillm_free.argtypes = [C.c_void_p]
        L.verillm_last_launch_count.restype = C.c_int32
        L.verillm_last_launch_count.argtypes = [C.c_void_p]
        L.verillm_load_weights.argtypes = [C.POINTER(Config), C.POINTER(Weights), C.POINTER(C.c_void_p)]
        L.verillm_load_layer.argtypes = [C.c_void_p, C.c_int32, C.POINTER(LayerWeights), C.c_int32]
        L.verillm_load_globals.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32]
        L.verillm_verify_prefill.argtypes = [
            C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32,
            C.POINTER(Tol), C.POINTER(ReportC), C.c_void_p,
        ]
        L.verillm_decode_commit.argtypes = [
            C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
            C.c_int32, C.c_void_p, C.c_void_p,
        ]
        L.verillm_compare.argtypes = [
            C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int32,
            C.POINTER(Tol), C.POINTER(ReportC), C.c_void_p,
        ]
        L.verillm_compare_noalloc.argtypes = L.verillm_compare.argtypes
        L.verillm_compare_noalloc.restype = C.c_int
        L.verillm_verify_segment.argtypes = [
            C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32,
            C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(Tol), C.POINTER(ReportC), C.c_void_p,
        ]
        L.verillm_verify_segment.restype = C.c_int
        L.verillm_spot_check.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                         C.c_float, C.c_float, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.verillm_spot_check.restype = C.c_int
        L.verillm_merkle_roots.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.verillm_merkle_roots.restype = C.c_int
        L.verillm_threshold_sweep.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(Tol), C.c_int32, C.c_void_p, C.c_void_p]
        L.verillm_threshold_sweep.restype = C.c_int
        L.verillm_selftest_wait_timeout.argtypes = [C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]
        L.verillm_selftest_wait_timeout.restype = C.c_int
        L.verillm_load_lm_head.argtypes = [C.c_void_p, C.c_void_p, C.c_int32]
        L.verillm_load_lm_head.restype = C.c_int
        L.verillm_token_match.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.verillm_token_match.restype = C.c_int
        L.verillm_op_gemm.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.verillm_op_rmsnorm.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_float, C.c_void_p]
        L.verillm_op_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.verillm_decode_commit_paged.argtypes = L.verillm_decode_commit.argtypes[:10] + [C.c_int32, C.c_void_p, C.c_void_p]
        L.verillm_decode_commit_paged.restype = C.c_int
        L.verillm_decode_commit_w4.argtypes = L.verillm_decode_commit_paged.argtypes
        L.verillm_quantise_w4.argtypes = [C.c_void_p, C.c_int32, C.c_void_p]
        L.verillm_decode_commit_w4.restype = L.verillm_quantise_w4.restype = C.c_int
        cache_p, rows_p = C.POINTER(KVCacheC), C.POINTER(KVRowsC)
        L.verillm_kv_write.argtypes = [cache_p, rows_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.verillm_kv_write.restype = C.c_int
        L.verillm_kv_read.argtypes = [cache_p, rows_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
        L.verillm_kv_read.restype = C.c_int
        L.verillm_op_attention_paged_workspace.argtypes = [cache_p, rows_p, C.c_int32]
        L.verillm_op_attention_paged_workspace.restype = C.c_int64
        L.verillm_op_attention_paged.argtypes = [cache_p, rows_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p,
                                                 C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.verillm_op_attention_paged.restype = C.c_int
        w4_p, pages_p = C.POINTER(W4C), C.POINTER(KVPagesC)
        L.verillm_w4_quantise.argtypes = [C.c_void_p, C.c_int64, w4_p, C.c_void_p]
        L.verillm_w4_dequantise.argtypes = [w4_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p]
        L.verillm_op_w4_matvec.argtypes = [w4_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32,
                                           C.c_void_p, C.c_void_p]
        L.verillm_verify_drafts.argtypes = [C.POINTER(DraftsC), C.POINTER(DraftReportC), C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.verillm_verify_drafts_workspace.argtypes = [C.c_int32]
        L.verillm_verify_drafts_workspace.restype = C.c_int64
        L.verillm_kv_pages_workspace.argtypes = [C.c_int32, C.c_int32]
        L.verillm_kv_pages_workspace.restype = C.c_int64
        L.verillm_kv_reserve.argtypes = [pages_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.verillm_kv_free.argtypes = [pages_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.verillm_kv_fork.argtypes = [pages_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.verillm_kv_compact.argtypes = [pages_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p]
        L.verillm_kv_copy.argtypes = [cache_p, cache_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        for name in ("w4_quantise", "w4_dequantise", "op_w4_matvec", "verify_drafts", "kv_reserve", "kv_free", "kv_fork", "kv_compact", "kv_copy"):
            getattr(L, "verillm_" + name).restype = C.c_int
        L.verillm_profile_enable.argtypes = [C.c_void_p, C.c_int32]
        L.verillm_profile_read.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_int32)]
        L.verillm_profile_enable.restype = C.c_int
        L.verillm_profile_read.restype = C.c_int
        for name in ("verillm_load_weights", "verillm_load_layer", "verillm_load_globals", "verillm_verify_prefill",
                     "verillm_decode_commit", "verillm_compare", "verillm_compare_noalloc", "verillm_op_gemm", "verillm_op_rmsnorm",
                     "verillm_op_attention"):
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def strerror(code: int) -> str:
    return lib().verillm_strerror(code).decode()


def _check(code: int, what: str) -> None:
    if code != 0:
        raise VerillmError(code, what)


def default_tol(**overrides) -> Tol:
    t = Tol()
    lib().verillm_default_tol(C.byref(t))
    for k, v in overrides.items():
        if k == "bit_aware":
            t.flags = (t.flags | TOL_BIT_AWARE) if v else (t.flags & ~TOL_BIT_AWARE)
        else:
            setattr(t, k, v)
    return t


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    return (stream or torch.cuda.current_stream()).cuda_stream


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


class Report:
    """Device tensors of one verification report; `.cpu()` copies them into numpy arrays."""

    def __init__(self, n_check: int, n_layers: int, batch: int, d_model: int, device, want_hidden: bool):
        nc = max(n_check, 1)
        self.n_check, self.n_layers, self.batch = n_check, n_layers, batch
        self.stats = torch.zeros(nc, n_layers, NSTAT, dtype=torch.float32, device=device)
        self.pos_ok = torch.zeros(nc, dtype=torch.uint8, device=device)
        self.first_bad_layer = torch.zeros(nc, dtype=torch.int32, device=device)
        self.seq_ok = torch.zeros(batch, dtype=torch.uint8, device=device)
        self.seq_score = torch.zeros(batch, dtype=torch.float32, device=device)
        self.hidden = torch.zeros(n_layers, nc, d_model, dtype=torch.float32, device=device) if want_hidden else None
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def c_struct(self) -> ReportC:
        return ReportC(_ptr(self.stats), _ptr(self.pos_ok), _ptr(self.first_bad_layer), _ptr(self.seq_ok),
                       _ptr(self.seq_score), _ptr(self.hidden), _ptr(self.status))

    def cpu(self) -> Dict[str, np.ndarray]:
        n = self.n_check
        out = {
            "stats": self.stats[:n].cpu().numpy(), "pos_ok": self.pos_ok[:n].cpu().numpy(),
            "first_bad_layer": self.first_bad_layer[:n].cpu().numpy(), "seq_ok": self.seq_ok.cpu().numpy(),
            "seq_score": self.seq_score.cpu().numpy(), "status": int(self.status.item()),
        }
        if self.hidden is not None:
            out["hidden"] = self.hidden[:, :n].cpu().numpy()
        return out


_LAYER_KEYS = ("attn_norm", "wq", "wk", "wv", "wo", "ffn_norm", "w_gate", "w_up", "w_down")


def _layer_struct(lw: Dict[str, torch.Tensor]) -> LayerWeights:
    for k in _LAYER_KEYS:
        t = lw[k]
        if t.dtype != torch.bfloat16 or not t.is_contiguous():
            raise ValueError(f"layer tensor {k} must be contiguous bf16")
    return LayerWeights(*[lw[k].data_ptr() for k in _LAYER_KEYS])


class Model:
    """Handle on the library's copy of a model (verillm_load_weights / verillm_free)."""

    def __init__(self, shape, max_tokens: int, max_checks: int, max_batch: int, device: str | torch.device = "cuda:0"):
        self.shape = shape
        self.device = torch.device(device)
        self.cfg = Config(shape.n_layers, shape.d_model, shape.n_heads, shape.n_kv_heads, shape.head_dim, shape.d_ffn,
                          shape.vocab, float(shape.rope_base), float(shape.rms_eps), max_tokens, max_checks, max_batch)
        self._h = C.c_void_p()
        with torch.cuda.device(self.device):
            _check(lib().verillm_load_weights(C.byref(self.cfg), None, C.byref(self._h)), "verillm_load_weights")

    @classmethod
    def from_weights(cls, shape, weights: Dict[str, object], max_tokens: int, max_checks: int, max_batch: int,
                     device: str | torch.device = "cuda:0") -> "Model":
        m = cls(shape, max_tokens, max_checks, max_batch, device)
        m.load_globals(weights["embed"], weights["final_norm"])
        for l, lw in enumerate(weights["layers"]):
            m.load_layer(l, lw)
        return m

    def load_globals(self, embed: torch.Tensor, final_norm: torch.Tensor) -> None:
        on_dev = int(embed.is_cuda)
        with torch.cuda.device(self.device):
            _check(lib().verillm_load_globals(self._h, embed.data_ptr(), final_norm.data_ptr(), on_dev), "verillm_load_globals")

    def load_layer(self, layer: int, lw: Dict[str, torch.Tensor]) -> None:
        on_dev = int(lw["wq"].is_cuda)
        st = _layer_struct(lw)
        with torch.cuda.device(self.device):
            _check(lib().verillm_load_layer(self._h, layer, C.byref(st), on_dev), "verillm_load_layer")

    def verify_prefill(self, tokens: torch.Tensor, cu_seqlens: Sequence[int], committed: Optional[torch.Tensor],
                       check_seq: Sequence[int], check_pos: Sequence[int], tol: Optional[Tol] = None,
                       want_hidden: bool = False, report: Optional[Report] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> Report:
        """tokens: int32 device [n_tokens]; committed: device [n_layers][n_check][d_model] bf16 or f32."""
        cu = _i32(cu_seqlens)
        cs, cp = _i32(check_seq), _i32(check_pos)
        n_check, batch = int(cs.shape[0]), int(cu.shape[0]) - 1
        tol = tol or default_tol()
        if report is None:
            report = Report(n_check, self.shape.n_layers, batch, self.shape.d_model, self.device, want_hidden)
        dtype = BF16
        if committed is not None:
            if committed.dtype == torch.float32:
                dtype = F32
            elif committed.dtype != torch.bfloat16:
                raise ValueError("committed states must be bf16 or float32")
            if not committed.is_contiguous():
                raise ValueError("committed states must be contiguous")
        if tokens.dtype != torch.int32 or not tokens.is_cuda:
            raise ValueError("tokens must be an int32 CUDA tensor")
        rc_struct = report.c_struct()
        with torch.cuda.device(self.device):
            code = lib().verillm_verify_prefill(
                self._h, tokens.data_ptr(), cu.ctypes.data, batch, _ptr(committed), dtype, cs.ctypes.data, cp.ctypes.data,
                n_check, C.byref(tol), C.byref(rc_struct), _stream_ptr(stream))
        _check(code, "verillm_verify_prefill")
        return report

    def verify_segment(self, input_states: torch.Tensor, layer_begin: int, layer_end: int, cu_seqlens: Sequence[int],
                       committed: Optional[torch.Tensor], check_seq: Sequence[int], check_pos: Sequence[int],
                       tol: Optional[Tol] = None, want_hidden: bool = False,
                       stream: Optional[torch.cuda.Stream] = None) -> Report:
        """input_states: device [n_tokens][d_model] bf16/f32; committed: device [layer_end-layer_begin][n_check][d_model]."""
        cu = _i32(cu_seqlens)
        cs, cp = _i32(check_seq), _i32(check_pos)
        n_check, batch = int(cs.shape[0]), int(cu.shape[0]) - 1
        tol = tol or default_tol()
        report = Report(n_check, layer_end - layer_begin, batch, self.shape.d_model, self.device, want_hidden)
        if not input_states.is_contiguous() or input_states.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError("input states must be contiguous bf16 or float32")
        cdt = BF16 if committed is None or committed.dtype == torch.bfloat16 else F32
        st = report.c_struct()
        with torch.cuda.device(self.device):
            code = lib().verillm_verify_segment(
                self._h, input_states.data_ptr(), BF16 if input_states.dtype == torch.bfloat16 else F32, layer_begin,
                layer_end, cu.ctypes.data, batch, _ptr(committed), cdt, cs.ctypes.data, cp.ctypes.data, n_check,
                C.byref(tol), C.byref(st), _stream_ptr(stream))
        _check(code, "verillm_verify_segment")
        return report

    def decode_commit(self, tokens: torch.Tensor, cu_seqlens: Sequence[int], n_prefill: int, check_seq: Sequence[int],
                      check_pos: Sequence[int], commit_dtype: torch.dtype = torch.bfloat16,
                      stream: Optional[torch.cuda.Stream] = None, cache_dtype: Optional[torch.dtype] = None, w4: bool = False) -> torch.Tensor:
        """cache_dtype: bf16, float8_e4m3fn or int8 decodes over a paged cache of that type; None over the contiguous bf16 one.  w4: on the
        4-bit weights that `quantise_w4` made."""
        cu = _i32(cu_seqlens)
        cs, cp = _i32(check_seq), _i32(check_pos)
        n_check, batch = int(cs.shape[0]), int(cu.shape[0]) - 1
        if cache_dtype is not None and cache_dtype not in _KV_DTYPES:
            raise ValueError("cache_dtype must be bf16, float8_e4m3fn or int8")
        out = torch.zeros(self.shape.n_layers, max(n_check, 1), self.shape.d_model, dtype=commit_dtype, device=self.device)
        status = torch.zeros(1, dtype=torch.int32, device=self.device)
        args = [self._h, tokens.data_ptr(), cu.ctypes.data, batch, int(n_prefill), cs.ctypes.data, cp.ctypes.data, n_check,
                out.data_ptr(), BF16 if commit_dtype == torch.bfloat16 else F32]
        name = "verillm_decode_commit_w4" if w4 else "verillm_decode_commit" if cache_dtype is None else "verillm_decode_commit_paged"
        if cache_dtype is not None or w4:
            args.append(-1 if cache_dtype is None else _KV_DTYPES[cache_dtype])
        with torch.cuda.device(self.device):
            code = getattr(lib(), name)(*args, status.data_ptr(), _stream_ptr(stream))
        _check(code, name)
        if int(status.item()) != 0:
            raise RuntimeError(f"{name}: device status {int(status.item())}")
        return out[:, :n_check]

    def quantise_w4(self, group: int = 128, stream: Optional[torch.cuda.Stream] = None) -> None:
        """Makes 4-bit copies of the projections, one scale per `group` inputs, for decode_commit(w4=True)."""
        with torch.cuda.device(self.device):
            _check(lib().verillm_quantise_w4(self._h, int(group), _stream_ptr(stream)), "verillm_quantise_w4")

    def load_lm_head(self, lm_head: torch.Tensor) -> None:
        if lm_head.dtype != torch.bfloat16 or not lm_head.is_contiguous():
            raise ValueError("the output head must be contiguous bf16")
        with torch.cuda.device(self.device):
            _check(lib().verillm_load_lm_head(self._h, lm_head.data_ptr(), int(lm_head.is_cuda)), "verillm_load_lm_head")

    def token_match(self, last_hidden: torch.Tensor, claimed: Sequence[int], stream: Optional[torch.cuda.Stream] = None):
        """last_hidden: float32 device [n_check][d_model].  Returns device tensors (argmax int32, match uint8, margin f32)."""
        cl = _i32(claimed)
        n = int(cl.shape[0])
        if last_hidden.dtype != torch.float32 or not last_hidden.is_contiguous() or last_hidden.shape[0] != n:
            raise ValueError("last_hidden must be contiguous float32 [n_check][d_model]")
        arg = torch.empty(n, dtype=torch.int32, device=self.device)
        match = torch.empty(n, dtype=torch.uint8, device=self.device)
        margin = torch.empty(n, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(lib().verillm_token_match(self._h, last_hidden.data_ptr(), cl.ctypes.data, n, arg.data_ptr(),
                                             match.data_ptr(), margin.data_ptr(), _stream_ptr(stream)), "verillm_token_match")
        return arg, match, margin

    def profile_enable(self, on: bool = True) -> None:
        with torch.cuda.device(self.device):
            _check(lib().verillm_profile_enable(self._h, int(on)), "verillm_profile_enable")

    def profile_read(self) -> Dict[str, tuple]:
        """{kernel class: (milliseconds, launches)} of the last verify_prefill call."""
        ms = (C.c_float * len(PROF_CLASSES))()
        n = (C.c_int32 * len(PROF_CLASSES))()
        with torch.cuda.device(self.device):
            _check(lib().verillm_profile_read(self._h, ms, n), "verillm_profile_read")
        return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(PROF_CLASSES)}

    def last_launch_count(self) -> int:
        return int(lib().verillm_last_launch_count(self._h))

    def close(self) -> None:
        if self._h:
            with torch.cuda.device(self.device):
                lib().verillm_free(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def compare(hidden: torch.Tensor, committed: torch.Tensor, check_seq: Sequence[int], batch: int,
            tol: Optional[Tol] = None, stream: Optional[torch.cuda.Stream] = None) -> Report:
    """Comparison and verdict on given states: hidden f32 [L][n][d], committed bf16/f32 [L][n][d] (device)."""
    n_layers, n_check, d = hidden.shape
    cs = _i32(check_seq)
    tol = tol or default_tol()
    rep = Report(n_check, n_layers, batch, d, hidden.device, False)
    st = rep.c_struct()
    with torch.cuda.device(hidden.device):
        code = lib().verillm_compare(hidden.data_ptr(), committed.data_ptr(), BF16 if committed.dtype == torch.bfloat16 else F32,
                                     n_layers, n_check, d, cs.ctypes.data, batch, C.byref(tol), C.byref(st), _stream_ptr(stream))
    _check(code, "verillm_compare")
    return rep


def compare_noalloc(hidden: torch.Tensor, committed: torch.Tensor, check_seq: Sequence[int], batch: int,
                    tol: Optional[Tol] = None, report: Optional[Report] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> Report:
    """verillm_compare_noalloc: like `compare`, but the library's scratch is a fixed array inside the library,
    so the call itself allocates nothing.  Pass a `report` made beforehand to keep this wrapper from
    allocating the output tensors too.  Raises E_SHAPE beyond n_layers * n_check = 65536."""
    n_layers, n_check, d = hidden.shape
    cs = _i32(check_seq)
    tol = tol or default_tol()
    rep = report or Report(n_check, n_layers, batch, d, hidden.device, False)
    st = rep.c_struct()
    with torch.cuda.device(hidden.device):
        code = lib().verillm_compare_noalloc(hidden.data_ptr(), committed.data_ptr(),
                                             BF16 if committed.dtype == torch.bfloat16 else F32, n_layers, n_check, d,
                                             cs.ctypes.data, batch, C.byref(tol), C.byref(st), _stream_ptr(stream))
    _check(code, "verillm_compare_noalloc")
    return rep


def spot_check(hidden: torch.Tensor, sample_row, sample_col, reference, eps: float, theta: float,
               stream: Optional[torch.cuda.Stream] = None):
    """Sampled value matching on hidden (float32 device [n_rows][d]).  Returns device (agree uint8 [n], p_hat f32 [1], ok uint8 [1])."""
    rows, cols = _i32(sample_row), _i32(sample_col)
    ref = np.ascontiguousarray(np.asarray(reference, dtype=np.float32))
    n = int(rows.shape[0])
    agree = torch.empty(n, dtype=torch.uint8, device=hidden.device)
    p_hat = torch.empty(1, dtype=torch.float32, device=hidden.device)
    ok = torch.empty(1, dtype=torch.uint8, device=hidden.device)
    with torch.cuda.device(hidden.device):
        _check(lib().verillm_spot_check(hidden.data_ptr(), hidden.shape[0], hidden.shape[1], rows.ctypes.data,
                                        cols.ctypes.data, ref.ctypes.data, n, float(eps), float(theta), agree.data_ptr(),
                                        p_hat.data_ptr(), ok.data_ptr(), _stream_ptr(stream)), "verillm_spot_check")
    return agree, p_hat, ok


def threshold_sweep(stats: torch.Tensor, is_attack: torch.Tensor, variants: Sequence[Tol],
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """stats float32 device [n_cells][NSTAT] (report.stats reshaped), is_attack uint8 device [n_cells], up to 64
    tolerance sets -> int32 device [n_variants][4] = honest accepted, honest rejected, attack accepted, attack rejected."""
    if stats.dtype != torch.float32 or not stats.is_contiguous() or stats.dim() != 2 or stats.shape[1] != NSTAT:
        raise ValueError("stats must be a contiguous float32 [n_cells][NSTAT] tensor")
    if is_attack.dtype != torch.uint8 or not is_attack.is_contiguous() or is_attack.numel() != stats.shape[0]:
        raise ValueError("is_attack must be a contiguous uint8 tensor with one entry per cell")
    arr = (Tol * len(variants))(*variants)
    counts = torch.empty(len(variants), 4, dtype=torch.int32, device=stats.device)
    with torch.cuda.device(stats.device):
        _check(lib().verillm_threshold_sweep(stats.data_ptr(), is_attack.data_ptr(), stats.shape[0], arr, len(variants),
                                             counts.data_ptr(), _stream_ptr(stream)), "verillm_threshold_sweep")
    return counts


def selftest_wait_timeout(limit_cycles: int, device="cuda:0", stream: Optional[torch.cuda.Stream] = None):
    """Runs the library's bounded wait on a barrier nobody signals.  Returns device tensors (status int32 [1],
    gave_up int32 [1])."""
    device = torch.device(device)
    status = torch.zeros(1, dtype=torch.int32, device=device)
    gave_up = torch.zeros(1, dtype=torch.int32, device=device)
    with torch.cuda.device(device):
        _check(lib().verillm_selftest_wait_timeout(int(limit_cycles), status.data_ptr(), gave_up.data_ptr(),
                                                   _stream_ptr(stream)), "verillm_selftest_wait_timeout")
    return status, gave_up


def merkle_roots(states: torch.Tensor, stream: Optional[torch.cuda.Stream] = None,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """states float32 device [n_vec][d] -> uint8 device [n_vec][32] SHA-256 Merkle roots over float32 leaves
    (written to `out` if given)."""
    if states.dtype != torch.float32 or not states.is_contiguous() or states.dim() != 2:
        raise ValueError("states must be a contiguous float32 matrix")
    roots = out if out is not None else torch.empty(states.shape[0], 32, dtype=torch.uint8, device=states.device)
    if roots.dtype != torch.uint8 or tuple(roots.shape) != (states.shape[0], 32) or not roots.is_contiguous():
        raise ValueError("out must be a contiguous uint8 [n_vec][32] tensor")
    with torch.cuda.device(states.device):
        _check(lib().verillm_merkle_roots(states.data_ptr(), states.shape[0], states.shape[1], roots.data_ptr(),
                                          _stream_ptr(stream)), "verillm_merkle_roots")
    return roots


def op_gemm(a: torch.Tensor, b: torch.Tensor, out_f32: bool = False) -> torch.Tensor:
    """a [M][K] bf16, b [N][K] bf16 -> a @ b.T"""
    M, K = a.shape
    N = b.shape[0]
    c = torch.empty(M, N, dtype=torch.float32 if out_f32 else torch.bfloat16, device=a.device)
    status = torch.zeros(1, dtype=torch.int32, device=a.device)
    with torch.cuda.device(a.device):
        _check(lib().verillm_op_gemm(a.data_ptr(), b.data_ptr(), c.data_ptr(), M, N, K, int(out_f32), status.data_ptr(),
                                     _stream_ptr(None)), "verillm_op_gemm")
    if int(status.item()) != 0:
        raise RuntimeError(f"verillm_op_gemm: device status {int(status.item())}")
    return c


def op_rmsnorm(x: torch.Tensor, gain: torch.Tensor, eps: float) -> torch.Tensor:
    M, d = x.shape
    y = torch.empty(M, d, dtype=torch.bfloat16, device=x.device)
    with torch.cuda.device(x.device):
        _check(lib().verillm_op_rmsnorm(x.data_ptr(), gain.data_ptr(), y.data_ptr(), M, d, float(eps), _stream_ptr(None)),
               "verillm_op_rmsnorm")
    return y


def op_attention(qkv: torch.Tensor, cu_seqlens: Sequence[int], n_heads: int, n_kv_heads: int, head_dim: int) -> torch.Tensor:
    cu = _i32(cu_seqlens)
    M = qkv.shape[0]
    cu_dev = torch.from_numpy(cu).to(qkv.device)
    out = torch.empty(M, n_heads * head_dim, dtype=torch.bfloat16, device=qkv.device)
    max_len = int(np.max(np.diff(cu)))
    with torch.cuda.device(qkv.device):
        _check(lib().verillm_op_attention(qkv.data_ptr(), cu_dev.data_ptr(), len(cu) - 1, max_len, M, n_heads, n_kv_heads,
                                          head_dim, out.data_ptr(), _stream_ptr(None)), "verillm_op_attention")
    return out


# --------------------------------------------------------------------------- paged key/value cache

_KV_DTYPES = {torch.bfloat16: KV_BF16, torch.float8_e4m3fn: KV_E4M3, torch.int8: KV_INT8}


class _Fixed:
    """Attributes are set once: what the C side is told about them was taken when they were set."""

    def __setattr__(self, name, value):
        if name in self.__dict__:
            raise AttributeError(f"{type(self).__name__}.{name} cannot be replaced; make a new {type(self).__name__}")
        object.__setattr__(self, name, value)


class KVCache(_Fixed):
    """The paged cache of one layer: pools k, v [n_pages][n_kv_heads][page_size][head_dim] (bf16, float8_e4m3fn or int8)
    and, for 8-bit pools, float32 scales [n_pages][n_kv_heads][page_size].  Wraps the caller's tensors; `alloc` makes
    zeroed ones."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        dtype, shape, dev = _KV_DTYPES.get(k.dtype), k.shape, k.get_device()
        if dtype is None or len(shape) != 4 or v.dtype != k.dtype or v.shape != shape:
            raise ValueError("k and v pools must be [n_pages][n_kv_heads][page_size][head_dim] of one type: bf16, float8_e4m3fn or int8")
        if dtype != KV_BF16:
            if k_scale is None or v_scale is None:
                raise ValueError("8-bit pools need k_scale and v_scale")
            for t in (k_scale, v_scale):
                if t.dtype != torch.float32 or t.shape != shape[:3]:
                    raise ValueError("scales must be float32 [n_pages][n_kv_heads][page_size]")
                if t.get_device() != dev or not t.is_contiguous():
                    raise ValueError("pools and scales must be contiguous and on one CUDA device")
        elif k_scale is not None or v_scale is not None:
            raise ValueError("bf16 pools have no scales")
        if dev < 0 or v.get_device() != dev or not k.is_contiguous() or not v.is_contiguous():
            raise ValueError("pools and scales must be contiguous and on one CUDA device")
        n_pages, n_kv_heads, page_size, head_dim = shape
        self.__dict__.update(  # (at once: a program may wrap its tensors for every call)
            k=k, v=v, k_scale=k_scale, v_scale=v_scale, device=k.device, n_pages=n_pages, n_kv_heads=n_kv_heads, page_size=page_size, head_dim=head_dim,
            c_struct=KVCacheC(k.data_ptr(), v.data_ptr(), _ptr(k_scale), _ptr(v_scale), n_pages, page_size, n_kv_heads, head_dim, dtype))

    @property
    def raw(self) -> bytes:
        return bytes(self.c_struct)

    @classmethod
    def alloc(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16,
              device: str | torch.device = "cuda:0") -> "KVCache":
        pools = [torch.zeros(n_pages, n_kv_heads, page_size, head_dim, dtype=dtype, device=device) for _ in range(2)]
        scales = [None, None]
        if dtype != torch.bfloat16:
            scales = [torch.zeros(n_pages, n_kv_heads, page_size, dtype=torch.float32, device=device) for _ in range(2)]
        return cls(*pools, *scales)


class PagedRows(_Fixed):
    """The rows of a paged call: int32 device tensors page_table [batch][width], cu_rows [batch+1], kv_len [batch] and
    max_rows, at least every sequence's number of rows.  Row i of sequence b is position kv_len[b] - n_b + i of it.
    Pass `status` (int32 [1], zeroed) to have problems that only the device can see reported there; `check` reads it."""

    def __init__(self, page_table: torch.Tensor, cu_rows: torch.Tensor, kv_len: torch.Tensor, max_rows: int,
                 status: Optional[torch.Tensor] = None):
        dev = page_table.get_device()
        for t in (page_table, cu_rows, kv_len) if status is None else (page_table, cu_rows, kv_len, status):
            if t.dtype != torch.int32 or t.get_device() != dev or dev < 0 or not t.is_contiguous():
                raise ValueError("page_table, cu_rows, kv_len and status must be contiguous int32 tensors on one CUDA device")
        table = page_table.shape
        if len(table) != 2 or kv_len.shape != table[:1] or cu_rows.shape != (table[0] + 1,):
            raise ValueError("page_table is [batch][width], cu_rows [batch + 1], kv_len [batch]")
        self.__dict__.update(page_table=page_table, cu_rows=cu_rows, kv_len=kv_len, max_rows=min(int(max_rows), 0x7FFFFFFF), status=status,
                             device=page_table.device, _last=None)

    def c_struct(self, n_rows: int) -> KVRowsC:
        last = self._last  # the struct of the last call, if it had as many rows; never changed once made
        if last is None or last.n_rows != n_rows:
            batch, width = self.page_table.shape
            last = self.__dict__["_last"] = KVRowsC(self.page_table.data_ptr(), self.cu_rows.data_ptr(), self.kv_len.data_ptr(),
                                                    width, batch, n_rows, self.max_rows)
        return last

    def check(self) -> None:
        """Waits for the device and raises if a call reported a problem."""
        if self.status is not None and int(self.status.item()) != 0:
            raise RuntimeError(f"paged cache: device status {int(self.status.item())}")


def _packed_rows(t: torch.Tensor, what: str, width: int, head_dim: int, device: torch.device, dtype=torch.bfloat16) -> int:
    """Row stride of a [rows][width] or [rows][heads][head_dim] tensor whose rows are contiguous."""
    shape, strides = t.shape, t.stride()
    if t.dtype != dtype or t.device != device or len(shape) not in (2, 3):
        raise ValueError(f"{what} must be a 2- or 3-dimensional {dtype} tensor on {device}")
    if len(shape) == 2:
        packed = shape[1] == width
    else:
        packed = shape[2] == head_dim and shape[1] * head_dim == width and (shape[1] == 1 or strides[1] == head_dim)
    if not packed or strides[-1] != 1:
        raise ValueError(f"{what} must have {width} consecutive entries per row, in heads of {head_dim}")
    return strides[0] if shape[0] > 1 else width


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # as current_stream().cuda_stream, without the object


def _launch(device: torch.device, stream: Optional[torch.cuda.Stream], call):
    """call(stream pointer) with `device`, and `stream` if one is given, current: what the call allocates then belongs to
    the stream it runs on.  The common case, current device and stream, takes a short way: a decode step makes many calls."""
    if stream is None:
        if _raw_stream is not None and torch.cuda.current_device() == device.index:
            return call(_raw_stream(device.index))
        with torch.cuda.device(device):
            return call(_stream_ptr(None))
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the cache on {device}")
    with torch.cuda.stream(stream):
        return call(stream.cuda_stream)


def kv_write(cache: KVCache, rows: PagedRows, k: torch.Tensor, v: torch.Tensor,
             stream: Optional[torch.cuda.Stream] = None) -> None:
    """Stores the rows' keys and values (bf16 [n_rows][n_kv_heads * head_dim], e.g. column slices of a fused
    projection; keys already rotated) at their positions, quantised to the cache's type."""
    width = cache.n_kv_heads * cache.head_dim
    stride = _packed_rows(k, "k", width, cache.head_dim, cache.device)
    if _packed_rows(v, "v", width, cache.head_dim, cache.device) != stride or v.shape[0] != k.shape[0]:
        raise ValueError("k and v must have the same rows and row stride")
    if rows.device != cache.device:
        raise ValueError("rows and cache must be on one device")
    rc = rows.c_struct(k.shape[0])
    code = _launch(cache.device, stream, lambda st: lib().verillm_kv_write(
        C.byref(cache.c_struct), C.byref(rc), k.data_ptr(), v.data_ptr(), stride, _ptr(rows.status), st))
    _check(code, "verillm_kv_write")


def kv_read(cache: KVCache, rows: PagedRows, n_rows: int, dtype: torch.dtype = torch.bfloat16, out=None,
            stream: Optional[torch.cuda.Stream] = None):
    """(k, v) [n_rows][n_kv_heads][head_dim] in bf16 or float32: the rows' positions as numbers.  Rows behind the last
    sequence keep what `out` (a pair of such tensors) holds; without `out` they are not defined."""
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dtype must be bf16 or float32")
    if rows.device != cache.device:
        raise ValueError("rows and cache must be on one device")
    width = cache.n_kv_heads * cache.head_dim

    def call(st):
        k, v = out or [torch.empty(n_rows, cache.n_kv_heads, cache.head_dim, dtype=dtype, device=cache.device) for _ in range(2)]
        stride = width
        if out is not None:
            stride = _packed_rows(k, "k", width, cache.head_dim, cache.device, dtype)
            if _packed_rows(v, "v", width, cache.head_dim, cache.device, dtype) != stride or k.shape[0] != n_rows or v.shape[0] != n_rows:
                raise ValueError("out must be two tensors of n_rows rows with the same row stride")
        rc = rows.c_struct(n_rows)
        _check(lib().verillm_kv_read(C.byref(cache.c_struct), C.byref(rc), k.data_ptr(), v.data_ptr(), stride,
                                     F32 if dtype == torch.float32 else BF16, _ptr(rows.status), st), "verillm_kv_read")
        return k, v

    return _launch(cache.device, stream, call)


def op_attention_paged(q: torch.Tensor, cache: KVCache, rows: PagedRows, out: Optional[torch.Tensor] = None,
                       lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Causal grouped-query attention of the rows' queries (bf16 [n_rows][n_heads * head_dim], already rotated) over
    the cache -> bf16 [n_rows][n_heads * head_dim].  lse: optional float32 [n_rows][n_heads] that receives the log of
    the sum of exp(scores).  workspace: optional uint8 tensor of `attention_paged_workspace` bytes to use instead of
    allocating one for the call.  Rows behind the last sequence keep what `out` and `lse` hold; without `out` they are not defined."""
    shape = q.shape
    if len(shape) not in (2, 3):
        raise ValueError("q must be [n_rows][n_heads * head_dim] or [n_rows][n_heads][head_dim]")
    n_rows, n_heads = shape[0], shape[1] if len(shape) == 3 else shape[1] // cache.head_dim
    width = n_heads * cache.head_dim
    q_stride = _packed_rows(q, "q", width, cache.head_dim, cache.device)
    if rows.device != cache.device:
        raise ValueError("rows and cache must be on one device")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (n_rows, n_heads) or not lse.is_contiguous() or lse.device != cache.device):
        raise ValueError("lse must be a contiguous float32 [n_rows][n_heads] tensor on the cache's device")
    rc = rows.c_struct(n_rows)
    L = lib()

    def call(st):
        o, stride, ws = out, width, workspace
        if o is None:
            o = torch.empty(n_rows, width, dtype=torch.bfloat16, device=cache.device)
        else:
            stride = _packed_rows(o, "out", width, cache.head_dim, cache.device)
            if o.shape[0] != n_rows:
                raise ValueError("out must have as many rows as q")
        if ws is None:
            need = L.verillm_op_attention_paged_workspace(C.byref(cache.c_struct), C.byref(rc), n_heads)
            if need < 0:
                raise VerillmError(int(need), "verillm_op_attention_paged_workspace")
            ws = torch.empty(need, dtype=torch.uint8, device=cache.device) if need else None
        elif ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.device != cache.device:
            raise ValueError("workspace must be a contiguous uint8 tensor on the cache's device")
        _check(L.verillm_op_attention_paged(C.byref(cache.c_struct), C.byref(rc), q.data_ptr(), q_stride, n_heads, o.data_ptr(),
                                            stride, _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel(), _ptr(rows.status), st),
               "verillm_op_attention_paged")
        return o

    return _launch(cache.device, stream, call)


def attention_paged_workspace(cache: KVCache, rows: PagedRows, n_rows: int, n_heads: int) -> int:
    """Bytes of workspace that op_attention_paged needs for calls of up to n_rows rows and as many sequences as `rows` has."""
    rc = rows.c_struct(n_rows)
    with torch.cuda.device(cache.device):
        need = lib().verillm_op_attention_paged_workspace(C.byref(cache.c_struct), C.byref(rc), n_heads)
    if need < 0:
        raise VerillmError(int(need), "verillm_op_attention_paged_workspace")
    return int(need)


# --------------------------------------------------------------------------- 4-bit weights


class W4Weights(_Fixed):
    """4-bit weights: codes uint8 [n][k / 2] (code + 8, the even input in the low half), scales bf16 [k / group][n].  Wraps the caller's tensors;
    `w4_quantise` makes them from bf16 weights."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, group: int = 128):
        shape, dev = codes.shape, codes.get_device()
        if codes.dtype != torch.uint8 or len(shape) != 2 or scales.dtype != torch.bfloat16 or group not in (32, 64, 128):
            raise ValueError("codes must be uint8 [n][k / 2], scales bf16 [k / group][n], group 32, 64 or 128")
        n, k = shape[0], 2 * shape[1]
        if k % group or scales.shape != (k // group, n):
            raise ValueError("codes must be uint8 [n][k / 2], scales bf16 [k / group][n], group 32, 64 or 128")
        if dev < 0 or scales.get_device() != dev or not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError("codes and scales must be contiguous and on one CUDA device")
        self.__dict__.update(codes=codes, scales=scales, group=group, n=n, k=k, device=codes.device,
                             c_struct=W4C(codes.data_ptr(), scales.data_ptr(), n, k, group))


def _strided(t: torch.Tensor, what: str, rows: int, width: int, dtype: torch.dtype, device: torch.device) -> int:
    """Row stride of a [rows][width] matrix whose rows are contiguous."""
    if t.dtype is not dtype or t.get_device() != device.index or t.shape != (rows, width):
        raise ValueError(f"{what} must be a {dtype} [{rows}][{width}] tensor with contiguous rows on {device}")
    strides = t.stride()
    if strides[1] != 1 and width > 1:
        raise ValueError(f"{what} must be a {dtype} [{rows}][{width}] tensor with contiguous rows on {device}")
    return strides[0] if rows > 1 else width


def w4_quantise(w: torch.Tensor, group: int = 128, stream: Optional[torch.cuda.Stream] = None) -> W4Weights:
    """bf16 [n][k] (rows may be strided) -> 4-bit weights with one scale per `group` inputs."""
    if w.dim() != 2 or not w.is_cuda or group not in (32, 64, 128) or w.shape[1] % group:
        raise ValueError("w must be a CUDA matrix whose rows are whole groups of 32, 64 or 128")
    stride = _strided(w, "w", w.shape[0], w.shape[1], torch.bfloat16, w.device)

    def call(st):
        out = W4Weights(torch.empty(w.shape[0], w.shape[1] // 2, dtype=torch.uint8, device=w.device),
                        torch.empty(w.shape[1] // group, w.shape[0], dtype=torch.bfloat16, device=w.device), group)
        _check(lib().verillm_w4_quantise(w.data_ptr(), stride, C.byref(out.c_struct), st), "verillm_w4_quantise")
        return out

    return _launch(w.device, stream, call)


def w4_dequantise(w: W4Weights, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """[n][k] in bf16 or float32: what the 4-bit weights stand for."""
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dtype must be bf16 or float32")

    def call(st):
        o = torch.empty(w.n, w.k, dtype=dtype, device=w.device) if out is None else out
        stride = _strided(o, "out", w.n, w.k, dtype, w.device)
        _check(lib().verillm_w4_dequantise(C.byref(w.c_struct), o.data_ptr(), stride, F32 if dtype == torch.float32 else BF16, st), "verillm_w4_dequantise")
        return o

    return _launch(w.device, stream, call)


def op_w4_matvec(x: torch.Tensor, w: W4Weights, residual: Optional[torch.Tensor] = None, dtype: Optional[torch.dtype] = None,
                 out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """x (bf16 [rows][k], rows may be strided) @ w.T (+ residual, float32 [rows][n]) -> [rows][n] in `dtype` (that of `out`, else bf16).
    residual may be `out` itself.  status: optional int32 [1] that device problems are reported in."""
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("x must be [rows][k]")
    rows, stride = shape[0], _strided(x, "x", shape[0], w.k, torch.bfloat16, w.device)
    res_stride = 0 if residual is None else _strided(residual, "residual", rows, w.n, torch.float32, w.device)
    dtype = dtype or (torch.bfloat16 if out is None else out.dtype)
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dtype must be bf16 or float32")
    _check_word(status, w.device)
    L = lib()

    def call(st):
        y = torch.empty(rows, w.n, dtype=dtype, device=w.device) if out is None else out
        y_stride = w.n if out is None else _strided(y, "out", rows, w.n, dtype, w.device)
        _check(L.verillm_op_w4_matvec(C.byref(w.c_struct), x.data_ptr(), stride, rows, _ptr(residual), res_stride, y.data_ptr(), y_stride,
                                      F32 if dtype == torch.float32 else BF16, _ptr(status), st), "verillm_op_w4_matvec")
        return y

    return _launch(w.device, stream, call)


def _check_word(t: Optional[torch.Tensor], device: torch.device) -> None:
    if t is not None and (t.dtype != torch.int32 or t.numel() != 1 or t.device != device):
        raise ValueError(f"status must be an int32 tensor of one entry on {device}")


def _vector(t: torch.Tensor, what: str, n: int, dtype: torch.dtype, index: int) -> None:
    if t.dtype is not dtype or t.dim() != 1 or t.shape[0] != n or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} [{n}] tensor on cuda:{index}")


def _call(what: str, device: torch.device, stream: Optional[torch.cuda.Stream], fn, *args) -> None:
    """fn(*args, stream pointer) as `_launch` makes it, and its answer checked; for calls that allocate nothing themselves."""
    if stream is None and _raw_stream is not None and torch.cuda.current_device() == device.index:
        code = fn(*args, _raw_stream(device.index))
    else:
        code = _launch(device, stream, lambda st: fn(*args, st))
    if code != 0:
        raise VerillmError(code, what)


# --------------------------------------------------------------------------- drafted tokens


class DraftReport:
    """Device tensors of one check: tokens int32 [n_rows] (what was emitted, -1 behind it), n_emitted int32 [batch], logp float32 [n_rows], new_len
    int32 [batch] (None without kv_len).  Rows behind the last sequence keep what the tensors held (nothing defined in a fresh report)."""

    def __init__(self, n_rows: int, batch: int, device, with_len: bool):
        self.tokens = torch.empty(n_rows, dtype=torch.int32, device=device)
        self.n_emitted = torch.empty(batch, dtype=torch.int32, device=device)
        self.logp = torch.empty(n_rows, dtype=torch.float32, device=device)
        self.new_len = torch.empty(batch, dtype=torch.int32, device=device) if with_len else None


def verify_drafts(target: torch.Tensor, tokens: torch.Tensor, cu_rows: torch.Tensor, max_rows: int, accept_u: torch.Tensor, sample_u: torch.Tensor,
                  draft: Optional[torch.Tensor] = None, temperature: Optional[torch.Tensor] = None, kv_len: Optional[torch.Tensor] = None,
                  report: Optional[DraftReport] = None, workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> DraftReport:
    """Checks drafted tokens against the target's logits (bf16 or float32 [n_rows][vocab], rows may be strided) with given random numbers: accept_u
    float32 [n_rows], sample_u float32 [batch].  tokens int32 [n_rows]: every row's input token; those of a sequence's rows behind its first are the
    drafted ones.  draft: the logits they were drawn from, the same type; without it they count as certain.  temperature float32 [batch], 0 for the
    largest logit; 1 without it.  kv_len int32 [batch]: gives the report's new_len.  All on one device; the header has the definitions."""
    if target.dim() != 2 or not target.is_cuda or target.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("target must be a bf16 or float32 CUDA matrix")
    dev, (n_rows, vocab), at = target.device, target.shape, target.get_device()
    batch = cu_rows.shape[0] - 1 if cu_rows.dim() == 1 else 0
    t_stride = _strided(target, "target", n_rows, vocab, target.dtype, dev)
    d_stride = 0 if draft is None else _strided(draft, "draft", n_rows, vocab, target.dtype, dev)
    _vector(cu_rows, "cu_rows", batch + 1, torch.int32, at)
    _vector(tokens, "tokens", n_rows, torch.int32, at)
    _vector(accept_u, "accept_u", n_rows, torch.float32, at)
    _vector(sample_u, "sample_u", batch, torch.float32, at)
    if temperature is not None:
        _vector(temperature, "temperature", batch, torch.float32, at)
    if kv_len is not None:
        _vector(kv_len, "kv_len", batch, torch.int32, at)
    _check_word(status, dev)
    if report is not None:
        _vector(report.tokens, "report.tokens", n_rows, torch.int32, at)
        _vector(report.n_emitted, "report.n_emitted", batch, torch.int32, at)
        if report.logp is not None:
            _vector(report.logp, "report.logp", n_rows, torch.float32, at)
        if report.new_len is not None:
            _vector(report.new_len, "report.new_len", batch, torch.int32, at)
            if kv_len is None or report.new_len.data_ptr() == kv_len.data_ptr():
                raise ValueError("report.new_len needs a kv_len, and one that it is not itself")
    L = lib()

    def call(st):
        rep = report or DraftReport(n_rows, batch, dev, kv_len is not None)
        ws = workspace
        if ws is None:
            ws = torch.empty(max(16, L.verillm_verify_drafts_workspace(n_rows)), dtype=torch.uint8, device=dev)
        elif ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.device != dev:
            raise ValueError("workspace must be a contiguous uint8 tensor on the logits' device")
        d = DraftsC(target.data_ptr(), _ptr(draft), t_stride, d_stride, F32 if target.dtype == torch.float32 else BF16, vocab, batch, n_rows,
                    min(int(max_rows), 0x7FFFFFFF), cu_rows.data_ptr(), tokens.data_ptr(), _ptr(kv_len), _ptr(temperature), accept_u.data_ptr(),
                    sample_u.data_ptr())
        r = DraftReportC(rep.tokens.data_ptr(), rep.n_emitted.data_ptr(), _ptr(rep.logp), _ptr(rep.new_len))
        _check(L.verillm_verify_drafts(C.byref(d), C.byref(r), ws.data_ptr(), ws.numel(), _ptr(status), st), "verillm_verify_drafts")
        return rep

    return _launch(dev, stream, call)


def verify_drafts_workspace(n_rows: int) -> int:
    """Bytes of workspace that verify_drafts needs for calls of up to n_rows rows."""
    need = lib().verillm_verify_drafts_workspace(n_rows)
    if need < 0:
        raise VerillmError(int(need), "verillm_verify_drafts_workspace")
    return int(need)


# --------------------------------------------------------------------------- pages of a paged cache


def _layers(caches: Sequence[KVCache]):
    """The caches' descriptions as a C array."""
    return (KVCacheC * len(caches)).from_buffer_copy(b"".join([c.raw for c in caches]))


class KVPages(_Fixed):
    """Who holds which page of a model's paged cache: caches (one KVCache per layer, one geometry), page_table int32 [batch][width], kv_len int32
    [batch], refs int32 [n_pages] (table entries that name a page; 0: free).  The calls on it change these tensors and must follow one
    another.  `alloc` makes an empty one.  Pass `status` (int32 [1], zeroed) to have device problems reported there; `check` reads it.  Only the tensors
    passed in have to outlive the calls' work on the device (and captured graphs), the holder itself need not."""

    def __init__(self, caches: Sequence[KVCache], page_table: torch.Tensor, kv_len: torch.Tensor, refs: torch.Tensor,
                 status: Optional[torch.Tensor] = None):
        caches = tuple(caches)
        if not caches:
            raise ValueError("at least one layer's cache")
        dev = caches[0].device
        if page_table.dim() != 2 or page_table.dtype != torch.int32 or page_table.device != dev or not page_table.is_contiguous():
            raise ValueError(f"page_table must be a contiguous int32 [batch][width] tensor on {dev}")
        batch, width = page_table.shape
        _vector(kv_len, "kv_len", batch, torch.int32, dev.index)
        _vector(refs, "refs", caches[0].n_pages, torch.int32, dev.index)
        if any(c.device != dev for c in caches):
            raise ValueError("all layers must be on one device")
        _check_word(status, dev)
        need = lib().verillm_kv_pages_workspace(batch, caches[0].n_pages)
        if need < 0:
            raise VerillmError(int(need), "verillm_kv_pages_workspace")
        layers = _layers(caches)
        workspace = torch.empty(int(need), dtype=torch.uint8, device=dev)
        c_struct = KVPagesC(layers, len(caches), page_table.data_ptr(), kv_len.data_ptr(), refs.data_ptr(), batch, width)
        self.__dict__.update(caches=caches, page_table=page_table, kv_len=kv_len, refs=refs, status=status, device=dev, layers=layers, batch=batch,
                             workspace=workspace, c_struct=c_struct, _ref=C.byref(c_struct), _ws=workspace.data_ptr(), _ws_bytes=int(need), _status=_ptr(status),
                             _index=dev.index, _ws_stream=_raw_stream(dev.index) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream)

    @classmethod
    def alloc(cls, n_layers: int, batch: int, width: int, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int,
              dtype: torch.dtype = torch.bfloat16, device: str | torch.device = "cuda:0") -> "KVPages":
        caches = [KVCache.alloc(n_pages, page_size, n_kv_heads, head_dim, dtype, device) for _ in range(n_layers)]
        return cls(caches, *[torch.zeros(*s, dtype=torch.int32, device=device) for s in ((batch, width), (batch,), (n_pages,), (1,))])

    def rows(self, cu_rows: torch.Tensor, max_rows: int) -> PagedRows:
        """The rows of a paged call on these sequences."""
        return PagedRows(self.page_table, cu_rows, self.kv_len, max_rows, self.status)

    def check(self) -> None:
        """Waits for the device and raises if a call reported a problem."""
        if self.status is not None and int(self.status.item()) != 0:
            raise RuntimeError(f"cache pages: device status {int(self.status.item())}")


def _pages_call(what: str, pages: KVPages, stream: Optional[torch.cuda.Stream], fn, *args) -> None:
    """fn(pages, *args, workspace, its bytes, status, stream pointer).  The holder's workspace belongs to the stream it was made on and goes with the
    holder: calls on another stream, and captured ones, allocate theirs."""
    index = pages._index
    if stream is None and _raw_stream is not None and torch.cuda.current_device() == index:
        st = _raw_stream(index)
        if st == pages._ws_stream and (st == 0 or not torch.cuda.is_current_stream_capturing()):  # (the default stream is never captured)
            code = fn(pages._ref, *args, pages._ws, pages._ws_bytes, pages._status, st)
            if code:
                raise VerillmError(code, what)
            return

    def call(st):
        ws = torch.empty(pages._ws_bytes, dtype=torch.uint8, device=pages.device)
        return fn(pages._ref, *args, ws.data_ptr(), pages._ws_bytes, pages._status, st)

    _check(_launch(pages.device, stream, call), what)


def kv_reserve(pages: KVPages, new_len: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Grows every sequence with new_len[b] > kv_len[b] (int32 [batch]) to new_len[b]: lowest free pages first, a copy of a partly filled page that
    others hold too.  Where the free pages do not suffice, that sequence and the later ones stay as they are (DEV_NO_PAGES)."""
    _vector(new_len, "new_len", pages.batch, torch.int32, pages.device.index)
    _pages_call("verillm_kv_reserve", pages, stream, lib().verillm_kv_reserve, new_len.data_ptr())


def kv_free(pages: KVPages, new_len: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Shortens every sequence with new_len[b] < kv_len[b] (int32 [batch]) to new_len[b] and lets go of the pages behind."""
    _vector(new_len, "new_len", pages.batch, torch.int32, pages.device.index)
    _call("verillm_kv_free", pages.device, stream, lib().verillm_kv_free, pages._ref, new_len.data_ptr(), pages._status)


def kv_fork(pages: KVPages, src: torch.Tensor, dst: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """The empty sequences dst (int32 [n]) come to share what the sequences src hold."""
    n = src.shape[0] if src.dim() == 1 else -1
    _vector(src, "src", n, torch.int32, pages.device.index)
    _vector(dst, "dst", n, torch.int32, pages.device.index)
    _pages_call("verillm_kv_fork", pages, stream, lib().verillm_kv_fork, src.data_ptr(), dst.data_ptr(), n)


def kv_compact(pages: KVPages, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Moves the pages in use to the front of the pools; returns their number (int32 [1], device)."""
    if stream is None:
        used = torch.empty(1, dtype=torch.int32, device=pages.device)
    else:
        used = _launch(pages.device, stream, lambda st: torch.empty(1, dtype=torch.int32, device=pages.device))
    _pages_call("verillm_kv_compact", pages, stream, lib().verillm_kv_compact, used.data_ptr())
    return used


def kv_copy(src: Sequence[KVCache], dst: Sequence[KVCache], src_pages: torch.Tensor, dst_pages: torch.Tensor,
            status: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Copies pages src_pages (int32 [n]) of the caches src, one per layer, to pages dst_pages of the caches dst; pairs with a -1 are left out."""
    if not dst:
        raise ValueError("at least one layer's cache")
    dev, n = dst[0].device, src_pages.shape[0] if src_pages.dim() == 1 else -1
    if len(src) != len(dst) or any(c.device != dev for c in src) or any(c.device != dev for c in dst):
        raise ValueError("src and dst must have the same number of layers, all on one device")
    _vector(src_pages, "src_pages", n, torch.int32, dev.index)
    _vector(dst_pages, "dst_pages", n, torch.int32, dev.index)
    _check_word(status, dev)
    _call("verillm_kv_copy", dev, stream, lib().verillm_kv_copy, _layers(src), _layers(dst), len(dst), src_pages.data_ptr(), dst_pages.data_ptr(), n, _ptr(status))
