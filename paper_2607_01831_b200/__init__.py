"""Thin Python binding of the Lynx C-ABI CUDA library (sm_100a).

Argument marshalling only: every step of the path runs in the library's kernels.  Torch is
used for device memory and streams.  There is no CPU fallback: if ``liblynx.so`` is missing
or a call returns an error status, an exception is raised.

Names mirror ``include/lynx.h``: split_quantize, recombine, anchor_attention,
merge_verify_attention, workspace_bytes.
"""
from __future__ import annotations

import ctypes
import functools
import os
import warnings
from dataclasses import dataclass
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liblynx.so")
_lib = None

D = 128


class LynxError(RuntimeError):
    pass


class _Plane(ctypes.Structure):
    _fields_ = [("anchor", ctypes.c_void_p), ("residual", ctypes.c_void_p), ("meta", ctypes.c_void_p)]


class _RotarySpec(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("cos_sin", ctypes.c_void_p), ("positions_stride", ctypes.c_int64),
                ("n_axes", ctypes.c_int32), ("n_positions", ctypes.c_int32), ("n_pairs", ctypes.c_int32),
                ("interleaved", ctypes.c_int32), ("pair_axis", ctypes.c_uint8 * 64)]


class _HeadNorm(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float), ("weight_float", ctypes.c_int32)]


class _Shape(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("block_tokens", ctypes.c_int32),
                ("num_blocks", ctypes.c_int32), ("max_blocks_per_seq", ctypes.c_int32)]


EXPORTS = ["lynx_split_quantize", "lynx_recombine", "lynx_workspace_bytes", "lynx_workspace_init",
           "lynx_anchor_attention", "lynx_merge_verify_attention", "lynx_anchor_attention_static",
           "lynx_bf16_workspace_bytes", "lynx_bf16_attention", "lynx_hier_quantize", "lynx_hier_dequantize",
           "lynx_token_verify", "lynx_workspace_lse", "lynx_bf16_workspace_lse", "lynx_lse_merge", "lynx_verify_decision", "lynx_split_quantize_bits", "lynx_recombine_bits",
           "lynx_rotary", "lynx_cache_append", "lynx_cache_read", "lynx_tree_workspace_bytes", "lynx_tree_attention",
           "lynx_norm_rotary", "lynx_norm_cache_append", "lynx_plan_blocks", "lynx_latent_append", "lynx_latent_read",
           "lynx_latent_workspace_bytes", "lynx_latent_attention",
           "lynx_check",
           "lynx_status_string", "lynx_version"]


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load liblynx.so (built in-tree by paper_2607_01831_b200/build.py). Fails loudly."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise LynxError(f"{_LIB_PATH} is missing: build it with `python -m paper_2607_01831_b200.build` "
                        "(there is no CPU fallback)")
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    lib.lynx_split_quantize.argtypes = [vp, i64, vp, i32, i32, vp, vp, vp, vp]
    lib.lynx_split_quantize.restype = ctypes.c_int
    lib.lynx_recombine.argtypes = [vp, vp, vp, i64, vp, vp, vp]
    lib.lynx_recombine.restype = ctypes.c_int
    lib.lynx_workspace_bytes.argtypes = [ctypes.POINTER(_Shape), i32, i32]
    lib.lynx_workspace_bytes.restype = ctypes.c_size_t
    lib.lynx_workspace_init.argtypes = [vp, ctypes.c_size_t, vp]
    lib.lynx_workspace_init.restype = ctypes.c_int
    lib.lynx_anchor_attention.argtypes = [ctypes.POINTER(_Shape), vp, i32, i32, i32, _Plane, _Plane,
                                          vp, vp, f32, vp, vp, ctypes.c_size_t, vp]
    lib.lynx_anchor_attention.restype = ctypes.c_int
    lib.lynx_merge_verify_attention.argtypes = [ctypes.POINTER(_Shape), vp, i32, i32, i32, _Plane,
                                                _Plane, vp, vp, f32, vp, f32, f32, vp, vp, vp, vp,
                                                ctypes.c_size_t, vp]
    lib.lynx_merge_verify_attention.restype = ctypes.c_int
    lib.lynx_anchor_attention_static.argtypes = [ctypes.POINTER(_Shape), vp, i32, i32, i32, _Plane,
                                                 _Plane, vp, vp, f32, vp, vp]
    lib.lynx_anchor_attention_static.restype = ctypes.c_int
    lib.lynx_bf16_workspace_bytes.argtypes = [ctypes.POINTER(_Shape), i32, i32]
    lib.lynx_bf16_workspace_bytes.restype = ctypes.c_size_t
    lib.lynx_bf16_attention.argtypes = [ctypes.POINTER(_Shape), vp, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp,
                                        ctypes.c_size_t, vp]
    lib.lynx_bf16_attention.restype = ctypes.c_int
    lib.lynx_hier_quantize.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.lynx_hier_quantize.restype = ctypes.c_int
    lib.lynx_hier_dequantize.argtypes = [vp, vp, i64, vp, vp, vp, vp, vp, vp]
    lib.lynx_hier_dequantize.restype = ctypes.c_int
    lib.lynx_token_verify.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp, vp]
    lib.lynx_token_verify.restype = ctypes.c_int
    lib.lynx_workspace_lse.argtypes = [ctypes.POINTER(_Shape), i32, i32, vp]
    lib.lynx_workspace_lse.restype = ctypes.c_void_p
    lib.lynx_bf16_workspace_lse.argtypes = [ctypes.POINTER(_Shape), i32, i32, vp]
    lib.lynx_bf16_workspace_lse.restype = ctypes.c_void_p
    lib.lynx_lse_merge.argtypes = [vp, vp, vp, vp, i64, vp, vp, vp]
    lib.lynx_lse_merge.restype = ctypes.c_int
    lib.lynx_verify_decision.argtypes = [vp, vp, i32, i32, i32, f32, f32, vp, vp, vp]
    lib.lynx_verify_decision.restype = ctypes.c_int
    lib.lynx_split_quantize_bits.argtypes = [vp, i64, i32, vp, vp, vp, vp]
    lib.lynx_split_quantize_bits.restype = ctypes.c_int
    lib.lynx_recombine_bits.argtypes = [vp, vp, vp, i64, i32, vp, vp, vp]
    lib.lynx_recombine_bits.restype = ctypes.c_int
    lib.lynx_rotary.argtypes = [ctypes.POINTER(_RotarySpec), vp, i64, i32, vp, i64, i32, i64, vp, i64, vp, i64, vp]
    lib.lynx_rotary.restype = ctypes.c_int
    lib.lynx_cache_append.argtypes = [ctypes.POINTER(_Shape), vp, i64, vp, i64, i64, vp, i64, vp, ctypes.POINTER(_RotarySpec),
                                      _Plane, _Plane, vp]
    lib.lynx_cache_append.restype = ctypes.c_int
    lib.lynx_cache_read.argtypes = [ctypes.POINTER(_Shape), _Plane, _Plane, vp, i32, vp, vp, i64, vp, vp, vp]
    lib.lynx_cache_read.restype = ctypes.c_int
    lib.lynx_tree_workspace_bytes.argtypes = [ctypes.POINTER(_Shape), i32, i32]
    lib.lynx_tree_workspace_bytes.restype = ctypes.c_size_t
    lib.lynx_tree_attention.argtypes = [ctypes.POINTER(_Shape), vp, i32, i32, _Plane, _Plane, vp, vp, vp, i64, vp, i64, vp, f32, i32,
                                        vp, vp, vp, ctypes.c_size_t, vp]
    lib.lynx_tree_attention.restype = ctypes.c_int
    lib.lynx_norm_rotary.argtypes = [ctypes.POINTER(_HeadNorm), ctypes.POINTER(_RotarySpec), i32, vp, i64, i32, vp, i64, i32, i64, vp, i64, vp,
                                     i64, vp]
    lib.lynx_norm_rotary.restype = ctypes.c_int
    lib.lynx_norm_cache_append.argtypes = [ctypes.POINTER(_Shape), vp, i64, vp, i64, i64, vp, i64, vp, ctypes.POINTER(_HeadNorm),
                                           ctypes.POINTER(_RotarySpec), _Plane, _Plane, vp]
    lib.lynx_norm_cache_append.restype = ctypes.c_int
    lib.lynx_plan_blocks.argtypes = [ctypes.POINTER(_Shape), vp, vp, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp]
    lib.lynx_plan_blocks.restype = ctypes.c_int
    lib.lynx_latent_append.argtypes = [ctypes.POINTER(_Shape), vp, i64, vp, i64, i64, vp, i64, vp, vp, i32, f32, ctypes.POINTER(_RotarySpec),
                                       _Plane, vp, vp]
    lib.lynx_latent_append.restype = ctypes.c_int
    lib.lynx_latent_read.argtypes = [ctypes.POINTER(_Shape), _Plane, vp, vp, i32, vp, vp, i64, vp, vp, vp]
    lib.lynx_latent_read.restype = ctypes.c_int
    lib.lynx_latent_workspace_bytes.argtypes = [ctypes.POINTER(_Shape), i32, i32]
    lib.lynx_latent_workspace_bytes.restype = ctypes.c_size_t
    lib.lynx_latent_attention.argtypes = [ctypes.POINTER(_Shape), vp, i64, vp, i64, i32, i32, i32, _Plane, vp, vp, vp, f32, i32, vp, vp, vp,
                                          ctypes.c_size_t, vp]
    lib.lynx_latent_attention.restype = ctypes.c_int
    lib.lynx_check.argtypes = [vp, vp]
    lib.lynx_check.restype = ctypes.c_int
    lib.lynx_status_string.argtypes = [ctypes.c_int]
    lib.lynx_status_string.restype = ctypes.c_char_p
    lib.lynx_version.restype = ctypes.c_int
    _lib = lib
    return lib


def _ok(status: int, what: str):
    if status != 0:
        msg = load().lynx_status_string(status).decode()
        raise LynxError(f"{what}: status {status} ({msg})")


def _result(r, what: str):
    """What a fast call returned: its result, or a status to raise."""
    if type(r) is int:
        _ok(r, what)
    return r


def _ptr(t: torch.Tensor | None):
    if t is None:
        return None
    if not t.is_cuda:
        raise LynxError("device tensors required")
    if not t.is_contiguous():
        raise LynxError("contiguous tensors required")
    return t.data_ptr()


# The current stream's handle without a Stream object on the way (two quantisations of 4096 arrived tokens: 18.7 -> 11.4 us,
# an anchor call on 4096 tokens 15.0 -> 13.6 us); builds of torch without these two functions go through one.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is None or _raw_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_raw_device())


# The calls below that a program makes per layer and step go through an extension (csrc/native.cpp) that does what their Python
# bodies do, in one call; it returns None for whatever is not plain, and then the Python body runs.  us of host time per call
# (marshalling through ctypes -> extension): anchor_attention 12 -> 5 to 8, merge_verify_attention 17 -> 10, the four calls of a decode with a BF16
# tail 45 -> 21, Algorithm 1 there and back for K and V 51 -> 28.
def _python_only(*_):
    return None


@functools.lru_cache(maxsize=None)
def _extension():
    """The extension, or None (with a warning, once) where it does not load or was compiled against another torch, whose tensors
    it would read wrongly."""
    load()   # (raises where the library is not built)
    try:
        from . import _native
        built = _native.torch_version
        if built == torch.__version__:
            return _native
        why = f"it was built for torch {built}, this is {torch.__version__}"
    except ImportError as e:
        why = str(e)
    warnings.warn(f"paper_2607_01831_b200._native is not used ({why}): calls go through ctypes and take about twice the host time; "
                  "rebuild with `python -m paper_2607_01831_b200.build`", RuntimeWarning)
    return None


def _fast(var: str, name: str):
    """The extension's function `name`, found when the global `var` that holds this is first called."""
    def first(*args):
        globals()[var] = getattr(_extension(), name, _python_only)
        return globals()[var](*args)
    return first


_fast_split_quantize, _fast_recombine = _fast("_fast_split_quantize", "split_quantize"), _fast("_fast_recombine", "recombine")
_fast_anchor, _fast_verify = _fast("_fast_anchor", "anchor_attention"), _fast("_fast_verify", "merge_verify_attention")
_fast_bf16, _fast_lse_view = _fast("_fast_bf16", "bf16_attention"), _fast("_fast_lse_view", "lse_view")
_fast_lse_merge = _fast("_fast_lse_merge", "lse_merge")
_fast_rotary, _fast_cache_append = _fast("_fast_rotary", "rotary"), _fast("_fast_cache_append", "cache_append")
_fast_cache_read, _fast_tree_attention = _fast("_fast_cache_read", "cache_read"), _fast("_fast_tree_attention", "tree_attention")
_fast_norm_rotary, _fast_norm_append = _fast("_fast_norm_rotary", "norm_rotary"), _fast("_fast_norm_append", "norm_cache_append")
_fast_plan_blocks = _fast("_fast_plan_blocks", "plan_blocks")
_fast_latent_attention = _fast("_fast_latent_attention", "latent_attention")
_fast_latent_append, _fast_latent_read = _fast("_fast_latent_append", "latent_append"), _fast("_fast_latent_read", "latent_read")
_fast_hier_quantize, _fast_hier_dequantize = _fast("_fast_hier_quantize", "hier_quantize"), _fast("_fast_hier_dequantize", "hier_dequantize")


@dataclass
class Planes:
    """Quantised K or V: anchor / residual u8 [..., 64], meta f32 [..., 2] (device tensors)."""
    anchor: torch.Tensor
    residual: torch.Tensor | None
    meta: torch.Tensor

    def _c(self) -> _Plane:
        return _Plane(_ptr(self.anchor), _ptr(self.residual), _ptr(self.meta))


def alloc_planes(lead_shape, device) -> Planes:
    lead = tuple(lead_shape)
    return Planes(torch.empty(lead + (64,), dtype=torch.uint8, device=device),
                  torch.empty(lead + (64,), dtype=torch.uint8, device=device),
                  torch.empty(lead + (2,), dtype=torch.float32, device=device))


def split_quantize(src: torch.Tensor, out: Planes | None = None, block_ids: torch.Tensor | None = None,
                   rows_per_block: int = 0) -> Planes:
    """lynx_split_quantize: src BF16 [..., 128] -> Planes with the same leading shape."""
    if src.dtype != torch.bfloat16 or src.shape[-1] != D:
        raise LynxError("src must be BF16 [..., 128]")
    if out is None:
        out = alloc_planes(src.shape[:-1], src.device)
    r = _fast_split_quantize(src, out, block_ids, rows_per_block)
    if r is not None:
        _ok(r, "lynx_split_quantize")
        return out
    n_rows = src.numel() // D
    nb = 0 if block_ids is None else block_ids.numel()
    _ok(load().lynx_split_quantize(_ptr(src), n_rows, _ptr(block_ids), nb, rows_per_block,
                                   _ptr(out.anchor), _ptr(out.residual), _ptr(out.meta), _stream()),
        "lynx_split_quantize")
    return out


def recombine(planes: Planes, want_codes: bool = True, want_bf16: bool = False):
    """lynx_recombine: returns (codes u8 [...,128] or None, dequantised BF16 [...,128] or None)."""
    r = _fast_recombine(planes, want_codes, want_bf16)
    if r is not None:
        return _result(r, "lynx_recombine")
    lead = tuple(planes.anchor.shape[:-1])
    dev = planes.anchor.device
    codes = torch.empty(lead + (D,), dtype=torch.uint8, device=dev) if want_codes else None
    deq = torch.empty(lead + (D,), dtype=torch.bfloat16, device=dev) if want_bf16 else None
    n_rows = planes.anchor.numel() // 64
    _ok(load().lynx_recombine(_ptr(planes.anchor), _ptr(planes.residual), _ptr(planes.meta), n_rows,
                              _ptr(codes), _ptr(deq), _stream()), "lynx_recombine")
    return codes, deq


@dataclass
class Geometry:
    num_q_heads: int
    num_kv_heads: int
    block_tokens: int
    num_blocks: int
    max_blocks_per_seq: int
    head_dim: int = D

    def _c(self) -> _Shape:
        return _Shape(self.num_q_heads, self.num_kv_heads, self.head_dim, self.block_tokens,
                      self.num_blocks, self.max_blocks_per_seq)


def workspace_bytes(geo: Geometry, batch: int, n_q: int) -> int:
    return int(load().lynx_workspace_bytes(ctypes.byref(geo._c()), batch, n_q))


def make_workspace(geo: Geometry, batch: int, n_q: int, device) -> torch.Tensor:
    """Allocate and zero a workspace large enough for (batch, n_q) attention calls."""
    n = workspace_bytes(geo, batch, n_q)
    if n == 0:
        raise LynxError("unsupported attention shape")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    _ok(load().lynx_workspace_init(_ptr(ws), n, _stream()), "lynx_workspace_init")
    return ws


def check(workspace: torch.Tensor):
    """lynx_check: synchronises and raises if a kernel recorded a bad block id or a timeout."""
    _ok(load().lynx_check(_ptr(workspace), _stream()), "lynx_check")


def anchor_attention(geo: Geometry, q: torch.Tensor, K: Planes, V: Planes, block_table: torch.Tensor,
                     seq_lens: torch.Tensor, workspace: torch.Tensor, causal: bool = False,
                     softmax_scale: float = 0.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """lynx_anchor_attention: q BF16 [B][n_q][Hq][128] -> float32 [B][n_q][Hq][128]."""
    r = _fast_anchor(geo, q, K, V, block_table, seq_lens, workspace, causal, softmax_scale, out)
    if r is not None:
        return _result(r, "lynx_anchor_attention")
    B, n_q, Hq, d = q.shape
    if q.dtype != torch.bfloat16 or d != D or Hq != geo.num_q_heads:
        raise LynxError("q must be BF16 [B][n_q][Hq][128]")
    if out is None:
        out = torch.empty(B, n_q, Hq, D, dtype=torch.float32, device=q.device)
    _ok(load().lynx_anchor_attention(ctypes.byref(geo._c()), _ptr(q), B, n_q, int(causal), K._c(),
                                     V._c(), _ptr(block_table), _ptr(seq_lens), softmax_scale,
                                     _ptr(out), _ptr(workspace), workspace.numel(), _stream()),
        "lynx_anchor_attention")
    return out


def anchor_attention_static(geo: Geometry, q: torch.Tensor, K: Planes, V: Planes,
                            block_table: torch.Tensor, seq_lens: torch.Tensor, causal: bool = False,
                            softmax_scale: float = 0.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """lynx_anchor_attention_static: anchor attention whose scratch memory is a fixed 8 MiB array
    inside the library, for callers that may not allocate a workspace.  Only `out` is allocated
    here when the caller does not pass it; the library call allocates nothing.  Calls share the
    array: keep them ordered on one stream.  Raises LynxError if the problem needs more scratch."""
    B, n_q, Hq, d = q.shape
    if q.dtype != torch.bfloat16 or d != D or Hq != geo.num_q_heads:
        raise LynxError("q must be BF16 [B][n_q][Hq][128]")
    if out is None:
        out = torch.empty(B, n_q, Hq, D, dtype=torch.float32, device=q.device)
    _ok(load().lynx_anchor_attention_static(ctypes.byref(geo._c()), _ptr(q), B, n_q, int(causal),
                                            K._c(), V._c(), _ptr(block_table), _ptr(seq_lens),
                                            softmax_scale, _ptr(out), _stream()),
        "lynx_anchor_attention_static")
    return out


def merge_verify_attention(geo: Geometry, q: torch.Tensor, K: Planes, V: Planes,
                           block_table: torch.Tensor, seq_lens: torch.Tensor, workspace: torch.Tensor,
                           draft_out: torch.Tensor | None = None, atol: float = 0.0, rtol: float = 0.0,
                           causal: bool = True, softmax_scale: float = 0.0,
                           out_full: torch.Tensor | None = None, first_reject: torch.Tensor | None = None,
                           dev: torch.Tensor | None = None):
    """lynx_merge_verify_attention -> (out_full f32 [B][k][Hq][128], first_reject i32 [B], dev f32 [B][k]).
    first_reject / dev are None when no draft is given."""
    r = _fast_verify(geo, q, K, V, block_table, seq_lens, workspace, draft_out, atol, rtol, causal, softmax_scale, out_full,
                     first_reject, dev)
    if r is not None:
        return _result(r, "lynx_merge_verify_attention")
    B, k, Hq, d = q.shape
    if q.dtype != torch.bfloat16 or d != D or Hq != geo.num_q_heads:
        raise LynxError("q must be BF16 [B][k][Hq][128]")
    if out_full is None:
        out_full = torch.empty(B, k, Hq, D, dtype=torch.float32, device=q.device)
    if draft_out is not None:
        if draft_out.dtype != torch.float32 or tuple(draft_out.shape) != (B, k, Hq, D):
            raise LynxError("draft_out must be float32 [B][k][Hq][128]")
        if first_reject is None:
            first_reject = torch.empty(B, dtype=torch.int32, device=q.device)
        if dev is None:
            dev = torch.empty(B, k, dtype=torch.float32, device=q.device)
    _ok(load().lynx_merge_verify_attention(ctypes.byref(geo._c()), _ptr(q), B, k, int(causal), K._c(),
                                           V._c(), _ptr(block_table), _ptr(seq_lens), softmax_scale,
                                           _ptr(draft_out), atol, rtol, _ptr(out_full),
                                           _ptr(first_reject), _ptr(dev), _ptr(workspace),
                                           workspace.numel(), _stream()),
        "lynx_merge_verify_attention")
    return out_full, first_reject, dev


def bf16_attention(geo: Geometry, q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                   block_table: torch.Tensor, seq_lens: torch.Tensor, workspace: torch.Tensor | None = None,
                   causal: bool = False, softmax_scale: float = 0.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """lynx_bf16_attention: decode attention over dequantised BF16 pages [num_blocks][Hkv][bt][128]
    (what recombine(want_bf16=True) writes).  q BF16 [B][n_q][Hq][128] -> float32 [B][n_q][Hq][128]."""
    r = _fast_bf16(geo, q, k_pages, v_pages, block_table, seq_lens, workspace, causal, softmax_scale, out)
    if r is not None:
        return _result(r, "lynx_bf16_attention")
    B, n_q, Hq, d = q.shape
    if q.dtype != torch.bfloat16 or d != D or Hq != geo.num_q_heads:
        raise LynxError("q must be BF16 [B][n_q][Hq][128]")
    if k_pages.dtype != torch.bfloat16 or v_pages.dtype != torch.bfloat16:
        raise LynxError("pages must be BF16")
    if out is None:
        out = torch.empty(B, n_q, Hq, D, dtype=torch.float32, device=q.device)
    if workspace is None:
        n = int(load().lynx_bf16_workspace_bytes(ctypes.byref(geo._c()), B, n_q))
        if n == 0:
            raise LynxError("unsupported attention shape")
        workspace = torch.empty(n, dtype=torch.uint8, device=q.device)
    _ok(load().lynx_bf16_attention(ctypes.byref(geo._c()), _ptr(q), B, n_q, int(causal), _ptr(k_pages),
                                   _ptr(v_pages), _ptr(block_table), _ptr(seq_lens), softmax_scale, _ptr(out),
                                   _ptr(workspace), workspace.numel(), _stream()), "lynx_bf16_attention")
    return out


def _lse_view(addr, workspace: torch.Tensor, B: int, n_q: int, Hq: int, what: str) -> torch.Tensor:
    if not addr:
        raise LynxError(f"{what}: unsupported shape")
    off = int(addr) - workspace.data_ptr()
    n = B * n_q * Hq * 4
    if workspace.dtype != torch.uint8 or off < 0 or off + n > workspace.numel():
        raise LynxError(f"{what}: the workspace is smaller than the call's")
    return workspace[off:off + n].view(torch.float32).view(B, n_q, Hq)


def workspace_lse(geo: Geometry, B: int, n_q: int, workspace: torch.Tensor) -> torch.Tensor:
    """lynx_workspace_lse: float32 [B][n_q][Hq] view, inside `workspace`, of the natural-log log-sum-exps the last
    anchor_attention / merge_verify_attention call with this (B, n_q) left there."""
    r = _fast_lse_view(geo, B, n_q, workspace, False)
    if r is not None:
        return r
    return _lse_view(load().lynx_workspace_lse(ctypes.byref(geo._c()), B, n_q, _ptr(workspace)), workspace, B, n_q,
                     geo.num_q_heads, "lynx_workspace_lse")


def bf16_workspace_lse(geo: Geometry, B: int, n_q: int, workspace: torch.Tensor) -> torch.Tensor:
    """lynx_bf16_workspace_lse: the same for the workspace of a bf16_attention call."""
    r = _fast_lse_view(geo, B, n_q, workspace, True)
    if r is not None:
        return r
    return _lse_view(load().lynx_bf16_workspace_lse(ctypes.byref(geo._c()), B, n_q, _ptr(workspace)), workspace, B,
                     n_q, geo.num_q_heads, "lynx_bf16_workspace_lse")


def lse_merge(out_a: torch.Tensor, lse_a: torch.Tensor, out_b: torch.Tensor, lse_b: torch.Tensor,
              out: torch.Tensor | None = None, want_lse: bool = False):
    """lynx_lse_merge: two attention results float32 [...][128] over disjoint key sets, with their log-sum-exps
    float32 [...], joined into the attention over the union.  Returns out, or (out, lse) with want_lse."""
    r = _fast_lse_merge(out_a, lse_a, out_b, lse_b, out, want_lse)
    if r is not None:
        return _result(r, "lynx_lse_merge")
    if out_a.dtype != torch.float32 or out_b.dtype != torch.float32 or out_a.shape != out_b.shape or out_a.shape[-1] != D:
        raise LynxError("out_a, out_b must be float32 [...][128] of one shape")
    rows = out_a.numel() // D
    if lse_a.dtype != torch.float32 or lse_b.dtype != torch.float32 or lse_a.numel() != rows or lse_b.numel() != rows:
        raise LynxError("lse_a, lse_b must be float32 with one value per row")
    if out is None:
        out = torch.empty_like(out_a)
    lse = torch.empty(out_a.shape[:-1], dtype=torch.float32, device=out_a.device) if want_lse else None
    _ok(load().lynx_lse_merge(_ptr(out_a), _ptr(lse_a), _ptr(out_b), _ptr(lse_b), rows, _ptr(out), _ptr(lse), _stream()),
        "lynx_lse_merge")
    return (out, lse) if want_lse else out


def split_quantize_bits(src: torch.Tensor, anchor_bits: int):
    """lynx_split_quantize_bits: src BF16 [...][128] -> (anchor u8 [...][16 A], residual u8 [...][16 (8 - A)],
    meta f32 [...][2]) for the split with A = anchor_bits top bits in the Anchor."""
    if src.dtype != torch.bfloat16 or src.shape[-1] != D:
        raise LynxError("src must be BF16 [...][128]")
    lead, rows = tuple(src.shape[:-1]), src.numel() // D
    anchor = torch.empty(lead + (16 * anchor_bits,), dtype=torch.uint8, device=src.device)
    residual = torch.empty(lead + (16 * (8 - anchor_bits),), dtype=torch.uint8, device=src.device)
    meta = torch.empty(lead + (2,), dtype=torch.float32, device=src.device)
    _ok(load().lynx_split_quantize_bits(_ptr(src), rows, anchor_bits, _ptr(anchor), _ptr(residual), _ptr(meta), _stream()),
        "lynx_split_quantize_bits")
    return anchor, residual, meta


def recombine_bits(anchor: torch.Tensor, residual: torch.Tensor | None, meta: torch.Tensor, anchor_bits: int,
                   want_codes: bool = True, want_bf16: bool = True):
    """lynx_recombine_bits -> (codes u8 [...][128] or None, dequantised BF16 [...][128] or None); residual None:
    the Anchor alone (bucket mid-points)."""
    lead, rows = tuple(anchor.shape[:-1]), anchor.numel() // (16 * anchor_bits)
    codes = torch.empty(lead + (D,), dtype=torch.uint8, device=anchor.device) if want_codes else None
    deq = torch.empty(lead + (D,), dtype=torch.bfloat16, device=anchor.device) if want_bf16 else None
    _ok(load().lynx_recombine_bits(_ptr(anchor), _ptr(residual), _ptr(meta), rows, anchor_bits, _ptr(codes), _ptr(deq),
                                   _stream()), "lynx_recombine_bits")
    return codes, deq


def verify_decision(out_full: torch.Tensor, draft_out: torch.Tensor, atol: float, rtol: float):
    """lynx_verify_decision: out_full, draft_out float32 [B][k][Hq][128] -> (first_reject i32 [B], dev f32 [B][k])."""
    if out_full.dtype != torch.float32 or draft_out.dtype != torch.float32 or out_full.shape != draft_out.shape \
            or out_full.dim() != 4 or out_full.shape[-1] != D:
        raise LynxError("out_full, draft_out must be float32 [B][k][Hq][128]")
    B, k, Hq, _ = out_full.shape
    first_reject = torch.empty(B, dtype=torch.int32, device=out_full.device)
    dev = torch.empty(B, k, dtype=torch.float32, device=out_full.device)
    _ok(load().lynx_verify_decision(_ptr(out_full), _ptr(draft_out), B, k, Hq, atol, rtol, _ptr(first_reject), _ptr(dev),
                                    _stream()), "lynx_verify_decision")
    return first_reject, dev


@dataclass
class HierPlanes:
    """Algorithm 1 output for pages of 256 tokens: packed nibbles and the per-channel metadata."""
    q_anc: torch.Tensor        # u8 [n_pages][256][64]
    q_res: torch.Tensor        # u8 [n_pages][256][64]
    gamma_min: torch.Tensor    # f32 [n_pages][128]
    gamma_scale: torch.Tensor  # f32 [n_pages][128]
    mu: torch.Tensor           # f32 [n_pages][8][128]
    sigma: torch.Tensor        # f32 [n_pages][8][128]


def hier_quantize(src: torch.Tensor) -> HierPlanes:
    """lynx_hier_quantize: src BF16 [n_pages][256][128] -> HierPlanes."""
    r = _fast_hier_quantize(src)
    if r is not None:
        return HierPlanes(*_result(r, "lynx_hier_quantize"))
    if src.dtype != torch.bfloat16 or src.dim() != 3 or tuple(src.shape[1:]) != (256, D):
        raise LynxError("src must be BF16 [n_pages][256][128]")
    n, dev = src.shape[0], src.device
    out = HierPlanes(torch.empty(n, 256, 64, dtype=torch.uint8, device=dev), torch.empty(n, 256, 64, dtype=torch.uint8, device=dev),
                     torch.empty(n, D, dtype=torch.float32, device=dev), torch.empty(n, D, dtype=torch.float32, device=dev),
                     torch.empty(n, 8, D, dtype=torch.float32, device=dev), torch.empty(n, 8, D, dtype=torch.float32, device=dev))
    _ok(load().lynx_hier_quantize(_ptr(src), n, _ptr(out.q_anc), _ptr(out.q_res), _ptr(out.gamma_min),
                                  _ptr(out.gamma_scale), _ptr(out.mu), _ptr(out.sigma), _stream()), "lynx_hier_quantize")
    return out


def hier_dequantize(h: HierPlanes, anchor_only: bool = False, out: torch.Tensor | None = None) -> torch.Tensor:
    """lynx_hier_dequantize -> BF16 [n_pages][256][128] (from the Anchor stream alone if asked)."""
    r = _fast_hier_dequantize(h.q_anc, None if anchor_only else h.q_res, h.gamma_min, h.gamma_scale, h.mu, h.sigma, out)
    if r is not None:
        return _result(r, "lynx_hier_dequantize")
    n = h.q_anc.shape[0]
    if out is None:
        out = torch.empty(n, 256, D, dtype=torch.bfloat16, device=h.q_anc.device)
    _ok(load().lynx_hier_dequantize(_ptr(h.q_anc), None if anchor_only else _ptr(h.q_res), n, _ptr(h.gamma_min),
                                    _ptr(h.gamma_scale), _ptr(h.mu), _ptr(h.sigma), _ptr(out), _stream()),
        "lynx_hier_dequantize")
    return out


def token_verify(p_probs: torch.Tensor, q_probs: torch.Tensor, draft_tokens: torch.Tensor, u: torch.Tensor,
                 r: torch.Tensor):
    """lynx_token_verify: p_probs f32 [B][k][V], q_probs f32 [B][k+1][V], draft_tokens i32 [B][k], u f32 [B][k],
    r f32 [B] -> (n_accepted i32 [B], next_token i32 [B])."""
    B, k, V = p_probs.shape
    if tuple(q_probs.shape) != (B, k + 1, V) or p_probs.dtype != torch.float32 or q_probs.dtype != torch.float32:
        raise LynxError("p_probs must be float32 [B][k][V], q_probs float32 [B][k+1][V]")
    if draft_tokens.dtype != torch.int32 or tuple(draft_tokens.shape) != (B, k):
        raise LynxError("draft_tokens must be int32 [B][k]")
    if u.dtype != torch.float32 or tuple(u.shape) != (B, k) or r.dtype != torch.float32 or tuple(r.shape) != (B,):
        raise LynxError("u must be float32 [B][k], r float32 [B]")
    for t in (p_probs, q_probs, draft_tokens, u, r):
        if not t.is_contiguous():
            raise LynxError("contiguous tensors required")
    n_acc = torch.empty(B, dtype=torch.int32, device=p_probs.device)
    nxt = torch.empty(B, dtype=torch.int32, device=p_probs.device)
    _ok(load().lynx_token_verify(_ptr(p_probs), _ptr(q_probs), _ptr(draft_tokens), _ptr(u), _ptr(r), B, k, V,
                                 _ptr(n_acc), _ptr(nxt), _stream()), "lynx_token_verify")
    return n_acc, nxt


# ---------------------------------------------------------------------------------------------- around the cache
_AXES = [bytes(range(n)) for n in range(257)]   # (the numbers of n axes)


@dataclass(frozen=True, init=False)
class Rotary:
    """Rotary positions: positions i32 [T] or [axes][T], cos_sin f32 [n_positions][2 P] (P cosines, P sines; P = 8, 16, ... 64
    pairs of channels), pair_axis: the axis of each pair (P ints; None: one axis).  Pairs are channels (i, i + P), or
    (2 i, 2 i + 1) if interleaved.  Made once per table and step, and used by any number of calls."""
    positions: torch.Tensor
    cos_sin: torch.Tensor
    pair_axis: tuple | list | None = None
    interleaved: bool = False

    def __init__(self, positions: torch.Tensor, cos_sin: torch.Tensor, pair_axis: tuple | list | None = None, interleaved: bool = False):
        # (made in every step of a decode loop: 1.9 us, 3.7 with the dataclass's own __init__ and checks of each pair in turn)
        shape = positions.shape
        if positions.dtype != torch.int32 or len(shape) not in (1, 2):
            raise LynxError("positions must be int32 [tokens] or [axes][tokens]")
        if cos_sin.dtype != torch.float32 or cos_sin.dim() != 2 or cos_sin.shape[1] % 2:
            raise LynxError("cos_sin must be float32 [positions][2 pairs]")
        axes, pairs = 1 if len(shape) == 1 else shape[0], cos_sin.shape[1] // 2
        try:
            axis = bytes(pairs) if pair_axis is None else bytes(pair_axis)
        except ValueError:   # (a number that is none of a byte)
            axis = b""
        if len(axis) != pairs or pairs > 64 or axis.translate(None, _AXES[min(axes, 256)]):
            raise LynxError("pair_axis must name one of the positions' axes for each pair, of at most 64")
        self.__dict__.update(positions=positions, cos_sin=cos_sin, pair_axis=pair_axis, interleaved=interleaved, _axis=axis)

    def _c(self, tokens: int):
        pos, table = self.positions, self.cos_sin
        if pos.shape[-1] < tokens:
            raise LynxError("positions must be int32 [tokens] or [axes][tokens]")
        return ctypes.byref(_RotarySpec(_ptr(pos), _ptr(table), pos.shape[-1], 1 if pos.dim() == 1 else pos.shape[0], table.shape[0],
                                        len(self._axis), int(self.interleaved), (ctypes.c_uint8 * 64)(*self._axis)))


def rotary_table(n_positions: int, pairs: int = 64, base: float = 10000.0, device=None) -> torch.Tensor:
    """A cos_sin table f32 [n_positions][2 pairs] of angles position * base^(-i / pairs), computed in 64 bits."""
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * \
        float(base) ** (-torch.arange(pairs, dtype=torch.float64, device=device) / pairs)
    return torch.cat((angle.cos(), angle.sin()), 1).float()


def _token_rows(t: torch.Tensor, what: str, width: int = D):
    """Pointer, token stride and heads of BF16 [tokens][heads][width] whose tokens may lie apart (a view of a fused projection)."""
    if t.dtype != torch.bfloat16 or t.dim() != 3 or t.shape[2] != width:
        raise LynxError(f"{what} must be BF16 [tokens][heads][{width}]")
    if not t.is_cuda:
        raise LynxError("device tensors required")
    T, H = t.shape[:2]
    if T and (t.stride(2) != 1 or (H > 1 and t.stride(1) != width)):
        raise LynxError(f"{what}: the heads of a token must lie one behind the other")
    return t.data_ptr(), t.stride(0) if T > 1 else H * width, H


def rotary(q: torch.Tensor | None, k: torch.Tensor | None, spec: Rotary, q_out: torch.Tensor | None = None,
           k_out: torch.Tensor | None = None):
    """lynx_rotary: q BF16 [T][Hq][128], k BF16 [T][Hkv][128] (either may be None; tokens may lie apart) -> (q_out, k_out), which may
    be the inputs."""
    r = _fast_rotary(q, k, spec, q_out, k_out)
    if r is not None:
        return _result(r, "lynx_rotary")
    if q is None and k is None:
        raise LynxError("q or k is needed")
    T = (q if q is not None else k).shape[0]
    rows = []
    for x, out, what in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None:
            rows.append((None, (None, 0, 0), (None, 0, 0)))
            continue
        if x.shape[0] != T or (out is not None and out.shape != x.shape):
            raise LynxError("q and k must have as many tokens, and the outputs their shapes")
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rows.append((out, _token_rows(x, what), _token_rows(out, what + "_out")))
    (qo, qi, qw), (ko, ki, kw) = rows
    _ok(load().lynx_rotary(spec._c(T), qi[0], qi[1], qi[2], ki[0], ki[1], ki[2], T, qw[0], qw[1], kw[0], kw[1], _stream()), "lynx_rotary")
    return qo, ko


def _here(*tensors):
    """Tensors (and planes) of a call must be on the current device, whose stream it uses."""
    for t in tensors:
        if isinstance(t, Planes):
            _here(t.anchor, t.residual, t.meta)
        elif isinstance(t, Rotary):
            _here(t.positions, t.cos_sin)
        elif isinstance(t, HeadNorm):
            _here(t.q_weight, t.k_weight)
        elif t is not None:
            if not t.is_cuda:
                raise LynxError("device tensors required")
            if t.device.index != torch.cuda.current_device():
                raise LynxError("tensors must be on the current device")


@dataclass(frozen=True)
class HeadNorm:
    """Norms of heads, y = x / sqrt(mean x^2 + eps) * weight: weights BF16 or float32 (both alike) of as many values as a head has channels.  A
    tensor whose weight is None is not normed."""
    q_weight: torch.Tensor | None = None
    k_weight: torch.Tensor | None = None
    eps: float = 1e-6

    def __post_init__(self):
        given = [w for w in (self.q_weight, self.k_weight) if w is not None]
        if any(w.dim() != 1 or w.dtype not in (torch.bfloat16, torch.float32) or w.dtype != given[0].dtype or w.shape != given[0].shape for w in given):
            raise LynxError("a norm's weights must be BF16 or float32 [channels of a head], both alike")
        object.__setattr__(self, "eps", float(self.eps))
        if not self.eps >= 0.0:
            raise LynxError("eps must be at least 0")

    def _c(self, width: int):
        some = self.k_weight if self.q_weight is None else self.q_weight
        if some is not None and some.shape[0] != width:
            raise LynxError(f"the norm's weights must be {width} values, as a head has channels")
        return ctypes.byref(_HeadNorm(_ptr(self.q_weight), _ptr(self.k_weight), self.eps, int(some is not None and some.dtype == torch.float32)))


def norm_rotary(q: torch.Tensor | None, k: torch.Tensor | None, norm: HeadNorm | None = None, spec: Rotary | None = None,
                q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """lynx_norm_rotary: q BF16 [T][Hq][W], k BF16 [T][Hkv][W], W = 64, 128 or 256 (either may be None; tokens may lie apart, the heads of a token
    not), each head normed and turned (128 channels of it at most) in one pass -> (q_out, k_out), which may be the inputs.  norm or spec None:
    that part is left out."""
    r = _fast_norm_rotary(q, k, norm, spec, q_out, k_out)
    if r is not None:
        return _result(r, "lynx_norm_rotary")
    if q is None and k is None:
        raise LynxError("q or k is needed")
    some = q if q is not None else k
    T, width = some.shape[0], some.shape[-1]
    if width not in (64, 128, 256):
        raise LynxError("heads must have 64, 128 or 256 channels")
    rows = []
    for x, out, what in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None:
            rows.append((None, (None, 0, 0), (None, 0, 0)))
            continue
        if x.shape[0] != T or (out is not None and out.shape != x.shape):
            raise LynxError("q and k must have as many tokens, and the outputs their shapes")
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rows.append((out, _token_rows(x, what, width), _token_rows(out, what + "_out", width)))
    _here(q, k, q_out, k_out, norm, spec)
    (qo, qi, qw), (ko, ki, kw) = rows
    _ok(load().lynx_norm_rotary(None if norm is None else norm._c(width), None if spec is None else spec._c(T), width, qi[0], qi[1], qi[2], ki[0],
                                ki[1], ki[2], T, qw[0], qw[1], kw[0], kw[1], _stream()), "lynx_norm_rotary")
    return qo, ko


def _planes_fit(geo: Geometry, *planes: Planes):
    rows = geo.num_blocks * geo.num_kv_heads * geo.block_tokens
    for p in planes:
        if p.anchor.dtype != torch.uint8 or p.anchor.numel() < rows * 64 or p.meta.dtype != torch.float32 or p.meta.numel() < rows * 2 or \
                (p.residual is not None and (p.residual.dtype != torch.uint8 or p.residual.numel() < rows * 64)):
            raise LynxError("planes must be u8 [num_blocks][Hkv][block_tokens][64] and f32 [...][2] of the geometry")


def cache_append(geo: Geometry, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, K: Planes, V: Planes,
                 rows: torch.Tensor | None = None, rotary: Rotary | None = None, norm: HeadNorm | None = None):
    """lynx_cache_append, with a norm lynx_norm_cache_append: quantises tokens' keys and values BF16 [T][Hkv][128] (tokens may lie apart) into the planes K and V.  slots
    i64 [n]: block * block_tokens + offset of each token written, negative for none; rows i32 [n]: the source row of each
    (None: row i); norm: its k_weight norms the keys first; rotary: positions for the keys, by source row."""
    r = _fast_cache_append(geo, k, v, slots, K, V, rows, rotary) if norm is None else \
        _fast_norm_append(geo, k, v, slots, K, V, rows, rotary, norm)
    if r is not None:
        return _ok(r, "lynx_cache_append" if norm is None else "lynx_norm_cache_append")
    (kp, ks, kh), (vp, vs, vh) = _token_rows(k, "k"), _token_rows(v, "v")
    if kh != geo.num_kv_heads or vh != kh or v.shape[0] != k.shape[0]:
        raise LynxError("k and v must be BF16 [tokens][num_kv_heads][128]")
    if slots.dtype != torch.int64 or slots.dim() != 1 or (rows is not None and (rows.dtype != torch.int32 or rows.shape != slots.shape)):
        raise LynxError("slots must be int64 [n], rows int32 [n]")
    _planes_fit(geo, K, V)
    T = k.shape[0]
    if norm is not None:
        _here(k, v, slots, rows, K, V, rotary, norm)
        return _ok(load().lynx_norm_cache_append(ctypes.byref(geo._c()), kp, ks, vp, vs, T, _ptr(rows), slots.numel(), _ptr(slots),
                                                 norm._c(D), None if rotary is None else rotary._c(T), K._c(), V._c(), _stream()),
                   "lynx_norm_cache_append")
    _ok(load().lynx_cache_append(ctypes.byref(geo._c()), kp, ks, vp, vs, T, _ptr(rows), slots.numel(), _ptr(slots),
                                 None if rotary is None else rotary._c(T), K._c(), V._c(), _stream()), "lynx_cache_append")


def cache_read(geo: Geometry, K: Planes, V: Planes, block_table: torch.Tensor, starts: torch.Tensor | None, offsets: torch.Tensor,
               n_rows: int, anchor_only: bool = False, k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None):
    """lynx_cache_read: tokens [starts[b], starts[b] + offsets[b + 1] - offsets[b]) of each sequence (starts i32 [B] or None for 0,
    offsets i32 [B + 1], n_rows = offsets[B]) -> k, v BF16 [n_rows][Hkv][128], from the full codes or from the Anchor alone."""
    r = _fast_cache_read(geo, K, V, block_table, starts, offsets, n_rows, anchor_only, k_out, v_out)
    if r is not None:
        return _result(r, "lynx_cache_read")
    B = block_table.shape[0]
    if block_table.dtype != torch.int32 or tuple(block_table.shape) != (B, geo.max_blocks_per_seq):
        raise LynxError("block_table must be int32 [B][max_blocks_per_seq]")
    if offsets.dtype != torch.int32 or tuple(offsets.shape) != (B + 1,) or \
            (starts is not None and (starts.dtype != torch.int32 or tuple(starts.shape) != (B,))):
        raise LynxError("offsets must be int32 [B + 1], starts int32 [B]")
    _planes_fit(geo, K, V)
    if not anchor_only and (K.residual is None or V.residual is None):
        raise LynxError("the Residual planes are needed unless anchor_only")
    shape = (n_rows, geo.num_kv_heads, D)
    outs = []
    for o in (k_out, v_out):
        if o is None:
            o = torch.empty(shape, dtype=torch.bfloat16, device=block_table.device)
        elif o.dtype != torch.bfloat16 or tuple(o.shape) != shape:
            raise LynxError("k_out, v_out must be BF16 [n_rows][num_kv_heads][128]")
        outs.append(o)
    planes = [_Plane(_ptr(p.anchor), None if anchor_only else _ptr(p.residual), _ptr(p.meta)) for p in (K, V)]
    _ok(load().lynx_cache_read(ctypes.byref(geo._c()), planes[0], planes[1], _ptr(block_table), B, _ptr(starts), _ptr(offsets), n_rows,
                               _ptr(outs[0]), _ptr(outs[1]), _stream()), "lynx_cache_read")
    return outs[0], outs[1]


@dataclass
class BlockPool:
    """Free blocks of a cache: ring i32 [num_blocks], state i32 [4] = {place of the first free block, number of free blocks, 0, 0}."""
    ring: torch.Tensor
    state: torch.Tensor


def make_block_pool(num_blocks: int, device) -> BlockPool:
    """All blocks free, in order."""
    return BlockPool(torch.arange(num_blocks, dtype=torch.int32, device=device),
                     torch.tensor([0, num_blocks, 0, 0], dtype=torch.int32, device=device))


class BlockPlan(NamedTuple):
    lens: torch.Tensor         # i32 [B] the length that each request has now
    offsets: torch.Tensor      # i32 [B + 1] first row of each request's new tokens
    slots: torch.Tensor        # i64 [max_tokens]
    positions: torch.Tensor    # i32 [max_tokens]


def plan_blocks(geo: Geometry, pool: BlockPool, block_table: torch.Tensor, old_lens: torch.Tensor, new_lens: torch.Tensor,
                max_tokens: int) -> BlockPlan:
    """lynx_plan_blocks: requests of old_lens i32 [B] tokens are to have new_lens i32 [B]; block_table i32 [B][max_blocks_per_seq] and the pool
    are brought up to date, and each new token gets its slot (for cache_append) and position (for Rotary); starts of a cache_read are old_lens."""
    r = _fast_plan_blocks(geo, pool.ring, pool.state, block_table, old_lens, new_lens, max_tokens)
    if r is not None:
        return BlockPlan(*_result(r, "lynx_plan_blocks"))
    B = block_table.shape[0]
    if block_table.dtype != torch.int32 or tuple(block_table.shape) != (B, geo.max_blocks_per_seq):
        raise LynxError("block_table must be int32 [B][max_blocks_per_seq]")
    if any(x.dtype != torch.int32 or tuple(x.shape) != (B,) for x in (old_lens, new_lens)):
        raise LynxError("old_lens, new_lens must be int32 [B]")
    if pool.ring.dtype != torch.int32 or tuple(pool.ring.shape) != (geo.num_blocks,) or pool.state.dtype != torch.int32 or \
            tuple(pool.state.shape) != (4,):
        raise LynxError("the pool must be int32 [num_blocks] and int32 [4]")
    if max_tokens < 0:
        raise LynxError("max_tokens must be at least 0")
    _here(block_table, old_lens, new_lens, pool.ring, pool.state)
    dev = block_table.device
    out = BlockPlan(torch.empty(B, dtype=torch.int32, device=dev), torch.empty(B + 1, dtype=torch.int32, device=dev),
                    torch.empty(max_tokens, dtype=torch.int64, device=dev), torch.empty(max_tokens, dtype=torch.int32, device=dev))
    _ok(load().lynx_plan_blocks(ctypes.byref(geo._c()), _ptr(old_lens), _ptr(new_lens), B, _ptr(block_table), _ptr(pool.ring), _ptr(pool.state),
                                max_tokens, _ptr(out.lens), _ptr(out.offsets), _ptr(out.slots), _ptr(out.positions), _stream()),
        "lynx_plan_blocks")
    return out


# ---------------------------------------------------------------------------------------------- caches of latents
LATENT, ROPE = 512, 64


def _latent_rows(t: torch.Tensor, width: int, what: str):
    """Pointer and token stride of BF16 [tokens][width] whose tokens may lie apart."""
    if t.dtype != torch.bfloat16 or t.dim() != 2 or t.shape[1] != width:
        raise LynxError(f"{what} must be BF16 [tokens][{width}]")
    return _token_rows(t[:, None], what, width)[:2]


def _latent_fit(geo: Geometry, C: Planes, pages: torch.Tensor):
    if geo.num_kv_heads != 4:
        raise LynxError("a latent is four rows of the planes: num_kv_heads must be 4")
    _planes_fit(geo, C)
    if pages.dtype != torch.bfloat16 or pages.numel() < geo.num_blocks * geo.block_tokens * ROPE:
        raise LynxError("rope_pages must be BF16 [num_blocks][block_tokens][64]")


def latent_append(geo: Geometry, latents: torch.Tensor, rope_keys: torch.Tensor, slots: torch.Tensor, C: Planes, rope_pages: torch.Tensor,
                  weight: torch.Tensor | None = None, eps: float = 1e-6, rows: torch.Tensor | None = None, rotary: Rotary | None = None):
    """lynx_latent_append: tokens' latents BF16 [T][512] (normed with weight BF16 or float32 [512], where given) into the planes C of a geometry with
    num_kv_heads = 4, and rotary keys BF16 [T][64] (turned, where rotary is given) into rope_pages BF16 [num_blocks][block_tokens][64].  slots and
    rows as for cache_append."""
    eps = float(eps)
    r = _fast_latent_append(geo, latents, rope_keys, slots, C, rope_pages, weight, eps, rows, rotary)
    if r is not None:
        return _ok(r, "lynx_latent_append")
    (cp, cs), (kp, ks) = _latent_rows(latents, LATENT, "latents"), _latent_rows(rope_keys, ROPE, "rope_keys")
    T = latents.shape[0]
    if rope_keys.shape[0] != T:
        raise LynxError("latents and rope_keys must have as many tokens")
    if slots.dtype != torch.int64 or slots.dim() != 1 or (rows is not None and (rows.dtype != torch.int32 or rows.shape != slots.shape)):
        raise LynxError("slots must be int64 [n], rows int32 [n]")
    if weight is not None and (weight.dtype not in (torch.bfloat16, torch.float32) or tuple(weight.shape) != (LATENT,)):
        raise LynxError("weight must be BF16 or float32 [512]")
    _latent_fit(geo, C, rope_pages)
    _here(latents, rope_keys, slots, C, rope_pages, weight, rows, rotary)
    _ok(load().lynx_latent_append(ctypes.byref(geo._c()), cp, cs, kp, ks, T, _ptr(rows), slots.numel(), _ptr(slots), _ptr(weight),
                                  int(weight is not None and weight.dtype == torch.float32), eps, None if rotary is None else rotary._c(T), C._c(),
                                  _ptr(rope_pages), _stream()), "lynx_latent_append")


def latent_read(geo: Geometry, C: Planes, rope_pages: torch.Tensor, block_table: torch.Tensor, starts: torch.Tensor | None, offsets: torch.Tensor,
                n_rows: int, anchor_only: bool = False):
    """lynx_latent_read: ranges of tokens as cache_read's -> latents BF16 [n_rows][512], rotary keys BF16 [n_rows][64]."""
    r = _fast_latent_read(geo, C, rope_pages, block_table, starts, offsets, n_rows, anchor_only)
    if r is not None:
        return _result(r, "lynx_latent_read")
    B = block_table.shape[0]
    if block_table.dtype != torch.int32 or tuple(block_table.shape) != (B, geo.max_blocks_per_seq):
        raise LynxError("block_table must be int32 [B][max_blocks_per_seq]")
    if offsets.dtype != torch.int32 or tuple(offsets.shape) != (B + 1,) or \
            (starts is not None and (starts.dtype != torch.int32 or tuple(starts.shape) != (B,))):
        raise LynxError("offsets must be int32 [B + 1], starts int32 [B]")
    _latent_fit(geo, C, rope_pages)
    if not anchor_only and C.residual is None:
        raise LynxError("the Residual plane is needed unless anchor_only")
    if n_rows < 0:
        raise LynxError("n_rows must be at least 0")
    _here(C, rope_pages, block_table, starts, offsets)
    out = torch.empty(n_rows, LATENT, dtype=torch.bfloat16, device=block_table.device)
    keys = torch.empty(n_rows, ROPE, dtype=torch.bfloat16, device=block_table.device)
    plane = _Plane(_ptr(C.anchor), None if anchor_only else _ptr(C.residual), _ptr(C.meta))
    _ok(load().lynx_latent_read(ctypes.byref(geo._c()), plane, _ptr(rope_pages), _ptr(block_table), B, _ptr(starts), _ptr(offsets), n_rows,
                                _ptr(out), _ptr(keys), _stream()), "lynx_latent_read")
    return out, keys


def latent_workspace_bytes(geo: Geometry, batch: int, n_q: int) -> int:
    return int(load().lynx_latent_workspace_bytes(ctypes.byref(geo._c()), batch, n_q))


def make_latent_workspace(geo: Geometry, batch: int, n_q: int, device) -> torch.Tensor:
    """Allocate a workspace for latent_attention calls of up to (batch, n_q) and zero it."""
    n = latent_workspace_bytes(geo, batch, n_q)
    if n == 0:
        raise LynxError("unsupported latent attention shape")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    _ok(load().lynx_workspace_init(_ptr(ws), n, _stream()), "lynx_workspace_init")
    return ws


def _query_rows(t: torch.Tensor, shape: tuple, what: str):
    """Pointer and row stride of BF16 [B][n][Hq][width] whose rows may lie apart, evenly."""
    if t.dtype != torch.bfloat16 or tuple(t.shape) != shape:
        raise LynxError(f"{what} must be BF16 [B][n_q][Hq][{shape[-1]}]")
    if not t.is_cuda:
        raise LynxError("device tensors required")
    apart, rows = None, 1
    for d in (2, 1, 0):
        if t.shape[d] > 1:      # (of dimensions with one entry the stride means nothing)
            if apart is None:
                apart = t.stride(d)
            elif t.stride(d) != apart * rows:
                raise LynxError(f"{what}: rows must lie evenly apart")
            rows *= t.shape[d]
    if t.stride(3) != 1:
        raise LynxError(f"{what}: the channels of a row must lie one behind the other")
    return t.data_ptr(), shape[-1] if apart is None else apart


def latent_attention(geo: Geometry, q_latent: torch.Tensor, q_rope: torch.Tensor, C: Planes, rope_pages: torch.Tensor, block_table: torch.Tensor,
                     seq_lens: torch.Tensor, workspace: torch.Tensor, causal: bool = True, anchor_only: bool = False, softmax_scale: float = 0.0,
                     out: torch.Tensor | None = None, lse: torch.Tensor | None = None) -> torch.Tensor:
    """lynx_latent_attention: q_latent BF16 [B][n][Hq][512] and q_rope BF16 [B][n][Hq][64] (rows may lie apart, evenly: views of one [..][576]) over
    the latents of a geometry with num_kv_heads = 4 -> BF16 [B][n][Hq][512], or what `out` (BF16 or float32) is; lse: float32 [B][n][Hq] to be filled.
    anchor_only: the Anchor's state of the planes.  softmax_scale 0: 1 / sqrt(192)."""
    r = _fast_latent_attention(geo, q_latent, q_rope, C, rope_pages, block_table, seq_lens, workspace, causal, anchor_only, softmax_scale, out, lse)
    if r is not None:
        return _result(r, "lynx_latent_attention")
    if q_latent.dim() != 4 or q_latent.dtype != torch.bfloat16 or q_latent.shape[2:] != (geo.num_q_heads, LATENT):
        raise LynxError("q_latent must be BF16 [B][n_q][Hq][512]")
    B, n, Hq, _ = q_latent.shape
    if block_table.dtype != torch.int32 or tuple(block_table.shape) != (B, geo.max_blocks_per_seq) or seq_lens.dtype != torch.int32 or \
            tuple(seq_lens.shape) != (B,):
        raise LynxError("block_table must be int32 [B][max_blocks_per_seq], seq_lens int32 [B]")
    if out is None:
        out = torch.empty(q_latent.shape, dtype=torch.bfloat16, device=q_latent.device)
    elif out.shape != q_latent.shape or out.dtype not in (torch.bfloat16, torch.float32):
        raise LynxError("out must be BF16 or float32 [B][n_q][Hq][512]")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (B, n, Hq)):
        raise LynxError("lse must be float32 [B][n_q][Hq]")
    if not anchor_only and C.residual is None:
        raise LynxError("the Residual plane is needed unless anchor_only")
    _latent_fit(geo, C, rope_pages)
    if B == 0:
        return out
    (qp, qs), (rp, rs) = _query_rows(q_latent, (B, n, Hq, LATENT), "q_latent"), _query_rows(q_rope, (B, n, Hq, ROPE), "q_rope")
    _here(q_latent, q_rope, C, rope_pages, block_table, seq_lens, workspace, out, lse)
    plane = _Plane(_ptr(C.anchor), None if anchor_only else _ptr(C.residual), _ptr(C.meta))
    _ok(load().lynx_latent_attention(ctypes.byref(geo._c()), qp, qs, rp, rs, B, n, int(causal), plane, _ptr(rope_pages), _ptr(block_table),
                                     _ptr(seq_lens), softmax_scale, int(out.dtype == torch.float32), _ptr(out), _ptr(lse), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream()), "lynx_latent_attention")
    return out


def tree_workspace_bytes(geo: Geometry, batch: int, n_nodes: int) -> int:
    return int(load().lynx_tree_workspace_bytes(ctypes.byref(geo._c()), batch, n_nodes))


def make_tree_workspace(geo: Geometry, batch: int, n_nodes: int, device) -> torch.Tensor:
    """Allocate a workspace for tree_attention calls of up to (batch, n_nodes) and zero it."""
    n = tree_workspace_bytes(geo, batch, n_nodes)
    if n == 0:
        raise LynxError("unsupported tree attention shape")
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    _ok(load().lynx_workspace_init(_ptr(ws), n, _stream()), "lynx_workspace_init")
    return ws


def _nodes(t: torch.Tensor, B: int, n: int, H: int, what: str):
    """Pointer and node stride of BF16 [B][n][Hkv][128] whose nodes may lie apart, evenly."""
    if t.dtype != torch.bfloat16 or tuple(t.shape) != (B, n, H, D):
        raise LynxError(f"{what} must be BF16 [B][n][Hkv][128]")
    if n > 1 and B > 1 and t.stride(0) != n * t.stride(1):
        raise LynxError(f"{what}: nodes must lie evenly apart")
    p, stride, _ = _token_rows(t[:, 0] if n == 1 else t[0], what)
    return p, stride


def tree_attention(geo: Geometry, q: torch.Tensor, K: Planes, V: Planes, block_table: torch.Tensor, seq_lens: torch.Tensor,
                   k_nodes: torch.Tensor, v_nodes: torch.Tensor, tree_mask: torch.Tensor, workspace: torch.Tensor,
                   anchor_only: bool = False, softmax_scale: float = 0.0, out: torch.Tensor | None = None,
                   lse: torch.Tensor | None = None) -> torch.Tensor:
    """lynx_tree_attention: q BF16 [B][n][Hq][128] of a tree's nodes over the planes' tokens [0, seq_lens[b]) and the nodes i with bit i
    of tree_mask i64 [B][n]; k_nodes, v_nodes BF16 [B][n][Hkv][128] (nodes may lie apart).  -> BF16 [B][n][Hq][128], or what `out`
    (BF16 or float32) is; lse: float32 [B][n][Hq] to be filled.  anchor_only: the Anchor's state of the planes."""
    r = _fast_tree_attention(geo, q, K, V, block_table, seq_lens, k_nodes, v_nodes, tree_mask, workspace, anchor_only, softmax_scale, out, lse)
    if r is not None:
        return _result(r, "lynx_tree_attention")
    if q.dim() != 4 or q.dtype != torch.bfloat16 or q.shape[2:] != (geo.num_q_heads, D):
        raise LynxError("q must be BF16 [B][n][Hq][128]")
    B, n, Hq, _ = q.shape
    if block_table.dtype != torch.int32 or tuple(block_table.shape) != (B, geo.max_blocks_per_seq) or seq_lens.dtype != torch.int32 or \
            tuple(seq_lens.shape) != (B,):
        raise LynxError("block_table must be int32 [B][max_blocks_per_seq], seq_lens int32 [B]")
    if tree_mask.dtype != torch.int64 or tuple(tree_mask.shape) != (B, n):
        raise LynxError("tree_mask must be int64 [B][n]")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.dtype not in (torch.bfloat16, torch.float32):
        raise LynxError("out must be BF16 or float32 [B][n][Hq][128]")
    if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (B, n, Hq)):
        raise LynxError("lse must be float32 [B][n][Hq]")
    if not anchor_only and (K.residual is None or V.residual is None):
        raise LynxError("the Residual planes are needed unless anchor_only")
    _planes_fit(geo, K, V)
    if B == 0:
        return out
    (kp, ks), (vp, vs) = _nodes(k_nodes, B, n, geo.num_kv_heads, "k_nodes"), _nodes(v_nodes, B, n, geo.num_kv_heads, "v_nodes")
    planes = [_Plane(_ptr(p.anchor), None if anchor_only else _ptr(p.residual), _ptr(p.meta)) for p in (K, V)]
    _ok(load().lynx_tree_attention(ctypes.byref(geo._c()), _ptr(q), B, n, planes[0], planes[1], _ptr(block_table), _ptr(seq_lens), kp, ks,
                                   vp, vs, _ptr(tree_mask), softmax_scale, int(out.dtype == torch.float32), _ptr(out), _ptr(lse),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(), _stream()), "lynx_tree_attention")
    return out
