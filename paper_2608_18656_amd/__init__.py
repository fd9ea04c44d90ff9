"""MI355X (gfx950) FlashAttention forward: MHA / GQA / MQA, prefill and decode.

Thin Python layer over the C ABI in include/fa.h (see ``_lib``); PyTorch is
used only for device memory and the current HIP stream.  Import is cheap: the
HIP library is loaded on first use and its absence raises (no CPU fallback).
"""
from __future__ import annotations

import ctypes
import math
import operator

from . import _lib

__all__ = ["fwd", "fwd_splitkv", "fwd_splitkv_noalloc", "fwd_kvcache", "fwd_kvcache_paged", "fwd_unfused",
           "unfused_workspace_bytes", "q8_0_gemv", "FaError", "validate", "workspace_bytes", "release_workspace",
           "set_workspace", "version", "DTYPE_CODES", "kvcache_append", "kvcache_append_paged",
           "fwd_window", "fwd_window_paged", "window_workspace_bytes", "fwd_prefix", "fwd_prefix_paged",
           "prefix_workspace_bytes"]


class FaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{message} (status {status})")
        self.status = status


def _torch():
    import torch

    return torch


DTYPE_CODES = {"f16": 0, "bf16": 1, "f32": 2}


class _Runtime:
    """What a call needs from PyTorch, looked up once: the type codes and the
    cheapest ways to the current device and to a device's current stream (a
    small call costs about as much on the host as on the GPU)."""

    def __init__(self):
        torch = _torch()
        self.torch = torch
        self.Tensor = torch.Tensor
        self.float32 = torch.float32
        self.uint8 = torch.uint8
        self.int32 = torch.int32
        self.codes = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
        self.contiguous = torch.contiguous_format
        self.current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        self.stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda index: torch.cuda.current_stream(index).cuda_stream)


_RUNTIME = None


def _runtime():
    global _RUNTIME
    if _RUNTIME is None:
        _RUNTIME = _Runtime()
    return _RUNTIME


def _check(lib, st: int):
    if st != 0:
        raise FaError(st, lib.fa_status_string(st).decode())


def _call(rt, lib, index, fn, args):
    """fn(*args) with device ``index`` current."""
    if rt.current_device() == index:
        st = fn(*args)
    else:
        with rt.torch.cuda.device(index):
            st = fn(*args)
    if st != 0:
        _check(lib, st)


def _like(rt, t, dtype):
    """An uninitialised contiguous tensor of t's shape and device."""
    if type(t) is rt.Tensor:
        return rt.torch.empty_like(t, dtype=dtype, memory_format=rt.contiguous)
    return rt.torch.empty(t.shape, dtype=dtype, device=t.device)


def _outputs(rt, q, out, lse, odt, return_lse, B, Hq, Nq):
    """The output tensors of a call: those given, checked, or new ones."""
    if out is None:
        out = _like(rt, q, odt)
    elif out.shape != q.shape or out.dtype != odt or not out.is_contiguous() or out.device != q.device:
        raise ValueError("out must be a contiguous [B, Nq, Hq, D] tensor of the output dtype")
    if lse is None:
        if return_lse:
            lse = rt.torch.empty(B, Hq, Nq, dtype=rt.float32, device=q.device)
    elif (tuple(lse.shape) != (B, Hq, Nq) or lse.dtype != rt.float32 or not lse.is_contiguous()
          or lse.device != q.device):
        raise ValueError("lse must be a contiguous float32 [B, Hq, Nq] tensor")
    return out, lse


def _prepare(rt, q, k, v, out, lse, out_dtype, return_lse):
    if not (q.is_cuda and k.is_cuda and v.is_cuda and q.is_contiguous() and k.is_contiguous()
            and v.is_contiguous() and q.dim() == 4 and k.dim() == 4 and v.dim() == 4):
        for name, t in (("q", q), ("k", k), ("v", v)):
            if not t.is_cuda:
                raise ValueError(f"{name} must be a GPU tensor")
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous ([B, N, H, D] row-major)")
            if t.dim() != 4:
                raise ValueError(f"{name} must be 4-D [B, N, H, D]")
    dt = q.dtype
    if not (q.get_device() == k.get_device() == v.get_device()):
        raise ValueError("q, k, v must be on the same device")
    if not (dt == k.dtype == v.dtype) or dt not in rt.codes:
        raise ValueError("q, k, v must share one dtype among float16, bfloat16, float32")
    B, Nq, Hq, D = q.shape
    kshape = k.shape
    Bk, Nk, Hkv, Dk = kshape
    if v.shape != kshape or Bk != B or Dk != D:
        raise ValueError("k and v must be [B, Nk, Hkv, D] with q's B and D")
    odt = dt if out_dtype is None else out_dtype
    out, lse = _outputs(rt, q, out, lse, odt, return_lse, B, Hq, Nq)
    return (B, Hq, Hkv, Nq, Nk, D), out, lse, odt


def _workspace_arg(workspace, device):
    """(pointer, bytes) of a caller-owned decode workspace tensor."""
    if (workspace.dtype != _runtime().uint8 or not workspace.is_contiguous()
            or workspace.device != device):
        raise ValueError("workspace must be a contiguous uint8 tensor on q's device")
    return workspace.data_ptr(), workspace.numel()


def fwd(q, k, v, causal: bool = False, scale: float | None = None, out=None, lse=None,
        out_dtype=None, return_lse: bool = True, num_splits: int | None = None,
        heads_per_workgroup: int | None = None, workspace=None, slots_per_workgroup: int | None = None):
    """Attention forward o = softmax(scale * q k^T) v on the GPU.

    q [B, Nq, Hq, D], k and v [B, Nk, Hkv, D] (contiguous, same dtype and
    device); Hq must be a multiple of Hkv (query head h uses key/value head
    h // (Hq // Hkv)); ``causal`` uses the bottom-right mask (key j visible to
    query i iff j <= i + Nk - Nq).  ``scale`` defaults to 1/sqrt(D).
    ``out_dtype=torch.float32`` returns the kernel's fp32 result before the
    final rounding.  ``num_splits`` forces the decode split count (decode
    shapes only); ``heads_per_workgroup`` (1, 2 or 4) forces the prefill
    query-head packing (see fa_fwd_packed) and ``slots_per_workgroup`` (1, 2, 4
    or 8) the prefill workgroup layout (fa_fwd_slots).  ``workspace`` (a contiguous uint8
    GPU tensor of at least workspace_bytes(...) bytes) is this call's own
    decode workspace (fa_fwd_ws); otherwise the library-owned one of the
    current stream is used.  Returns (out, lse) with lse
    [B, Hq, Nq] float32 natural-log
    log-sum-exp (None if return_lse is False and no lse tensor was given).
    """
    lib = _lib.load()
    rt = _runtime()
    (B, Hq, Hkv, Nq, Nk, D), out, lse, odt = _prepare(rt, q, k, v, out, lse, out_dtype, return_lse)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    index = q.device.index
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
            lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Nq, Nk, D,
            1 if causal else 0, float(scale), rt.stream(index), rt.codes[q.dtype], rt.codes.get(odt, -1))
    if num_splits is None and heads_per_workgroup is None and workspace is None and slots_per_workgroup is None:
        fn = lib.fa_fwd
    elif heads_per_workgroup is not None and slots_per_workgroup is None and (num_splits is not None
                                                                              or workspace is not None):
        raise ValueError("heads_per_workgroup excludes num_splits and workspace")
    elif slots_per_workgroup is not None:
        if num_splits is not None or workspace is not None:
            raise ValueError("slots_per_workgroup excludes num_splits and workspace")
        fn, args = lib.fa_fwd_slots, (*args, int(slots_per_workgroup), int(heads_per_workgroup or 0))
    elif workspace is not None:
        fn, args = lib.fa_fwd_ws, (*args, int(num_splits or 0), *_workspace_arg(workspace, q.device))
    elif num_splits is not None:
        fn, args = lib.fa_fwd_splitkv, (*args, int(num_splits))
    else:
        fn, args = lib.fa_fwd_packed, (*args, int(heads_per_workgroup))
    _call(rt, lib, index, fn, args)
    return out, lse


def unfused_workspace_bytes(B: int, Hq: int, Nq: int, Nk: int) -> int:
    """Workspace bytes of fwd_unfused (fa_unfused_workspace_bytes)."""
    return int(_lib.load().fa_unfused_workspace_bytes(B, Hq, Nq, Nk))


def fwd_unfused(q, k, v, causal: bool = False, scale: float | None = None, out=None, lse=None,
                out_dtype=None, return_lse: bool = True, workspace=None):
    """Unfused self-attention (fa_fwd_unfused): the result of ``fwd`` with the
    score matrix materialised -- S = scale q k^T in fp32, P = softmax(S) in
    fp16, then O = P v, three kernels through HBM.  fp16 / bf16, D in {64,
    128}.  ``workspace``: a contiguous uint8 GPU tensor of at least
    unfused_workspace_bytes(B, Hq, Nq, Nk) bytes (allocated per call when
    None); afterwards it holds S [B, Hq, Nq, NkP] fp32 followed by P
    [B, Hq, Nq, NkP] fp16 (NkP = Nk rounded up to 64) on each row's visible
    keys.  Returns (out, lse) as ``fwd``.
    """
    lib = _lib.load()
    rt = _runtime()
    (B, Hq, Hkv, Nq, Nk, D), out, lse, odt = _prepare(rt, q, k, v, out, lse, out_dtype, return_lse)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if workspace is None:
        need = int(lib.fa_unfused_workspace_bytes(B, Hq, Nq, Nk))
        workspace = rt.torch.empty(max(need, 1), dtype=rt.uint8, device=q.device)
    index = q.device.index
    _call(rt, lib, index, lib.fa_fwd_unfused,
          (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
           lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Nq, Nk, D, int(bool(causal)),
           float(scale), rt.stream(index), rt.codes[q.dtype], rt.codes.get(odt, -1),
           *_workspace_arg(workspace, q.device)))
    return out, lse


def _check_lengths(rt, seqlens_k, B, device):
    if (seqlens_k.dtype != rt.int32 or seqlens_k.shape != (B,) or not seqlens_k.is_contiguous()
            or seqlens_k.get_device() != device.index):
        raise ValueError("seqlens_k must be a contiguous int32 [B] tensor on q's device")


def fwd_kvcache(q, k_cache, v_cache, seqlens_k, causal: bool = False, scale: float | None = None,
                out=None, lse=None, out_dtype=None, return_lse: bool = True, workspace=None):
    """Attention against K/V caches [B, Nk, Hkv, D] of which the first
    ``seqlens_k[b]`` rows are valid (``seqlens_k``: int32 [B] on the same
    device); q [B, Nq, Hq, D] holds each sequence's last Nq positions (decode
    for Nq = 1, chunked prefill otherwise).  Rows that see no key give 0 and
    lse -inf.  ``workspace``: this call's own decode workspace (uint8 GPU
    tensor; fa_fwd_kvcache_ws).  See fa_fwd_kvcache in include/fa.h."""
    lib = _lib.load()
    rt = _runtime()
    (B, Hq, Hkv, Nq, Nk, D), out, lse, odt = _prepare(rt, q, k_cache, v_cache, out, lse, out_dtype,
                                                      return_lse)
    _check_lengths(rt, seqlens_k, B, q.device)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    index = q.device.index
    args = (q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr(),
            lse.data_ptr() if lse is not None else None, seqlens_k.data_ptr(),
            B, Hq, Hkv, Nq, Nk, D, 1 if causal else 0, float(scale), rt.stream(index),
            rt.codes[q.dtype], rt.codes.get(odt, -1))
    if workspace is not None:
        _call(rt, lib, index, lib.fa_fwd_kvcache_ws, (*args, *_workspace_arg(workspace, q.device)))
    else:
        _call(rt, lib, index, lib.fa_fwd_kvcache, args)
    return out, lse


def _prepare_paged(rt, q, k_pages, v_pages, block_table, seqlens_k, out, lse, out_dtype, return_lse):
    """As ``_prepare`` for a paged cache; the sizes are B, Hq, Hkv, Nq, D,
    page_size, max_pages, num_pages."""
    for name, t in (("q", q), ("k_pages", k_pages), ("v_pages", v_pages)):
        if not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError(f"{name} must be a contiguous 4-D GPU tensor")
    dt, index = q.dtype, q.get_device()
    if not (index == k_pages.get_device() == v_pages.get_device()):
        raise ValueError("q and the page pools must be on the same device")
    if not (dt == k_pages.dtype == v_pages.dtype) or dt not in rt.codes:
        raise ValueError("q and the page pools must share one dtype")
    if k_pages.shape != v_pages.shape:
        raise ValueError("k_pages and v_pages must have the same shape")
    B, Nq, Hq, D = q.shape
    num_pages, page_size, Hkv, Dk = k_pages.shape
    if Dk != D:
        raise ValueError("the page pools' head size differs from q's")
    for name, t in (("block_table", block_table), ("seqlens_k", seqlens_k)):
        if (t.dtype != rt.int32 or not t.is_contiguous() or t.get_device() != index
                or (t is seqlens_k and t.shape != (B,))):
            raise ValueError(f"{name} must be a contiguous int32 tensor on q's device")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B, max_pages]")
    odt = dt if out_dtype is None else out_dtype
    out, lse = _outputs(rt, q, out, lse, odt, return_lse, B, Hq, Nq)
    return (B, Hq, Hkv, Nq, D, page_size, block_table.shape[1], num_pages), out, lse, odt


def fwd_kvcache_paged(q, k_pages, v_pages, block_table, seqlens_k, causal: bool = False,
                      scale: float | None = None, out=None, lse=None, out_dtype=None,
                      return_lse: bool = True, workspace=None):
    """Attention against a paged K/V cache: ``k_pages``, ``v_pages``
    [num_pages, page_size, Hkv, D] (page_size a multiple of 64), ``block_table``
    int32 [B, max_pages] (page of each block of page_size keys of each
    sequence), ``seqlens_k`` int32 [B]; q [B, Nq, Hq, D] holds each sequence's
    last Nq positions.  ``workspace``: this call's own decode workspace
    (uint8 GPU tensor; fa_fwd_kvcache_paged_ws).  See fa_fwd_kvcache_paged in
    include/fa.h."""
    lib = _lib.load()
    rt = _runtime()
    dims, out, lse, odt = _prepare_paged(rt, q, k_pages, v_pages, block_table, seqlens_k, out, lse, out_dtype, return_lse)
    if scale is None:
        scale = 1.0 / math.sqrt(dims[4])
    index = q.device.index
    args = (q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), out.data_ptr(),
            lse.data_ptr() if lse is not None else None, seqlens_k.data_ptr(), block_table.data_ptr(),
            *dims, 1 if causal else 0, float(scale), rt.stream(index), rt.codes[q.dtype], rt.codes.get(odt, -1))
    if workspace is not None:
        _call(rt, lib, index, lib.fa_fwd_kvcache_paged_ws, (*args, *_workspace_arg(workspace, q.device)))
    else:
        _call(rt, lib, index, lib.fa_fwd_kvcache_paged, args)
    return out, lse


def window_workspace_bytes(B, Hq, Hkv, Nq, Nk, D, window, in_dtype: str, sinks: int = 0) -> int:
    """Workspace bytes of fwd_window (fa_window_workspace_bytes)."""
    return int(_lib.load().fa_window_workspace_bytes(B, Hq, Hkv, Nq, Nk, D, _int32(window), _int32(sinks),
                                                     DTYPE_CODES[in_dtype]))


def fwd_window(q, k, v, window: int, sinks: int = 0, seqlens_k=None, scale: float | None = None, out=None, lse=None,
               out_dtype=None, return_lse: bool = True, workspace=None):
    """Causal attention with a sliding window: the query at position p sees the
    ``window`` keys p - window + 1 .. p and the first ``sinks`` keys
    (fa_fwd_window).  q [B, Nq, Hq, D] holds the last Nq of each sequence's
    ``seqlens_k`` (int32 [B]; None: Nk) keys in k, v [B, Nk, Hkv, D]: a whole
    prompt, a chunk of one, or one token.  Rows that see no key give 0 and lse
    -inf.  ``workspace``: this call's own scratch (uint8 GPU tensor of
    window_workspace_bytes(...) bytes).  Returns (out, lse) as ``fwd``."""
    lib = _lib.load()
    rt = _runtime()
    dims, out, lse, odt = _prepare(rt, q, k, v, out, lse, out_dtype, return_lse)
    if seqlens_k is not None:
        _check_lengths(rt, seqlens_k, dims[0], q.device)
    if scale is None:
        scale = 1.0 / math.sqrt(dims[5])
    index = q.device.index
    _call(rt, lib, index, lib.fa_fwd_window,
          (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr() if lse is not None else None,
           seqlens_k.data_ptr() if seqlens_k is not None else None, *dims, _int32(window), _int32(sinks), float(scale),
           rt.stream(index), rt.codes[q.dtype], rt.codes.get(odt, -1),
           *((None, 0) if workspace is None else _workspace_arg(workspace, q.device))))
    return out, lse


def fwd_window_paged(q, k_pages, v_pages, block_table, seqlens_k, window: int, sinks: int = 0,
                     scale: float | None = None, out=None, lse=None, out_dtype=None, return_lse: bool = True,
                     workspace=None):
    """``fwd_window`` against the paged cache of ``fwd_kvcache_paged``.  Pages
    that hold no visible key are not read (fa_fwd_window_paged)."""
    lib = _lib.load()
    rt = _runtime()
    dims, out, lse, odt = _prepare_paged(rt, q, k_pages, v_pages, block_table, seqlens_k, out, lse, out_dtype, return_lse)
    if scale is None:
        scale = 1.0 / math.sqrt(dims[4])
    index = q.device.index
    _call(rt, lib, index, lib.fa_fwd_window_paged,
          (q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), out.data_ptr(),
           lse.data_ptr() if lse is not None else None, seqlens_k.data_ptr(), block_table.data_ptr(), *dims,
           _int32(window), _int32(sinks), float(scale), rt.stream(index), rt.codes[q.dtype], rt.codes.get(odt, -1),
           *((None, 0) if workspace is None else _workspace_arg(workspace, q.device))))
    return out, lse


def prefix_workspace_bytes(B, Hq, Hkv, Nq, Np, Nk, D, in_dtype: str) -> int:
    """Workspace bytes of fwd_prefix (fa_prefix_workspace_bytes)."""
    return int(_lib.load().fa_prefix_workspace_bytes(B, Hq, Hkv, Nq, Np, Nk, D, DTYPE_CODES[in_dtype]))


def fwd_prefix(q, k_prefix, v_prefix, k, v, seqlens_k=None, causal: bool = False, scale: float | None = None,
               out=None, lse=None, out_dtype=None, return_lse: bool = True, workspace=None):
    """Attention of a batch whose sequences share a prefix, which is read once
    for all of them: ``fwd_kvcache`` on each sequence's prefix and suffix one
    after the other (fa_fwd_prefix).  ``k_prefix``, ``v_prefix`` [Np, Hkv, D]; ``k``,
    ``v`` [B, Nk, Hkv, D], each sequence's own keys, of which the first
    ``seqlens_k`` (int32 [B]; None: Nk) are valid; q [B, Nq, Hq, D] holds the last
    Nq positions of each.  fp16 / bf16, D in {64, 128}.  ``workspace``: this call's
    own scratch (uint8 GPU tensor of prefix_workspace_bytes(...) bytes).  Returns
    (out, lse) as ``fwd``."""
    lib = _lib.load()
    rt = _runtime()
    (B, Hq, Hkv, Nq, Nk, D), out, lse, odt = _prepare(rt, q, k, v, out, lse, out_dtype, return_lse)
    dt, index, shape = q.dtype, q.get_device(), k_prefix.shape
    if (len(shape) != 3 or shape[1] != Hkv or shape[2] != D or v_prefix.shape != shape or not k_prefix.is_contiguous()
            or not v_prefix.is_contiguous() or k_prefix.dtype != dt or v_prefix.dtype != dt
            or k_prefix.get_device() != index or v_prefix.get_device() != index):
        raise ValueError("k_prefix and v_prefix must be contiguous [Np, Hkv, D] tensors of q's dtype and device")
    if seqlens_k is not None:
        _check_lengths(rt, seqlens_k, B, q.device)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    _call(rt, lib, index, lib.fa_fwd_prefix,
          (q.data_ptr(), k_prefix.data_ptr(), v_prefix.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
           lse.data_ptr() if lse is not None else None, seqlens_k.data_ptr() if seqlens_k is not None else None,
           B, Hq, Hkv, Nq, shape[0], Nk, D, 1 if causal else 0, float(scale), rt.stream(index), rt.codes[dt],
           rt.codes.get(odt, -1),
           *((None, 0) if workspace is None else _workspace_arg(workspace, q.device))))
    return out, lse


def fwd_prefix_paged(q, k_pages, v_pages, block_table, seqlens_k, prefix_len: int, causal: bool = False,
                     scale: float | None = None, out=None, lse=None, out_dtype=None, return_lse: bool = True,
                     workspace=None):
    """``fwd_kvcache_paged`` for sequences whose first ``prefix_len`` keys (a
    multiple of the page size) lie in the same pages, which every row of
    ``block_table`` names: these are read once for the whole batch
    (fa_fwd_prefix_paged)."""
    lib = _lib.load()
    rt = _runtime()
    dims, out, lse, odt = _prepare_paged(rt, q, k_pages, v_pages, block_table, seqlens_k, out, lse, out_dtype, return_lse)
    if scale is None:
        scale = 1.0 / math.sqrt(dims[4])
    index = q.device.index
    _call(rt, lib, index, lib.fa_fwd_prefix_paged,
          (q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(), out.data_ptr(),
           lse.data_ptr() if lse is not None else None, seqlens_k.data_ptr(), block_table.data_ptr(), *dims,
           _int32(prefix_len), 1 if causal else 0, float(scale), rt.stream(index), rt.codes[q.dtype],
           rt.codes.get(odt, -1), *((None, 0) if workspace is None else _workspace_arg(workspace, q.device))))
    return out, lse


def _int32(n):
    """n, at most what a C int holds (a window past every cache is like any other), and
    at least -1 (refused like any negative number)."""
    return max(min(int(n), 0x7fffffff), -1)


def _token_stride(t, name, B, N, H, D):
    """Elements between the consecutive tokens of t [B, N, H, D], whose heads and
    columns are dense and whose sequences follow each other."""
    sb, sn, sh, sd = t.stride()
    row = H * D
    step = sn if N > 1 else sb if B > 1 else row
    if ((sd != 1 and D > 1) or (sh != D and H > 1) or (N > 1 and B > 1 and sb != N * sn)
            or step < row):   # (0, to the call, means dense)
        raise ValueError(f"{name} must be [B, N, H, D] with dense heads and one stride between its tokens")
    return step


def _rotary(rt, inv_freq, positions, pair_axes, interleaved, B, N, index):
    """The fa_rotary_t of a call (None: no rotation)."""
    if inv_freq is None:
        if positions is not None or pair_axes is not None:
            raise ValueError("positions and pair_axes need inv_freq")
        return None
    if (inv_freq.dtype != rt.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous()
            or inv_freq.get_device() != index):
        raise ValueError("inv_freq must be a contiguous float32 [rot_dim / 2] tensor on k's device")
    pairs, axes, at = inv_freq.shape[0], 1, None
    if positions is not None:
        shape = tuple(positions.shape)
        if (positions.dtype != rt.int32 or not positions.is_contiguous() or positions.get_device() != index
                or shape[-2:] != (B, N) or len(shape) > 3):
            raise ValueError("positions must be a contiguous int32 [B, N] or [axes, B, N] tensor on k's device")
        axes, at = shape[0] if len(shape) == 3 else 1, positions.data_ptr()
    r = _lib.Rotary(inv_freq.data_ptr(), at, 2 * pairs, 1 if interleaved else 0, axes)
    if axes > 1:
        if pair_axes is None or len(pair_axes) != pairs:
            raise ValueError("several axes need pair_axes, the axis of each of the rot_dim / 2 pairs")
        if pairs <= _lib.FA_MAX_ROTARY_PAIRS:   # (more are refused by the call)
            # item by item: bytes() of an array of wider integers is its memory
            if not isinstance(pair_axes, bytes):
                pair_axes = bytes(operator.index(a) for a in pair_axes)
            ctypes.memmove(r.pair_axis, pair_axes, pairs)
    return r


def _append(k, v, k_cache, v_cache, block_table, seqlens_k, q, q_out, inv_freq, positions, pair_axes, interleaved):
    lib = _lib.load()
    rt = _RUNTIME or _runtime()
    dt, index = k.dtype, k.get_device()
    if index < 0 or k.dim() != 4 or dt not in rt.codes:
        raise ValueError("k must be a 4-D [B, N, Hkv, D] GPU tensor of float16, bfloat16 or float32")
    shape, cshape = k.shape, k_cache.shape
    if v.shape != shape or v.dtype != dt or v.get_device() != index:
        raise ValueError("v must have k's shape, dtype and device")
    B, N, Hkv, D = shape
    if (len(cshape) != 4 or v_cache.shape != cshape or not k_cache.is_contiguous() or not v_cache.is_contiguous()
            or k_cache.dtype != dt or v_cache.dtype != dt or k_cache.get_device() != index
            or v_cache.get_device() != index):
        raise ValueError("the caches must be contiguous and 4-D, of one shape, and of k's dtype and device")
    first, rows, ch, cd = cshape
    if ch != Hkv or cd != D or (block_table is None and first != B):
        raise ValueError("the caches must have k's heads and head size" + ("" if block_table is not None else " and batch"))
    if (seqlens_k.dtype != rt.int32 or seqlens_k.shape != (B,) or not seqlens_k.is_contiguous()
            or seqlens_k.get_device() != index):
        raise ValueError("seqlens_k must be a contiguous int32 [B] tensor on k's device")
    Hq = qs = 0
    qp = qo = None
    if q is not None:
        if q.dim() != 4 or q.dtype != dt or q.get_device() != index:
            raise ValueError("q must be [B, N, Hq, D] with k's B, N, D, dtype and device")
        qb, qn, Hq, qd = q.shape
        if qb != B or qn != N or qd != D:
            raise ValueError("q must be [B, N, Hq, D] with k's B, N, D, dtype and device")
        qs = _token_stride(q, "q", B, N, Hq, D)
        if q_out is None:
            q_out = _like(rt, q, dt)
        elif q_out.shape != q.shape or q_out.dtype != dt or not q_out.is_contiguous() or q_out.get_device() != index:
            raise ValueError("q_out must be a contiguous tensor of q's shape, dtype and device")
        qp, qo = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out needs q")
    r = _rotary(rt, inv_freq, positions, pair_axes, interleaved, B, N, index)
    ks, vs = _token_stride(k, "k", B, N, Hkv, D), _token_stride(v, "v", B, N, Hkv, D)
    rp = None if r is None else ctypes.addressof(r)
    if block_table is None:
        _call(rt, lib, index, lib.fa_kvcache_append,
              (k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), qp, qo, seqlens_k.data_ptr(),
               B, Hq, Hkv, N, rows, D, qs, ks, vs, rp, rt.stream(index), rt.codes[dt]))
    else:
        if (block_table.dtype != rt.int32 or block_table.dim() != 2 or block_table.shape[0] != B
                or not block_table.is_contiguous() or block_table.get_device() != index):
            raise ValueError("block_table must be a contiguous int32 [B, max_pages] tensor on k's device")
        _call(rt, lib, index, lib.fa_kvcache_append_paged,
              (k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), qp, qo, seqlens_k.data_ptr(),
               block_table.data_ptr(), B, Hq, Hkv, N, D, rows, block_table.shape[1], first, qs, ks, vs, rp,
               rt.stream(index), rt.codes[dt]))
    return q_out


def kvcache_append(k, v, k_cache, v_cache, seqlens_k, q=None, q_out=None, inv_freq=None, positions=None,
                   pair_axes=None, interleaved: bool = False):
    """Write new keys and values into the caches that ``fwd_kvcache`` reads and
    rotate them, and the new queries, by their positions (fa_kvcache_append).

    ``k``, ``v`` [B, N, Hkv, D] are the last N of each sequence's ``seqlens_k``
    (int32 [B], the new tokens included) keys: token i goes to row seqlens_k[b] -
    N + i of the contiguous ``k_cache``, ``v_cache`` [B, Nk, Hkv, D]; rows below
    0 (padding) and past the cache are not written.  ``k``, ``v`` and ``q``
    [B, N, Hq, D] may be parts of one projection's result (dense heads, one
    stride between tokens).  ``inv_freq`` (float32 [rot_dim / 2], None: no
    rotation): radians per position of each pair of columns, j and j + rot_dim /
    2, or 2 j and 2 j + 1 if ``interleaved``.  ``positions``: int32 [B, N], or
    [axes, B, N] with ``pair_axes``, the axis that turns each pair (bytes or any
    sequence of integers); None: the cache rows.  Returns the rotated queries
    (``q_out`` if given, which may be ``q`` if that is contiguous; None without
    ``q``)."""
    return _append(k, v, k_cache, v_cache, None, seqlens_k, q, q_out, inv_freq, positions, pair_axes, interleaved)


def kvcache_append_paged(k, v, k_pages, v_pages, block_table, seqlens_k, q=None, q_out=None, inv_freq=None,
                         positions=None, pair_axes=None, interleaved: bool = False):
    """``kvcache_append`` into the paged cache of ``fwd_kvcache_paged``: ``k_pages``,
    ``v_pages`` [num_pages, page_size, Hkv, D], ``block_table`` int32 [B,
    max_pages].  Tokens whose table entry is outside the pool are not written
    (fa_kvcache_append_paged)."""
    if block_table is None:
        raise ValueError("block_table must be a contiguous int32 [B, max_pages] tensor on k's device")
    return _append(k, v, k_pages, v_pages, block_table, seqlens_k, q, q_out, inv_freq, positions, pair_axes, interleaved)


def q8_0_gemv(w, x, out=None, out_dtype=None):
    """Q8_0 matrix-vector product y = W x (the decode-time linear layers).

    ``w``: uint8 GPU tensor holding M rows of K / 32 Q8_0 blocks of 34 bytes
    (binary16 scale, little-endian, then 32 int8 values), shaped [M, K/32, 34]
    or [M, K/32 * 34], contiguous.  ``x``: [K] float16, bfloat16 or float32 on
    the same device.  Returns y [M] in ``out_dtype`` (x's dtype, or float32).
    See fa_q8_0_gemv in include/fa.h."""
    lib = _lib.load()
    rt = _runtime()
    dev, dt = x.device, x.dtype
    if not (w.is_cuda and x.is_cuda) or w.device != dev:
        raise ValueError("w and x must be GPU tensors on one device")
    if w.dtype != rt.uint8 or not w.is_contiguous() or w.dim() not in (2, 3):
        raise ValueError("w must be a contiguous uint8 [M, K/32, 34] or [M, K/32*34] tensor")
    if x.dim() != 1 or not x.is_contiguous() or dt not in rt.codes:
        raise ValueError("x must be a contiguous 1-D float16, bfloat16 or float32 tensor")
    wshape, K = w.shape, x.shape[0]
    M = wshape[0]
    row_bytes = (wshape[1] if len(wshape) == 2 else wshape[1] * wshape[2]) if M > 0 else 0
    if (len(wshape) == 3 and wshape[2] != 34) or K % 32 != 0 or row_bytes != K // 32 * 34:
        raise ValueError("w must hold K/32 blocks of 34 bytes per row, K = len(x) a multiple of 32")
    odt = dt if out_dtype is None else out_dtype
    if out is None:
        out = rt.torch.empty(M, dtype=odt, device=dev)
    elif tuple(out.shape) != (M,) or out.dtype != odt or not out.is_contiguous() or out.device != dev:
        raise ValueError("out must be a contiguous [M] tensor of the output dtype")
    index = dev.index
    _call(rt, lib, index, lib.fa_q8_0_gemv, (w.data_ptr(), x.data_ptr(), out.data_ptr(), M, K, rt.codes[dt],
                                             rt.codes.get(odt, -1), rt.stream(index)))
    return out


def fwd_splitkv_noalloc(q, k, v, num_splits: int = 0, causal: bool = False, scale: float | None = None,
                        out=None, lse=None, out_dtype=None, return_lse: bool = True):
    """fa_fwd_splitkv_noalloc: the decode forward with its split-KV partial
    results in the library's fixed device scratch (32 MiB per GPU) -- the C
    call allocates nothing (pass ``out``/``lse`` to keep this function from
    allocating them).  Calls that overlap on one GPU share the scratch and
    must be ordered."""
    lib = _lib.load()
    rt = _runtime()
    (B, Hq, Hkv, Nq, Nk, D), out, lse, odt = _prepare(rt, q, k, v, out, lse, out_dtype, return_lse)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    index = q.device.index
    _call(rt, lib, index, lib.fa_fwd_splitkv_noalloc,
          (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
           lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Nq, Nk, D, int(bool(causal)),
           float(scale), rt.stream(index), rt.codes[q.dtype], rt.codes.get(odt, -1), int(num_splits)))
    return out, lse


def fwd_splitkv(q, k, v, num_splits: int, **kw):
    """``fwd`` with an explicit decode split count (0 = default choice)."""
    return fwd(q, k, v, num_splits=num_splits, **kw)


def validate(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, Hq, Hkv, Nq, Nk, D, causal, scale,
             in_dtype: str, out_dtype: str | None = None) -> int:
    """Status code of the library's host-side argument checks (no GPU use)."""
    lib = _lib.load()
    def code(x):
        return DTYPE_CODES[x] if x in DTYPE_CODES else int(x)

    in_code = code(in_dtype)
    out_code = in_code if out_dtype is None else code(out_dtype)
    return int(lib.fa_validate(q_ptr, k_ptr, v_ptr, o_ptr, lse_ptr, B, Hq, Hkv, Nq, Nk, D,
                               int(causal), float(scale), in_code, out_code))


def workspace_bytes(B, Hq, Hkv, Nq, Nk, D, in_dtype: str, num_splits: int = 0) -> int:
    return int(_lib.load().fa_workspace_bytes(B, Hq, Hkv, Nq, Nk, D, DTYPE_CODES[in_dtype],
                                              num_splits))


def release_workspace():
    lib = _lib.load()
    _check(lib, lib.fa_release_workspace())


_USER_WORKSPACE = {}   # device index -> caller tensor kept alive while set


def set_workspace(buf=None):
    """Use the device tensor ``buf`` (contiguous, on the current device) as
    the decode workspace of its device, or return to the library-owned one
    with ``None``; see fa_set_workspace in include/fa.h."""
    torch = _torch()
    lib = _lib.load()
    if buf is None:
        dev = torch.cuda.current_device()
        _check(lib, lib.fa_set_workspace(None, 0))
        _USER_WORKSPACE.pop(dev, None)
        return
    if not buf.is_cuda or not buf.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    if buf.device.index != torch.cuda.current_device():
        raise ValueError("workspace must be on the current device")
    nbytes = buf.numel() * buf.element_size()
    _check(lib, lib.fa_set_workspace(buf.data_ptr() if nbytes else None, nbytes))
    _USER_WORKSPACE[buf.device.index] = buf


def version() -> tuple:
    v = _lib.load().fa_version()
    return (v >> 16, (v >> 8) & 0xFF, v & 0xFF)
