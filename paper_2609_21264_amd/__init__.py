"""Attention forward for AMD Instinct MI355X (gfx950): the fused kernel and the unfused baseline.

A thin Python binding over ``libfa.so``, whose C ABI is declared in ``include/fa.h``. PyTorch only
supplies device memory and the stream; every step of the computation runs in the library's HIP
kernel. The functions below marshal arguments and translate status codes, nothing more.

* :func:`fa_fwd`, :func:`fa_fwd_ex`, :func:`fa_fwd_split`, :func:`fa_fwd_split_workspace_bytes`,
  :func:`fa_status_str`, :func:`fa_block_rows`, :func:`fa_fwd_rows`, :func:`fa_fwd_instance` -- the C entry
  points under the same names, taking raw device pointers (ints) and sizes.
* :func:`fa_lbl_scores`, :func:`fa_lbl_softmax`, :func:`fa_lbl_pv`, :func:`fa_lbl_ld`,
  :func:`fa_lbl_workspace_bytes`, :func:`fa_fwd_unfused` -- the layer-by-layer (unfused) operators
  and their composition, under the same names.
* :func:`fa_fwd_decode`, :func:`fa_fwd_decode_parts` -- the decode-shaped path (few query rows per
  key/value head); :func:`fa_fwd_decode_noalloc` -- the same with its partial results in the
  library's static device scratch, for callers that cannot allocate.
* :func:`forward` -- convenience wrapper over torch tensors (``n_split`` > 1 selects split mode and
  takes the workspace from torch's allocator; ``decode=True`` the decode-shaped path).
* :func:`forward_unfused` -- the same over the unfused path (``fa_fwd_unfused``).
* :func:`kv_append`, :func:`forward_paged` -- a paged key/value cache: appending new tokens to it with their
  position rotation, and their attention over it (C: ``fa_kv_append``, ``fa_fwd_paged``, whose descriptions are the
  ctypes structures :class:`PagedCache` and :class:`PagedBatch`; with positions ``fa_kv_append_at``, :class:`Positions`).
* :func:`rotate` -- the position rotation alone, and the way back (``fa_rotate``).
* :func:`tree_mask`, :func:`kv_compact`, :func:`kv_copy` -- around the paged cache: mask and positions of drafted
  trees, closing up the tokens that are kept, copies of pages (``fa_tree_mask``, ``fa_kv_compact``, ``fa_kv_copy``).
"""

from __future__ import annotations

import contextlib
import ctypes
import math
from typing import Optional

from . import _lib
from ._lib import (AppendStrides, PagedBatch, PagedCache, PagedScores, PagedStrides, Positions, RotateStrides,  # noqa: F401
                   FA_MAX_SOFTCAP,
                   FA_CACHE_BF16, FA_CACHE_E4M3, FA_PAGED_AUTO, FA_PAGED_FEW, FA_PAGED_MANY, FA_TREE_TOKENS, FA_TREE_WORDS,
                   FA_ERR_BAD_SCALE, FA_ERR_BAD_SHAPE, FA_ERR_HIP, FA_ERR_NULL_POINTER,
                   FA_ERR_UNSUPPORTED, FA_ERR_WORKSPACE, FA_INSTANCE_HALVES, FA_INSTANCE_LONG, FA_INSTANCE_NONE,
                   FA_INSTANCE_QUARTERS, FA_INSTANCE_SHORT, FA_INSTANCE_SHORT_WIDE, FA_NOALLOC_SCRATCH_BYTES, FA_OK,
                   LIB_PATH)

__all__ = ["fa_fwd", "fa_fwd_ex", "fa_fwd_split", "fa_fwd_split_workspace_bytes", "fa_fwd_split_parts",
           "fa_status_str", "fa_block_rows", "fa_fwd_rows", "fa_lbl_scores", "fa_lbl_softmax", "fa_lbl_pv", "fa_lbl_ld",
           "fa_lbl_workspace_bytes", "fa_fwd_unfused", "fa_fwd_decode", "fa_fwd_decode_parts",
           "fa_fwd_decode_noalloc", "fa_fwd_instance", "forward", "forward_unfused", "FaError", "LIB_PATH", "FA_NOALLOC_SCRATCH_BYTES",
           "fa_kv_append", "fa_fwd_paged", "fa_fwd_paged_workspace_bytes", "PagedCache", "PagedBatch", "AppendStrides",
           "PagedStrides", "FA_CACHE_BF16", "FA_CACHE_E4M3", "FA_PAGED_AUTO", "FA_PAGED_FEW",
           "FA_PAGED_MANY", "kv_append", "forward_paged", "fa_kv_append_at", "fa_rotate", "fa_tree_mask", "fa_kv_compact",
           "fa_kv_copy", "Positions", "RotateStrides", "FA_TREE_TOKENS", "FA_TREE_WORDS", "rotate", "tree_mask", "kv_compact",
           "kv_copy", "fa_fwd_paged_ex", "fa_fwd_paged_ex_workspace_bytes", "PagedScores", "FA_MAX_SOFTCAP"]


class FaError(RuntimeError):
    """A non-FA_OK status from the library."""

    def __init__(self, status: int):
        self.status = status
        super().__init__(f"{fa_status_str(status)} ({status})")


def fa_status_str(status: int) -> str:
    return _lib.load().fa_status_str(int(status)).decode()


def fa_block_rows(d_qk: int, d_v: int, causal: bool) -> int:
    return int(_lib.load().fa_block_rows(int(d_qk), int(d_v), int(bool(causal))))


def fa_fwd_rows(B: int, Hq: int, Sq: int, d_qk: int, d_v: int, causal: bool) -> int:
    return int(_lib.load().fa_fwd_rows(int(B), int(Hq), int(Sq), int(d_qk), int(d_v), int(bool(causal))))


def fa_fwd_instance(B: int, Hq: int, Hkv: int, Sq: int, Sk: int, d_qk: int, d_v: int, causal: bool,
                    n_split: int = 0) -> int:
    """C ``fa_fwd_instance``: the FA_INSTANCE_* value of the kernel instance a call of these sizes runs
    (``n_split`` >= 1: in split mode)."""
    return int(_lib.load().fa_fwd_instance(int(B), int(Hq), int(Hkv), int(Sq), int(Sk), int(d_qk), int(d_v),
                                           int(bool(causal)), int(n_split)))


def fa_fwd(Q: int, K: int, V: int, O: int, B: int, Hq: int, Hkv: int, Sq: int, Sk: int, d: int,
           scale: float, causal: bool, stream: int) -> int:
    """C ``fa_fwd``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd(Q, K, V, O, B, Hq, Hkv, Sq, Sk, d, float(scale), int(bool(causal)), stream))


def fa_fwd_ex(Q: int, K: int, V: int, O: int, LSE: Optional[int], B: int, Hq: int, Hkv: int, Sq: int,
              Sk: int, d_qk: int, d_v: int, scale: float, causal: bool, stream: int) -> int:
    """C ``fa_fwd_ex``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd_ex(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, float(scale),
                                     int(bool(causal)), stream))


def fa_fwd_split(Q: int, K: int, V: int, O: int, LSE: Optional[int], B: int, Hq: int, Hkv: int, Sq: int,
                 Sk: int, d_qk: int, d_v: int, scale: float, causal: bool, n_split: int, workspace: Optional[int],
                 workspace_bytes: int, stream: int) -> int:
    """C ``fa_fwd_split``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd_split(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, float(scale),
                                        int(bool(causal)), int(n_split), workspace, int(workspace_bytes), stream))


def fa_fwd_split_workspace_bytes(B: int, Hq: int, Sq: int, d_v: int, n_split: int) -> int:
    """C ``fa_fwd_split_workspace_bytes``."""
    return int(_lib.load().fa_fwd_split_workspace_bytes(int(B), int(Hq), int(Sq), int(d_v), int(n_split)))


def fa_fwd_split_parts(n_cu: int, B: int, Hq: int, Sq: int, Sk: int, d_qk: int, d_v: int, causal: bool) -> int:
    """C ``fa_fwd_split_parts``."""
    return int(_lib.load().fa_fwd_split_parts(int(n_cu), int(B), int(Hq), int(Sq), int(Sk), int(d_qk), int(d_v),
                                              int(bool(causal))))


def fa_fwd_decode(Q: int, K: int, V: int, O: int, LSE: Optional[int], B: int, Hq: int, Hkv: int, Sq: int,
                  Sk: int, d_qk: int, d_v: int, scale: float, causal: bool, n_parts: int, workspace: Optional[int],
                  workspace_bytes: int, stream: int) -> int:
    """C ``fa_fwd_decode``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd_decode(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, float(scale),
                                         int(bool(causal)), int(n_parts), workspace, int(workspace_bytes), stream))


def fa_fwd_decode_noalloc(Q: int, K: int, V: int, O: int, LSE: Optional[int], B: int, Hq: int, Hkv: int, Sq: int,
                          Sk: int, d_qk: int, d_v: int, scale: float, causal: bool, n_parts: int, stream: int) -> int:
    """C ``fa_fwd_decode_noalloc``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd_decode_noalloc(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, float(scale),
                                                 int(bool(causal)), int(n_parts), stream))


def fa_fwd_decode_parts(n_cu: int, B: int, Hq: int, Hkv: int, Sq: int, Sk: int) -> int:
    """C ``fa_fwd_decode_parts``."""
    return int(_lib.load().fa_fwd_decode_parts(int(n_cu), int(B), int(Hq), int(Hkv), int(Sq), int(Sk)))


def fa_lbl_scores(Q: int, K: int, S: int, B: int, Hq: int, Hkv: int, Sq: int, Sk: int, d_qk: int, scale: float,
                  causal: bool, stream: int) -> int:
    """C ``fa_lbl_scores``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_lbl_scores(Q, K, S, B, Hq, Hkv, Sq, Sk, d_qk, float(scale), int(bool(causal)), stream))


def fa_lbl_softmax(S: int, P: int, LSE: Optional[int], B: int, Hq: int, Sq: int, Sk: int, causal: bool,
                   stream: int) -> int:
    """C ``fa_lbl_softmax``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_lbl_softmax(S, P, LSE, B, Hq, Sq, Sk, int(bool(causal)), stream))


def fa_lbl_pv(P: int, V: int, O: int, B: int, Hq: int, Hkv: int, Sq: int, Sk: int, d_v: int, causal: bool,
              stream: int) -> int:
    """C ``fa_lbl_pv``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_lbl_pv(P, V, O, B, Hq, Hkv, Sq, Sk, d_v, int(bool(causal)), stream))


def fa_lbl_ld(Sk: int) -> int:
    """C ``fa_lbl_ld``: row stride (elements) of the layer-by-layer spill buffers."""
    return int(_lib.load().fa_lbl_ld(int(Sk)))


def fa_lbl_workspace_bytes(B: int, Hq: int, Sq: int, Sk: int) -> int:
    """C ``fa_lbl_workspace_bytes``."""
    return int(_lib.load().fa_lbl_workspace_bytes(int(B), int(Hq), int(Sq), int(Sk)))


def fa_fwd_unfused(Q: int, K: int, V: int, O: int, LSE: Optional[int], B: int, Hq: int, Hkv: int, Sq: int,
                   Sk: int, d_qk: int, d_v: int, scale: float, causal: bool, workspace: Optional[int],
                   workspace_bytes: int, stream: int) -> int:
    """C ``fa_fwd_unfused``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd_unfused(Q, K, V, O, LSE, B, Hq, Hkv, Sq, Sk, d_qk, d_v, float(scale),
                                          int(bool(causal)), workspace, int(workspace_bytes), stream))


def fa_kv_append(cache: PagedCache, batch: PagedBatch, K: int, V: int, Q: Optional[int], Q_out: Optional[int], Hq: int,
                 strides: AppendStrides, cos_sin: Optional[int], n_pos: int, rot_begin: int, rot_dim: int,
                 interleaved: bool, stream: int) -> int:
    """C ``fa_kv_append``: descriptions, raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_kv_append(cache, batch, K, V, Q, Q_out, Hq, strides, cos_sin, n_pos, rot_begin,
                                        rot_dim, int(bool(interleaved)), stream))


def fa_kv_append_at(cache: PagedCache, batch: PagedBatch, K: int, V: int, Q: Optional[int], Q_out: Optional[int], Hq: int,
                    strides: AppendStrides, positions: Positions, cos_sin: Optional[int], n_pos: int, rot_begin: int,
                    rot_dim: int, interleaved: bool, stream: int) -> int:
    """C ``fa_kv_append_at``: descriptions, raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_kv_append_at(cache, batch, K, V, Q, Q_out, Hq, strides, positions, cos_sin, n_pos, rot_begin,
                                           rot_dim, int(bool(interleaved)), stream))


def fa_rotate(X: int, Y: int, B: int, H: int, S: int, d: int, strides: RotateStrides, positions: Optional[Positions],
              cos_sin: Optional[int], n_pos: int, rot_begin: int, rot_dim: int, interleaved: bool, inverse: bool,
              stream: int) -> int:
    """C ``fa_rotate``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_rotate(X, Y, B, H, S, d, strides, positions, cos_sin, n_pos, rot_begin, rot_dim,
                                     int(bool(interleaved)), int(bool(inverse)), stream))


def fa_tree_mask(parents: int, q_starts: int, kv_lens: int, B: int, T: int, max_keys: int, mask: int, words: int,
                 mask_stride: int, positions: int, stream: int) -> int:
    """C ``fa_tree_mask``: raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_tree_mask(parents, q_starts, kv_lens, B, T, max_keys, mask, words, mask_stride, positions, stream))


def fa_kv_compact(cache: PagedCache, batch: PagedBatch, kept: Optional[int], kept_stride: int, max_kept: int, n_kept: int,
                  kv_lens_out: int, stream: int) -> int:
    """C ``fa_kv_compact``: descriptions, raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_kv_compact(cache, batch, kept, kept_stride, max_kept, n_kept, kv_lens_out, stream))


def fa_kv_copy(cache: PagedCache, src: int, dst: int, n: int, stream: int) -> int:
    """C ``fa_kv_copy``: description, raw device addresses and the number of pairs; returns the status code."""
    return int(_lib.load().fa_kv_copy(cache, src, dst, n, stream))


def fa_fwd_paged(cache: PagedCache, batch: PagedBatch, Q: int, O: int, LSE: Optional[int], Hq: int,
                 strides: PagedStrides, max_q: int, path: int, scale: float, causal: bool, workspace: Optional[int],
                 workspace_bytes: int, stream: int) -> int:
    """C ``fa_fwd_paged``: descriptions, raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd_paged(cache, batch, Q, O, LSE, Hq, strides, max_q, path, float(scale),
                                        int(bool(causal)), workspace, int(workspace_bytes), stream))


def fa_fwd_paged_workspace_bytes(B: int, T: int, max_keys: int, Hq: int, Hkv: int, d_qk: int, d_v: int, type: int,
                                 max_q: int, path: int = FA_PAGED_AUTO) -> int:
    """C ``fa_fwd_paged_workspace_bytes`` (``max_keys``: blocks of the table times page size)."""
    return int(_lib.load().fa_fwd_paged_workspace_bytes(B, T, max_keys, Hq, Hkv, d_qk, d_v, type, max_q, path))


def fa_fwd_paged_ex(cache: PagedCache, batch: PagedBatch, scores: Optional[PagedScores], Q: int, O: int, LSE: Optional[int],
                    Hq: int, strides: PagedStrides, max_q: int, path: int, scale: float, causal: bool,
                    workspace: Optional[int], workspace_bytes: int, stream: int) -> int:
    """C ``fa_fwd_paged_ex``: descriptions, raw device addresses and sizes; returns the status code."""
    return int(_lib.load().fa_fwd_paged_ex(cache, batch, scores, Q, O, LSE, Hq, strides, max_q, path, float(scale),
                                           int(bool(causal)), workspace, int(workspace_bytes), stream))


def fa_fwd_paged_ex_workspace_bytes(B: int, T: int, max_keys: int, Hq: int, Hkv: int, d_qk: int, d_v: int, type: int,
                                    max_q: int, path: int = FA_PAGED_AUTO) -> int:
    """C ``fa_fwd_paged_ex_workspace_bytes`` (``max_keys``: blocks of the table times page size)."""
    return int(_lib.load().fa_fwd_paged_ex_workspace_bytes(B, T, max_keys, Hq, Hkv, d_qk, d_v, type, max_q, path))


# What a call costs on the host bounds the smallest problems (one head S256 d64: a 4.7 us kernel in a call
# of 11.9 us, of which the C entry point and its launch are 4.2). So a call on torch's current stream asks
# for the raw handle only (0.1 us against 2.1 for a Stream object; the function has no public name in torch,
# whose compiled graphs call it for the same purpose), the device is switched only where it is not the current
# one (0.3 against 1.4), and the usual case of the checks is one expression.

def _stream(stream, device):
    """(torch stream, raw handle) for ``stream``. None is torch's current stream of ``device``, given as
    (None, handle): workspaces allocated for the call belong to that stream already. A torch.cuda.Stream
    is used as is; a raw integer handle is wrapped in torch.cuda.ExternalStream so that workspaces can be
    recorded on it (the caching allocator then does not hand them out again before the kernels on that
    stream have run)."""
    import torch

    if stream is None:
        return None, torch._C._cuda_getCurrentRawStream(device.index)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    elif stream.device != torch.device(device):
        raise ValueError(f"stream is on {stream.device}, the tensors on {device}")
    return stream, stream.cuda_stream


_NO_SWITCH = contextlib.nullcontext()


def _on_device(device):
    """Context in which ``device`` is the current one."""
    import torch

    return _NO_SWITCH if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _workspace(nbytes, device, stream):
    """A workspace from torch's allocator for kernels on ``stream`` (None: the current one of ``device``,
    which is the current device)."""
    import torch

    ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    if stream is not None:
        ws.record_stream(stream)  # not reused before the kernels on `stream` ran
    return ws


def _check_qkv(q, k, v):
    import torch

    T, bf16 = torch.Tensor, torch.bfloat16
    if not (isinstance(q, T) and isinstance(k, T) and isinstance(v, T) and q.dim() == k.dim() == v.dim() == 4
            and q.dtype == bf16 and k.dtype == bf16 and v.dtype == bf16 and q.is_cuda and k.is_cuda and v.is_cuda
            and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
        for name, t in (("q", q), ("k", k), ("v", v)):
            if not isinstance(t, T) or t.dim() != 4:
                raise ValueError(f"{name} must be a 4-d torch tensor (BHSD)")
            if t.dtype != bf16:
                raise ValueError(f"{name} must be bfloat16")
            if not t.is_cuda:
                raise ValueError(f"{name} must be on a GPU")
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
    if not (q.device == k.device == v.device):
        raise ValueError("q, k, v must be on the same device")
    B, Hq, Sq, dqk = q.shape
    Bk, Hkv, Sk, dk = k.shape
    Bv, Hv, Sv, dv = v.shape
    if Bk != B or dk != dqk or Bv != Bk or Hv != Hkv or Sv != Sk:
        raise ValueError(f"inconsistent shapes q{tuple(q.shape)} k{tuple(k.shape)} v{tuple(v.shape)}")
    return B, Hq, Hkv, Sq, Sk, dqk, dv


def forward_unfused(q, k, v, causal: bool = False, scale: Optional[float] = None, return_lse: bool = False,
                    workspace=None, stream=None):
    """Attention forward through the unfused layer-by-layer path (``fa_fwd_unfused``): scores, mask +
    softmax and P V as three kernels with S and P spilled to device memory in bf16. Same tensors and
    defaults as :func:`forward`. ``workspace`` is a uint8 CUDA tensor for the spill buffer (default: one
    sized for the whole problem from torch's allocator; a smaller one runs the problem in chunks)."""
    import torch

    B, Hq, Hkv, Sq, Sk, dqk, dv = _check_qkv(q, k, v)
    if scale is None:
        scale = 1.0 / math.sqrt(dqk)
    out = torch.empty((B, Hq, Sq, dv), dtype=torch.bfloat16, device=q.device)
    lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device) if return_lse else None
    stream, handle = _stream(stream, q.device)
    with _on_device(q.device):
        if workspace is None:
            nbytes = fa_lbl_workspace_bytes(B, Hq, Sq, Sk)
            workspace = _workspace(max(nbytes, 16), q.device, stream)
        st = fa_fwd_unfused(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                            lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, Sk, dqk, dv, scale, causal,
                            workspace.data_ptr(), workspace.numel() * workspace.element_size(), handle)
    if st != FA_OK:
        if st in (FA_ERR_NULL_POINTER, FA_ERR_BAD_SHAPE, FA_ERR_UNSUPPORTED, FA_ERR_BAD_SCALE, FA_ERR_WORKSPACE):
            raise ValueError(f"fa_fwd_unfused rejected the arguments: {fa_status_str(st)}")
        raise FaError(st)
    return (out, lse) if return_lse else out


def forward(q, k, v, causal: bool = False, scale: Optional[float] = None, return_lse: bool = False,
            out=None, lse=None, stream=None, n_split=1, decode: bool = False):
    """Attention forward over contiguous bf16 BHSD torch tensors on one GPU.

    q [B, Hq, Sq, d_qk], k [B, Hkv, Sk, d_qk], v [B, Hkv, Sk, d_v]; returns O [B, Hq, Sq, d_v] (bf16)
    and, with ``return_lse``, LSE [B, Hq, Sq] (float32, natural log). ``scale`` defaults to
    1/sqrt(d_qk). ``n_split`` > 1 runs split mode (``fa_fwd_split``) with that many key-range parts
    per query block and a workspace from torch's allocator; ``n_split="auto"`` takes the count
    ``fa_fwd_split_parts`` suggests for the device. ``decode=True`` runs the decode-shaped path
    (``fa_fwd_decode``, for few query rows per key/value head) with ``n_split`` parts ("auto":
    ``fa_fwd_decode_parts``). The kernels are enqueued on ``stream`` (default: torch's current
    stream); the call does not synchronise.
    """
    import torch

    B, Hq, Hkv, Sq, Sk, dqk, dv = _check_qkv(q, k, v)
    if scale is None:
        scale = 1.0 / math.sqrt(dqk)
    if out is None:
        out = torch.empty((B, Hq, Sq, dv), dtype=torch.bfloat16, device=q.device)
    elif (not isinstance(out, torch.Tensor) or out.shape != (B, Hq, Sq, dv) or out.dtype != torch.bfloat16
          or not out.is_contiguous()):
        raise ValueError("out must be a contiguous bf16 tensor of shape [B, Hq, Sq, d_v]")
    elif out.device != q.device:
        raise ValueError(f"out must be on the inputs' device {q.device}, not {out.device}")
    if return_lse and lse is None:
        lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device)
    if lse is not None:
        if (not isinstance(lse, torch.Tensor) or lse.shape != (B, Hq, Sq) or lse.dtype != torch.float32
                or not lse.is_contiguous()):
            raise ValueError("lse must be a contiguous float32 tensor of shape [B, Hq, Sq]")
        if lse.device != q.device:
            raise ValueError(f"lse must be on the inputs' device {q.device}, not {lse.device}")
    stream, handle = _stream(stream, q.device)
    name = "fa_fwd_ex"
    if decode:
        n_cu = torch.cuda.get_device_properties(q.device).multi_processor_count
        parts = fa_fwd_decode_parts(n_cu, B, Hq, Hkv, Sq, Sk) if n_split == "auto" else int(n_split)
        with _on_device(q.device):
            nbytes = fa_fwd_split_workspace_bytes(B, Hq, Sq, dv, parts)
            ws = _workspace(max(nbytes, 1), q.device, stream)
            st = fa_fwd_decode(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                               lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, Sk, dqk, dv, scale, causal,
                               parts, ws.data_ptr(), nbytes, handle)
        if st != FA_OK:
            if st in (FA_ERR_NULL_POINTER, FA_ERR_BAD_SHAPE, FA_ERR_UNSUPPORTED, FA_ERR_BAD_SCALE, FA_ERR_WORKSPACE):
                raise ValueError(f"fa_fwd_decode rejected the arguments: {fa_status_str(st)}")
            raise FaError(st)
        return (out, lse) if return_lse else out
    if n_split == "auto":
        n_cu = torch.cuda.get_device_properties(q.device).multi_processor_count
        n_split = fa_fwd_split_parts(n_cu, B, Hq, Sq, Sk, dqk, dv, causal)
    with _on_device(q.device):
        if n_split is not None and int(n_split) > 1:
            name = "fa_fwd_split"
            nbytes = fa_fwd_split_workspace_bytes(B, Hq, Sq, dv, int(n_split))
            ws = _workspace(max(nbytes, 1), q.device, stream)
            st = fa_fwd_split(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                              lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, Sk, dqk, dv, scale,
                              causal, int(n_split), ws.data_ptr(), nbytes, handle)
        else:
            st = fa_fwd_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                           lse.data_ptr() if lse is not None else None,
                           B, Hq, Hkv, Sq, Sk, dqk, dv, scale, causal, handle)
    if st != FA_OK:
        if st in (FA_ERR_NULL_POINTER, FA_ERR_BAD_SHAPE, FA_ERR_UNSUPPORTED, FA_ERR_BAD_SCALE, FA_ERR_WORKSPACE):
            raise ValueError(f"{name} rejected the arguments: {fa_status_str(st)}")
        raise FaError(st)
    return (out, lse) if return_lse else out


# The paged calls are short (an append of one token takes the GPU 3.4 us), so their checks are, as above, one expression
# each where everything is as it should be, and what is wrong is looked for only then. A call on another stream or
# device than the current one makes that the current one and starts again, so that new tensors belong to the stream whose
# kernels use them.

def _elsewhere(stream, device):
    """Context for a call that is not on the current stream of the current device; None if it is."""
    import torch

    if stream is None:
        return None if torch._C._cuda_getDevice() == device else torch.cuda.device(device)
    return torch.cuda.stream(_stream(stream, torch.device("cuda", device))[0])


def _rows_error(name, t, shape, device, writes):
    """What is wrong with a packed [T, H, d] bf16 tensor."""
    import torch

    if not isinstance(t, torch.Tensor) or t.dim() != 3 or t.dtype != torch.bfloat16:
        return ValueError(f"{name} must be a 3-d bfloat16 torch tensor [tokens, heads, d]")
    if not t.is_cuda or t.get_device() != device:
        return ValueError(f"{name} must be on the cache's device cuda:{device}, not {t.device}")
    if t.shape != shape:
        return ValueError(f"{name} must have shape {list(shape)}, not {list(t.shape)}")
    if t.stride(2) != 1:
        return ValueError(f"the elements of a head of {name} must lie one after the other")
    return ValueError(f"rows of {name} overlap" if writes else f"{name} is not supported")


def _rows(name, t, shape, device, bf16, writes=False):
    """Checks a packed [T, H, d] bf16 tensor with any strides of T and H (rows apart, where it is written to) and
    returns them, 0 for a dimension of one."""
    try:
        st, sh, sd = t.stride()
        if t.shape != shape or t.dtype != bf16 or t.get_device() != device or sd != 1:
            raise _rows_error(name, t, shape, device, writes)
    except (AttributeError, TypeError, ValueError):
        raise _rows_error(name, t, shape, device, writes) from None
    T, H, d = shape
    if T <= 1:
        st = 0
    if H <= 1:
        sh = 0
    if writes and not ((sh >= d or H <= 1) and (st >= (H - 1) * sh + d or T <= 1)
                       or (st >= d or T <= 1) and (sh >= (T - 1) * st + d or H <= 1)):
        raise _rows_error(name, t, shape, device, writes)
    return st, sh


def _paged_error(k_cache, v_cache, block_table, kv_lens, q_starts, k_scale, v_scale):
    """What is wrong with a paged cache or its batch."""
    import torch

    tensor = torch.Tensor
    for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
        if not isinstance(t, tensor) or t.dim() != 4 or t.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
            return ValueError(f"{name} must be a 4-d torch tensor [pages, heads, page_size, d], bfloat16 or float8_e4m3fn")
        if not t.is_cuda:
            return ValueError(f"{name} must be on a GPU")
        if t.stride(3) != 1:
            return ValueError(f"the elements of a head of {name} must lie one after the other")
    device = k_cache.device
    if k_cache.dtype != v_cache.dtype or k_cache.shape[:3] != v_cache.shape[:3] or v_cache.device != device:
        return ValueError("k_cache and v_cache must agree in type, device, pages, heads and page size")
    for name, t, dim in (("block_table", block_table, 2), ("kv_lens", kv_lens, 1), ("q_starts", q_starts, 1)):
        if not isinstance(t, tensor) or t.dim() != dim or t.dtype != torch.int32:
            return ValueError(f"{name} must be a {dim}-d int32 torch tensor")
        if t.device != device:
            return ValueError(f"{name} must be on the cache's device {device}, not {t.device}")
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            return ValueError(f"the entries of {name} must lie one after the other")
    for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
        if t is None:
            continue
        if k_cache.dtype != torch.float8_e4m3fn:
            return ValueError(f"{name} goes with a float8_e4m3fn cache")
        if not isinstance(t, tensor) or t.dtype != torch.float32 or t.shape != (k_cache.shape[1],) or not t.is_contiguous():
            return ValueError(f"{name} must be a contiguous float32 tensor [heads]")
        if t.device != device:
            return ValueError(f"{name} must be on the cache's device {device}, not {t.device}")
    return ValueError(f"block_table [B, blocks], kv_lens [B] and q_starts [B + 1] do not agree: "
                      f"{list(block_table.shape)}, {list(kv_lens.shape)}, {list(q_starts.shape)}")


def _scale(t, heads, device, float32):
    """Address of a scale tensor; None where it is not one."""
    if t.dtype != float32 or t.shape != (heads,) or t.get_device() != device or not t.is_contiguous():
        return None
    return t.data_ptr()


def _paged(k_cache, v_cache, block_table, kv_lens, q_starts, k_scale, v_scale, T, torch):
    """Checks a paged cache and its batch; the device's index and their C descriptions."""
    try:
        (pages, hkv, page, dqk), (kp, kh, ks, kd) = k_cache.shape, k_cache.stride()
        vpages, vhkv, vpage, dv = v_cache.shape
        vp, vh, vs, vd = v_cache.stride()
        (B, blocks), (bs, be) = block_table.shape, block_table.stride()
        (lens,), (starts,) = kv_lens.shape, q_starts.shape
        device, dtype, i32 = k_cache.get_device(), k_cache.dtype, torch.int32
        fp8 = dtype == torch.float8_e4m3fn
        ok = (device >= 0 and (fp8 or dtype == torch.bfloat16) and v_cache.dtype == dtype and vpages == pages
              and vhkv == hkv and vpage == page and kd == 1 and vd == 1 and lens == B and starts == B + 1
              and v_cache.get_device() == device and block_table.dtype == i32 and kv_lens.dtype == i32
              and q_starts.dtype == i32 and block_table.get_device() == device and kv_lens.get_device() == device
              and q_starts.get_device() == device and (be == 1 or blocks <= 1) and (B <= 1 or kv_lens.stride(0) == 1)
              and (B == 0 or q_starts.stride(0) == 1))
        ksp = vsp = None
        if ok and k_scale is not None:
            ksp = _scale(k_scale, hkv, device, torch.float32)
            ok = fp8 and ksp is not None
        if ok and v_scale is not None:
            vsp = _scale(v_scale, hkv, device, torch.float32)
            ok = fp8 and vsp is not None
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        raise _paged_error(k_cache, v_cache, block_table, kv_lens, q_starts, k_scale, v_scale)
    if pages <= 1:  # the stride of a dimension of one means nothing
        kp = vp = 0
    if hkv <= 1:
        kh = vh = 0
    return (device, PagedCache(k_cache.data_ptr(), v_cache.data_ptr(), ksp, vsp, kp, kh, ks, vp, vh, vs, pages, page, hkv, dqk,
                               dv, 1 if fp8 else 0),
            PagedBatch(block_table.data_ptr(), bs if B > 1 else 0, kv_lens.data_ptr(), q_starts.data_ptr(), B, blocks, T),
            B, blocks * page, hkv, dqk, dv, 1 if fp8 else 0)


def _raise(name, st):
    if st in (FA_ERR_NULL_POINTER, FA_ERR_BAD_SHAPE, FA_ERR_UNSUPPORTED, FA_ERR_BAD_SCALE, FA_ERR_WORKSPACE):
        raise ValueError(f"{name} rejected the arguments: {fa_status_str(st)}")
    raise FaError(st)


def kv_append(k, v, k_cache, v_cache, block_table, kv_lens, q_starts, q=None, q_out=None, cos_sin=None,
              rot_begin: int = 0, interleaved: bool = False, k_scale=None, v_scale=None, stream=None, positions=None,
              pair_axes=None):
    """Write the keys and values of new tokens to a paged cache, turning keys and queries by their positions.

    k [T, Hkv, d_qk] and v [T, Hkv, d_v] (bf16) hold the packed new tokens; those of sequence b are
    ``q_starts[b]`` to ``q_starts[b + 1] - 1``, the last of its ``kv_lens[b]`` keys. k_cache and v_cache are
    [pages, Hkv, page_size, d] in bf16 or float8_e4m3fn (an element then stands for itself times ``k_scale[h]``,
    ``v_scale[h]``); ``block_table`` [B, blocks] names every sequence's pages in order (int32, like the lengths). Any strides
    of the outer dimensions. ``cos_sin`` float32 [positions, rot_dim] holds the cosines and then the sines of a
    position's angles; dims ``rot_begin`` to ``rot_begin + rot_dim - 1`` of k and q turn, in pairs (c, c + rot_dim / 2) or,
    ``interleaved``, (2c, 2c + 1). With ``q`` [T, Hq, d_qk] returns the turned queries, in ``q_out`` (``q`` itself, or apart
    from it in memory) or a new tensor; rows of tokens that belong to no sequence are left as they were, so a new tensor's
    hold anything.

    ``positions`` (int32 [T], or [T, axes] with ``pair_axes`` uint8 [rot_dim / 2], the axis of each pair; any strides)
    are where the tokens stand if not at their places among their sequence's keys: drafted tokens (:func:`tree_mask`), images
    and video (time, height, width). A position outside the table counts as its first or last row.

    The kernel is enqueued on ``stream`` (default: torch's current stream; a new tensor belongs to that
    stream); the call does not synchronise, and reads no array on the host."""
    import torch

    bf16 = torch.bfloat16
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise _rows_error("k", k, (), 0, False)
    T = k.shape[0]
    device, cache, batch, _, _, hkv, dqk, dv, _ = _paged(k_cache, v_cache, block_table, kv_lens, q_starts, k_scale, v_scale, T,
                                                         torch)
    kt, kh = _rows("k", k, (T, hkv, dqk), device, bf16)
    vt, vh = _rows("v", v, (T, hkv, dv), device, bf16)
    n_pos = rot = 0
    table = qp = op = None
    if cos_sin is not None:
        if (not isinstance(cos_sin, torch.Tensor) or cos_sin.dim() != 2 or cos_sin.dtype != torch.float32
                or not cos_sin.is_contiguous()):
            raise ValueError("cos_sin must be a contiguous float32 tensor [positions, rotated dims]")
        if cos_sin.get_device() != device:
            raise ValueError(f"cos_sin must be on the cache's device cuda:{device}, not {cos_sin.device}")
        n_pos, rot = cos_sin.shape
        table = cos_sin.data_ptr()
    at = None
    if positions is not None or pair_axes is not None:
        if cos_sin is None:
            raise ValueError("positions and pair_axes go with cos_sin")
        at = _positions(positions, pair_axes, (T,), rot, device)
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return kv_append(k, v, k_cache, v_cache, block_table, kv_lens, q_starts, q, q_out, cos_sin, rot_begin, interleaved,
                             k_scale, v_scale, None, positions, pair_axes)
    hq = qt = qh = ot = oh = 0
    if q is not None:
        hq = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else -1
        qt, qh = _rows("q", q, (T, hq, dqk), device, bf16, q_out is q)
        qp = q.data_ptr()
        if q_out is None:
            q_out = torch.empty_like(q) if q.is_contiguous() else q.new_empty((T, hq, dqk))
            ot, oh = hq * dqk, dqk
        elif q_out is q:
            ot, oh = qt, qh
        else:
            ot, oh = _rows("q_out", q_out, (T, hq, dqk), device, bf16, True)
            # Bytes from the first element to behind the last, of q and of q_out.
            q0, o0, n, m = q.data_ptr(), q_out.data_ptr(), T - 1, hq - 1
            if (T > 0 and hq > 0 and q0 < o0 + 2 * (n * ot + m * oh + dqk) and o0 < q0 + 2 * (n * qt + m * qh + dqk)
                    and (q0, qt, qh) != (o0, ot, oh)):
                raise ValueError("q_out must be q itself or lie before or behind it in memory")
        op = q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out goes with q")
    strides, stream = AppendStrides(qt, qh, ot, oh, kt, kh, vt, vh), torch._C._cuda_getCurrentRawStream(device)
    inter = 1 if interleaved else 0
    if at is None:
        st = _lib.load().fa_kv_append(cache, batch, k.data_ptr(), v.data_ptr(), qp, op, hq, strides, table, n_pos,
                                      int(rot_begin), rot, inter, stream)
    else:
        st = _lib.load().fa_kv_append_at(cache, batch, k.data_ptr(), v.data_ptr(), qp, op, hq, strides, at, table, n_pos,
                                         int(rot_begin), rot, inter, stream)
    if st != FA_OK:
        _raise("fa_kv_append" if at is None else "fa_kv_append_at", st)
    return q_out


def _positions(positions, pair_axes, tokens, rot, device):
    """The C description of positions [*tokens] or [*tokens, axes] and of the axes of the pairs."""
    import torch

    n = len(tokens)
    if (not isinstance(positions, torch.Tensor) or positions.dtype != torch.int32 or (shape := positions.shape)[:n] != tokens
            or len(shape) > n + 1):
        raise ValueError(f"positions must be an int32 tensor of shape {list(tokens)} or {list(tokens)} + [axes]")
    if positions.get_device() != device:
        raise ValueError(f"positions must be on the device cuda:{device}, not {positions.device}")
    strides = positions.stride()
    axes, axis = (shape[n], strides[n]) if len(shape) > n else (1, 0)
    where = None
    if pair_axes is not None:
        if (not isinstance(pair_axes, torch.Tensor) or pair_axes.dtype != torch.uint8 or pair_axes.shape != (rot // 2,)
                or not pair_axes.is_contiguous()):
            raise ValueError(f"pair_axes must be a contiguous uint8 tensor [{rot // 2}], an axis for each pair of turned dims")
        if pair_axes.get_device() != device:
            raise ValueError(f"pair_axes must be on the device cuda:{device}, not {pair_axes.device}")
        where = pair_axes.data_ptr()
    elif axes > 1:
        raise ValueError("positions of several axes need pair_axes")
    return Positions(positions.data_ptr(), where, strides[0] if n > 1 else 0, strides[n - 1], axis, axes)


def _apart(shape, strides):
    """Whether no two elements of a tensor share a place in memory."""
    reach = 1
    for st, n in sorted((st, n) for st, n in zip(strides, shape) if n > 1):
        if st < reach:
            return False
        reach += (n - 1) * st
    return True


def _rotate_strides(name, strides, B, H, S, d):
    """Strides of batches, heads and tokens of a [B, H, S, d] or [S, H, d] tensor, 0 for a dimension of one."""
    if len(strides) == 4:
        b, h, s, e = strides
    else:
        b, (s, h, e) = 0, strides
    if e != 1 and d > 1:
        raise ValueError(f"the elements of a head of {name} must lie one after the other")
    return (b if B > 1 else 0, h if H > 1 else 0, s if S > 1 else 0)


def rotate(x, cos_sin, positions=None, pair_axes=None, rot_begin: int = 0, interleaved: bool = False, inverse: bool = False,
           out=None, stream=None):
    """The position rotation of :func:`kv_append` for queries or keys x [B, H, S, d] or [T, H, d] (bf16, any strides of
    whole rows) that are in no cache, as :func:`forward` takes them: dims ``rot_begin`` to ``rot_begin + rot_dim - 1`` turn by the
    angles of ``cos_sin`` float32 [positions, rot_dim], the others are copied. ``inverse`` turns back; the
    gradient with respect to x is that of the output's gradient (to be called by the program: like all calls here, this one records
    nothing for autograd).

    ``positions`` int32 [B, S] or [B, S, axes] ([T] or [T, axes]; any strides, so one row may be expanded over the batch) with
    ``pair_axes`` as in :func:`kv_append`; default: token s stands at s. Returns ``out`` (x itself, or apart from it in
    memory) or a new contiguous tensor. The kernel is enqueued on ``stream`` (default: torch's current stream; a new tensor
    belongs to that stream); the call does not synchronise, and reads no array on the host."""
    import torch

    if not isinstance(x, torch.Tensor) or x.dim() not in (3, 4) or x.dtype != torch.bfloat16:
        raise ValueError("x must be a bfloat16 torch tensor [B, H, S, d] or [T, H, d]")
    if not x.is_cuda:
        raise ValueError("x must be on a GPU")
    device, shape = x.get_device(), x.shape
    if len(shape) == 4:
        B, H, S, d = shape
        tokens = (B, S)
    else:
        B, (S, H, d) = 1, shape
        tokens = (S,)
    xs = _rotate_strides("x", x.stride(), B, H, S, d)
    if (not isinstance(cos_sin, torch.Tensor) or cos_sin.dim() != 2 or cos_sin.dtype != torch.float32
            or not cos_sin.is_contiguous()):
        raise ValueError("cos_sin must be a contiguous float32 tensor [positions, rotated dims]")
    if cos_sin.get_device() != device:
        raise ValueError(f"cos_sin must be on x's device {x.device}, not {cos_sin.device}")
    n_pos, rot = cos_sin.shape
    at = None
    if positions is not None:
        at = _positions(positions, pair_axes, tokens, rot, device)
    elif pair_axes is not None:
        raise ValueError("pair_axes goes with positions")
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return rotate(x, cos_sin, positions, pair_axes, rot_begin, interleaved, inverse, out)
    if out is None:
        out = x.new_empty(shape)
        ys = (H * S * d, S * d, d) if len(shape) == 4 else (0, d, H * d)
    else:
        if out is not x and (not isinstance(out, torch.Tensor) or out.shape != shape or out.dtype != x.dtype
                             or out.get_device() != device):
            raise ValueError(f"out must be a bfloat16 tensor {list(shape)} on {x.device}")
        ys = xs if out is x else _rotate_strides("out", out.stride(), B, H, S, d)
        if out is not x and x.numel() > 0:
            # Bytes from the first element to behind the last, of x and of out.
            x0, o0 = x.data_ptr(), out.data_ptr()
            x1, o1 = (a + 2 * ((B - 1) * b + (H - 1) * h + (S - 1) * s + d) for a, (b, h, s) in ((x0, xs), (o0, ys)))
            if x0 < o1 and o0 < x1 and (x0, xs) != (o0, ys):
                raise ValueError("out must be x itself or lie before or behind it in memory")
        if not _apart((B, H, S, d), (*ys, 1)):
            raise ValueError("rows of out overlap")
    st = _lib.load().fa_rotate(x.data_ptr(), out.data_ptr(), B, H, S, d, RotateStrides(*xs, *ys), at, cos_sin.data_ptr(), n_pos,
                               int(rot_begin), rot, 1 if interleaved else 0, 1 if inverse else 0,
                               torch._C._cuda_getCurrentRawStream(device))
    if st != FA_OK:
        _raise("fa_rotate", st)
    return out


def _int32(name, t, dim, device):
    """Checks an int32 tensor of `dim` dimensions on the device (None: on some GPU) whose last dimension's entries lie one after
    the other; its shape."""
    import torch

    try:
        shape, at = t.shape, t.get_device()
        if (t.dtype == torch.int32 and len(shape) == dim and (at == device or device is None and at >= 0)
                and (t.stride(-1) == 1 or shape[-1] <= 1)):
            return shape
    except (AttributeError, TypeError):
        pass
    if not isinstance(t, torch.Tensor) or t.dim() != dim or t.dtype != torch.int32:
        raise ValueError(f"{name} must be a {dim}-d int32 torch tensor")
    if not t.is_cuda or (device is not None and t.get_device() != device):
        raise ValueError(f"{name} must be on {'a GPU' if device is None else f'the device cuda:{device}'}, not {t.device}")
    raise ValueError(f"the entries of {name} must lie one after the other")


def _spans(t):
    """Addresses of the first byte of a tensor of 4-byte elements and of that behind its last."""
    n = t.numel() and 1 + sum((m - 1) * s for m, s in zip(t.shape, t.stride()))
    return t.data_ptr(), t.data_ptr() + 4 * n


def _apart_from(name, out, others):
    """Refuses an output of 4-byte elements that shares memory with other tensors of such."""
    a, z = _spans(out)
    for other, t in others:
        b, y = _spans(t)
        if a < y and b < z:
            raise ValueError(f"{name} must not overlap {other}")


def tree_mask(parents, q_starts, kv_lens, words: Optional[int] = None, max_keys: Optional[int] = None, mask=None, positions=None,
              stream=None):
    """Mask and positions of trees of drafted tokens. ``parents`` int32 [T] (packed as in :func:`kv_append`, with its
    ``q_starts`` [B + 1] and ``kv_lens`` [B], which count the drafted tokens) holds the number of each token's parent among its
    sequence's new tokens, a smaller one than its own, or -1: it follows the cached keys. Returns (mask, positions): int32
    [T, ``words``], whose bit j % 32 of word j / 32 says whether the sequence's new token j is the token or one of its ancestors,
    for :func:`forward_paged`, and int32 [T], cached keys + ancestors, for :func:`kv_append`. ``words`` (up to 64) has to cover the
    largest tree: tokens from 32 * ``words`` on have no bit, not even their own. The default, that of ``mask`` where one is given,
    covers any tree of the T tokens (2048 at most); a program that knows its largest tree saves memory by naming it. Rows of
    tokens that belong to no sequence are left as they were, so new tensors' hold anything; those of a sequence of more than 4096
    new tokens too, but in new tensors they are zeros: such tokens see the cached keys alone.

    ``max_keys`` clamps ``kv_lens`` (default 2^30). The kernel is enqueued on ``stream`` (default: torch's current stream; new
    tensors belong to that stream); the call does not synchronise, and reads no array on the host."""
    import torch

    (T,) = _int32("parents", parents, 1, None)
    device = parents.get_device()
    (starts,) = _int32("q_starts", q_starts, 1, device)
    (B,) = _int32("kv_lens", kv_lens, 1, device)
    if words is not None:
        words = int(words)
    elif mask is not None:
        words = _int32("mask", mask, 2, device)[1]
    else:
        words = min(max((T + 31) // 32, 1), FA_TREE_WORDS)
    if starts != B + 1:
        raise ValueError(f"q_starts [B + 1] and kv_lens [B] do not agree: {list(q_starts.shape)}, {list(kv_lens.shape)}")
    if not 1 <= words <= FA_TREE_WORDS:
        raise ValueError(f"words must be 1 to {FA_TREE_WORDS}, not {words}")
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return tree_mask(parents, q_starts, kv_lens, words, max_keys, mask, positions)
    new_mask = mask is None
    new = parents.new_empty if T <= FA_TREE_TOKENS else parents.new_zeros
    if new_mask:
        mask = new((T, words))
    else:
        if _int32("mask", mask, 2, device) != (T, words) or (T > 1 and mask.stride(0) < words):
            raise ValueError(f"mask must have shape {[T, words]}, its rows apart")
    if positions is None:
        positions = new(T)
    else:
        if _int32("positions", positions, 1, device) != (T,):
            raise ValueError(f"positions must have shape {[T]}")
        _apart_from("positions", positions, (("parents", parents), ("q_starts", q_starts), ("kv_lens", kv_lens), ("mask", mask)))
    if not new_mask:
        _apart_from("mask", mask, (("parents", parents), ("q_starts", q_starts), ("kv_lens", kv_lens)))
    st = _lib.load().fa_tree_mask(parents.data_ptr(), q_starts.data_ptr(), kv_lens.data_ptr(), B, T,
                                  1 << 30 if max_keys is None else int(max_keys), mask.data_ptr(), words,
                                  mask.stride(0) if T > 1 else words, positions.data_ptr(),
                                  torch._C._cuda_getCurrentRawStream(device))
    if st != FA_OK:
        _raise("fa_tree_mask", st)
    return mask, positions


def _cache(k_cache, v_cache, device):
    """Checks a paged cache alone; its C description."""
    import torch

    try:
        (pages, hkv, page, dqk), (kp, kh, ks, kd) = k_cache.shape, k_cache.stride()
        (vpages, vhkv, vpage, dv), (vp, vh, vs, vd) = v_cache.shape, v_cache.stride()
        fp8 = k_cache.dtype == torch.float8_e4m3fn
        ok = ((fp8 or k_cache.dtype == torch.bfloat16) and v_cache.dtype == k_cache.dtype and k_cache.get_device() == device
              and v_cache.get_device() == device and kd == 1 and vd == 1 and (vpages, vhkv, vpage) == (pages, hkv, page))
    except (AttributeError, TypeError, ValueError):
        ok = False
    if not ok:
        for name, t in (("k_cache", k_cache), ("v_cache", v_cache)):
            if not isinstance(t, torch.Tensor) or t.dim() != 4 or t.dtype not in (torch.bfloat16, torch.float8_e4m3fn):
                raise ValueError(f"{name} must be a 4-d torch tensor [pages, heads, page_size, d], bfloat16 or float8_e4m3fn")
            if t.get_device() != device:
                raise ValueError(f"{name} must be on the device cuda:{device}, not {t.device}")
            if t.stride(3) != 1:
                raise ValueError(f"the elements of a head of {name} must lie one after the other")
        raise ValueError("k_cache and v_cache must agree in type, pages, heads and page size")
    if pages <= 1:  # the stride of a dimension of one means nothing
        kp = vp = 0
    if hkv <= 1:
        kh = vh = 0
    return PagedCache(k_cache.data_ptr(), v_cache.data_ptr(), None, None, kp, kh, ks, vp, vh, vs, pages, page, hkv, dqk, dv,
                      1 if fp8 else 0)


def kv_compact(k_cache, v_cache, block_table, kv_lens, q_starts, kept, n_kept, new_lens=None, stream=None):
    """Close up the new tokens that each sequence keeps, such as the accepted ones of a drafted tree: of the new tokens of
    sequence b, which :func:`kv_append` has written, number ``kept[b, i]`` moves to the i-th place behind the cached keys, for i <
    ``n_kept[b]``. ``kept`` int32 [B, m] holds increasing numbers, ``n_kept`` is int32 [B]; cache, table and lengths as in
    :func:`kv_append`. Returns int32 [B], ``kv_lens - new + n_kept``, in ``new_lens`` (not ``kv_lens`` itself) or a new tensor. Keys
    keep the rotation that they were written with.

    A buffer that holds the caches of all layers, [pages, layers, Hkv, page_size, d], closes up in one call as
    ``k_all.flatten(1, 2)``. The kernel is enqueued on ``stream`` (default: torch's current stream; a new tensor belongs to
    that stream); the call does not synchronise, and reads no array on the host."""
    import torch

    device, cache, batch, B, *_ = _paged(k_cache, v_cache, block_table, kv_lens, q_starts, None, None, 0, torch)
    rows, most = _int32("kept", kept, 2, device)
    if rows != B or _int32("n_kept", n_kept, 1, device) != (B,):
        raise ValueError(f"kept [B, m] and n_kept [B] do not agree with B = {B}: {list(kept.shape)}, {list(n_kept.shape)}")
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return kv_compact(k_cache, v_cache, block_table, kv_lens, q_starts, kept, n_kept, new_lens)
    if new_lens is None:
        new_lens = kv_lens.new_empty(B)
    else:
        if _int32("new_lens", new_lens, 1, device) != (B,):
            raise ValueError(f"new_lens must have shape {[B]}")
        _apart_from("new_lens", new_lens, (("kv_lens", kv_lens), ("q_starts", q_starts), ("kept", kept), ("n_kept", n_kept),
                                           ("block_table", block_table)))
    st = _lib.load().fa_kv_compact(cache, batch, kept.data_ptr(), kept.stride(0) if B > 1 else 0, most,
                                   n_kept.data_ptr(), new_lens.data_ptr(), torch._C._cuda_getCurrentRawStream(device))
    if st != FA_OK:
        _raise("fa_kv_compact", st)
    return new_lens


def kv_copy(k_cache, v_cache, src, dst, stream=None):
    """Copy pages of a paged cache: page ``src[i]`` to page ``dst[i]`` (int32 [n]), keys and values of all heads, for sequences
    that fork and go on in pages of their own. A pair with a page number that is none of the cache's does nothing; no page
    should be copied to twice, or copied both to and from. All layers of one buffer are copied as ``k_all.flatten(1, 2)``, see
    :func:`kv_compact`. The kernel is enqueued on ``stream`` (default: torch's current stream); the call does not
    synchronise, and reads no array on the host."""
    import torch

    (n,) = _int32("src", src, 1, None)
    device = src.get_device()
    if _int32("dst", dst, 1, device) != (n,):
        raise ValueError(f"src and dst must have as many pages: {list(src.shape)}, {list(dst.shape)}")
    cache = _cache(k_cache, v_cache, device)
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return kv_copy(k_cache, v_cache, src, dst)
    st = _lib.load().fa_kv_copy(cache, src.data_ptr(), dst.data_ptr(), n, torch._C._cuda_getCurrentRawStream(device))
    if st != FA_OK:
        _raise("fa_kv_copy", st)


def forward_paged(q, k_cache, v_cache, block_table, kv_lens, q_starts, max_q: Optional[int] = None, causal: bool = True,
                  scale: Optional[float] = None, k_scale=None, v_scale=None, return_lse: bool = False, out=None, lse=None,
                  workspace=None, stream=None, path: Optional[str] = None, softcap: Optional[float] = None, slopes=None,
                  window: Optional[int] = None, prefix_lens=None, tree_mask=None):
    """Attention of the new tokens q [T, Hq, d_qk] over a paged cache (see :func:`kv_append` for the cache and the
    batch, whose new tokens are in the cache already): returns O [T, Hq, d_v] (bf16) and, with ``return_lse``, LSE
    [T, Hq] (float32, natural log). Token i of the n new ones of sequence b sees the keys up to its position
    ``kv_lens[b] - n + i`` (all ``kv_lens[b]`` where not ``causal``). ``max_q``, the most new tokens of one sequence, helps to
    choose the kernels (default: not known), ``path`` ("few", "many") chooses them: for single tokens and short prompts, or for
    longer ones; the results are right for any. Rows of tokens that belong to no
    sequence are left as they were, so a new tensor's hold anything.

    Scores x = scale * q . k may be changed and keys hidden, for the token at position p and key j: ``softcap`` makes x softcap
    * tanh(x / softcap) (up to 1024); ``slopes`` (float32 [Hq]) takes slopes[h] * abs(p - j) off (slopes beyond +-5e28 count as
    that); ``window`` hides keys with abs(p - j) >= window; ``prefix_lens`` (int32 [B]) shows all tokens of a sequence its first
    keys, whatever window and causal masking say; ``tree_mask`` (int32 [T, words], see :func:`tree_mask`) says which of their
    sequence's new tokens drafted ones see, beside all cached keys (causal calls without slopes, window and prefix).

    ``scale`` defaults to 1/sqrt(d_qk). ``workspace`` is a CUDA tensor of ``fa_fwd_paged_workspace_bytes`` (with any of the
    options above ``fa_fwd_paged_ex_workspace_bytes``; default: from
    torch's allocator). The kernels are enqueued on ``stream`` (default: torch's current stream; new tensors belong to that
    stream); the call does not synchronise, and reads no array on the host: captured into a graph, it serves
    whatever lengths the arrays hold at a replay."""
    import torch

    bf16 = torch.bfloat16
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise _rows_error("q", q, (), 0, False)
    T, hq = q.shape[:2]
    device, cache, batch, B, max_keys, hkv, dqk, dv, type = _paged(k_cache, v_cache, block_table, kv_lens, q_starts, k_scale,
                                                                   v_scale, T, torch)
    qt, qh = _rows("q", q, (T, hq, dqk), device, bf16)
    if scale is None:
        scale = 1.0 / math.sqrt(dqk) if dqk else 1.0
    if max_q is None:
        max_q = 0
    max_q = int(max_q)
    way = 0
    if path is not None:
        if path not in ("few", "many"):
            raise ValueError(f'path must be "few", "many" or None, not {path!r}')
        way = FA_PAGED_FEW if path == "few" else FA_PAGED_MANY
    scores = None
    if not (softcap is None and slopes is None and window is None and prefix_lens is None and tree_mask is None):
        scores = _scores(softcap, slopes, window, prefix_lens, tree_mask, T, hq, B, device)
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return forward_paged(q, k_cache, v_cache, block_table, kv_lens, q_starts, max_q, causal, scale, k_scale, v_scale,
                                 return_lse, out, lse, workspace, None, path, softcap, slopes, window, prefix_lens, tree_mask)
    if out is not None:
        ot, oh = _rows("out", out, (T, hq, dv), device, bf16, True)
    else:
        out = torch.empty_like(q) if dqk == dv and q.is_contiguous() else q.new_empty((T, hq, dv))
        ot, oh = hq * dv, dv
    if lse is not None:
        if (not isinstance(lse, torch.Tensor) or lse.shape != (T, hq) or lse.dtype != torch.float32
                or not lse.is_contiguous()):
            raise ValueError("lse must be a contiguous float32 tensor [T, Hq]")
        if lse.get_device() != device:
            raise ValueError(f"lse must be on the cache's device cuda:{device}, not {lse.device}")
    elif return_lse:
        lse = q.new_empty((T, hq), dtype=torch.float32)
    lib, ws = _lib.load(), None
    if workspace is None:
        size = lib.fa_fwd_paged_workspace_bytes if scores is None else lib.fa_fwd_paged_ex_workspace_bytes
        nbytes = size(B, T, max_keys, hq, hkv, dqk, dv, type, max_q, way)
        if nbytes > 0:
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
            ws = workspace.data_ptr()
    elif not isinstance(workspace, torch.Tensor) or workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{device}")
    else:
        nbytes, ws = workspace.numel() * workspace.element_size(), workspace.data_ptr()
    lsep, strides, stream = None if lse is None else lse.data_ptr(), PagedStrides(qt, qh, ot, oh), \
        torch._C._cuda_getCurrentRawStream(device)
    if scores is None:
        st = lib.fa_fwd_paged(cache, batch, q.data_ptr(), out.data_ptr(), lsep, hq, strides, max_q, way, scale,
                              1 if causal else 0, ws, nbytes, stream)
    else:
        st = lib.fa_fwd_paged_ex(cache, batch, scores, q.data_ptr(), out.data_ptr(), lsep, hq, strides, max_q, way, scale,
                                 1 if causal else 0, ws, nbytes, stream)
    if st != FA_OK:
        _raise("fa_fwd_paged" if scores is None else "fa_fwd_paged_ex", st)
    return (out, lse) if return_lse else out


def _scores(softcap, slopes, window, prefix_lens, tree_mask, T, hq, B, device):
    """The C description of how scores are changed and keys hidden."""
    import torch

    cap = wide = words = stride = 0
    sp = pp = mp = None
    if softcap is not None:
        if not (0 < softcap <= FA_MAX_SOFTCAP and ctypes.c_float(softcap).value > 0):  # 0 would be no cap
            raise ValueError(f"softcap must be above 0 and at most {FA_MAX_SOFTCAP:g}, not {softcap}")
        cap = softcap
    if window is not None:
        if not 0 < window < 1 << 31:
            raise ValueError(f"window must be at least 1 key, not {window}")
        wide = window
    if slopes is not None:
        if (not isinstance(slopes, torch.Tensor) or slopes.dtype != torch.float32 or slopes.shape != (hq,)
                or not slopes.is_contiguous()):
            raise ValueError(f"slopes must be a contiguous float32 tensor [{hq}]")
        if slopes.get_device() != device:
            raise ValueError(f"slopes must be on the cache's device cuda:{device}, not {slopes.device}")
        sp = slopes.data_ptr()
    if prefix_lens is not None:
        if _int32("prefix_lens", prefix_lens, 1, device) != (B,):
            raise ValueError(f"prefix_lens must have shape {[B]}, not {list(prefix_lens.shape)}")
        pp = prefix_lens.data_ptr()
    if tree_mask is not None:
        rows, words = _int32("tree_mask", tree_mask, 2, device)
        if rows != T or not 1 <= words <= FA_TREE_WORDS:
            raise ValueError(f"tree_mask must have shape [{T}, 1 to {FA_TREE_WORDS}], not {list(tree_mask.shape)}")
        mp, stride = tree_mask.data_ptr(), tree_mask.stride(0) if T > 1 else words
    return PagedScores(cap, wide, sp, pp, mp, stride, words)
