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
  ctypes structures :class:`PagedCache` and :class:`PagedBatch`).
"""

from __future__ import annotations

import contextlib
import math
from typing import Optional

from . import _lib
from ._lib import (AppendStrides, PagedBatch, PagedCache, PagedStrides, FA_CACHE_BF16, FA_CACHE_E4M3,  # noqa: F401
                   FA_PAGED_AUTO, FA_PAGED_FEW, FA_PAGED_MANY,
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
           "FA_PAGED_MANY", "kv_append", "forward_paged"]


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
              rot_begin: int = 0, interleaved: bool = False, k_scale=None, v_scale=None, stream=None):
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
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return kv_append(k, v, k_cache, v_cache, block_table, kv_lens, q_starts, q, q_out, cos_sin, rot_begin, interleaved,
                             k_scale, v_scale)
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
    st = _lib.load().fa_kv_append(cache, batch, k.data_ptr(), v.data_ptr(), qp, op, hq,
                                  AppendStrides(qt, qh, ot, oh, kt, kh, vt, vh), table, n_pos, int(rot_begin), rot,
                                  1 if interleaved else 0, torch._C._cuda_getCurrentRawStream(device))
    if st != FA_OK:
        _raise("fa_kv_append", st)
    return q_out


def forward_paged(q, k_cache, v_cache, block_table, kv_lens, q_starts, max_q: Optional[int] = None, causal: bool = True,
                  scale: Optional[float] = None, k_scale=None, v_scale=None, return_lse: bool = False, out=None, lse=None,
                  workspace=None, stream=None, path: Optional[str] = None):
    """Attention of the new tokens q [T, Hq, d_qk] over a paged cache (see :func:`kv_append` for the cache and the
    batch, whose new tokens are in the cache already): returns O [T, Hq, d_v] (bf16) and, with ``return_lse``, LSE
    [T, Hq] (float32, natural log). Token i of the n new ones of sequence b sees the keys up to its position
    ``kv_lens[b] - n + i`` (all ``kv_lens[b]`` where not ``causal``). ``max_q``, the most new tokens of one sequence, helps to
    choose the kernels (default: not known), ``path`` ("few", "many") chooses them: for single tokens and short prompts, or for
    longer ones; the results are right for any. Rows of tokens that belong to no
    sequence are left as they were, so a new tensor's hold anything.

    ``scale`` defaults to 1/sqrt(d_qk). ``workspace`` is a CUDA tensor of ``fa_fwd_paged_workspace_bytes`` (default: from
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
    elsewhere = _elsewhere(stream, device)
    if elsewhere is not None:
        with elsewhere:
            return forward_paged(q, k_cache, v_cache, block_table, kv_lens, q_starts, max_q, causal, scale, k_scale, v_scale,
                                 return_lse, out, lse, workspace, path=path)
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
        nbytes = lib.fa_fwd_paged_workspace_bytes(B, T, max_keys, hq, hkv, dqk, dv, type, max_q, way)
        if nbytes > 0:
            workspace = q.new_empty(nbytes, dtype=torch.uint8)
            ws = workspace.data_ptr()
    elif not isinstance(workspace, torch.Tensor) or workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{device}")
    else:
        nbytes, ws = workspace.numel() * workspace.element_size(), workspace.data_ptr()
    st = lib.fa_fwd_paged(cache, batch, q.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr(), hq,
                          PagedStrides(qt, qh, ot, oh), max_q, way, scale, 1 if causal else 0, ws, nbytes,
                          torch._C._cuda_getCurrentRawStream(device))
    if st != FA_OK:
        _raise("fa_fwd_paged", st)
    return (out, lse) if return_lse else out
