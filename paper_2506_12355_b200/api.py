"""Python binding of the C ABI in include/attn_fwd.h.

Argument marshalling only: every step of the attention forward pass runs in the
CUDA kernels of libattn_fwd.so.  PyTorch supplies device memory and streams.
There is no fallback: if the library is missing the import of a symbol fails.
"""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

DTYPE_FP16 = 0
DTYPE_BF16 = 1

STATUS_NAMES = {
    0: "ATTN_OK", 1: "ATTN_ERR_NULL_POINTER", 2: "ATTN_ERR_BAD_SHAPE",
    3: "ATTN_ERR_UNSUPPORTED_HEAD_DIM", 4: "ATTN_ERR_UNSUPPORTED_DTYPE", 5: "ATTN_ERR_MISALIGNED",
    6: "ATTN_ERR_BAD_SCALE", 7: "ATTN_ERR_UNSUPPORTED_ARCH", 8: "ATTN_ERR_CUDA",
    9: "ATTN_ERR_DEVICE_TIMEOUT", 10: "ATTN_ERR_WORKSPACE", 11: "ATTN_ERR_STATIC_CAPACITY",
    12: "ATTN_ERR_COUNTER_SLOTS", 13: "ATTN_ERR_DEVICE_INDEX",
}

# every symbol include/attn_fwd.h declares
EXPORTS = ["attn_bwd", "attn_bwd_workspace_bytes", "attn_fwd", "attn_fwd_gqa", "attn_fwd_partial", "attn_combine", "attn_combine_gather", "attn_fwd_qkv_dims", "attn_fwd_splitkv", "attn_fwd_splitkv_workspace_bytes", "attn_fwd_fp8", "attn_fwd_simt", "attn_fwd_host", "attn_fwd_host_workspace_bytes",
           "attn_fwd_host_static", "attn_fwd_host_static_capacity",
           "attn_fwd_window", "attn_bwd_window", "attn_bwd_window_workspace_bytes",
           "attn_qk_norm_rope", "attn_qk_norm_rope_bwd", "attn_qk_norm_rope_bwd_workspace_bytes", "attn_paged_append", "attn_paged_decode",
           "attn_paged_decode_workspace_bytes",
           "attn_query_support", "attn_last_device_status", "attn_status_string"]

_lib = None


class AttnError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, STATUS_NAMES.get(status, "?"), status))


def lib_path() -> str:
    return _build.LIB_PATH


def load() -> ctypes.CDLL:
    """Loads libattn_fwd.so (built in-tree).  Raises if it does not exist: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError("libattn_fwd.so is not built; run `python -m paper_2506_12355_b200.build` "
                          "or __graft_entry__.build()")
    lib = ctypes.CDLL(path)
    vp, i, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    sig = [vp, vp, vp, vp, vp, i, i, i, i, i, f, i, i, vp]
    lib.attn_fwd.restype = i
    lib.attn_fwd.argtypes = sig
    lib.attn_fwd_gqa.restype = i
    lib.attn_fwd_gqa.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, f, i, i, vp]
    lib.attn_fwd_partial.restype = i
    lib.attn_fwd_partial.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, f, i, i, i, vp]
    lib.attn_combine.restype = i
    lib.attn_combine.argtypes = [vp, vp, i, vp, vp, i, i, i, i, i, vp]
    lib.attn_combine_gather.restype = i
    lib.attn_combine_gather.argtypes = [vp, vp, i, vp, vp, i, i, i, i, i, ctypes.c_longlong, ctypes.c_longlong, vp]
    lib.attn_fwd_qkv_dims.restype = i
    lib.attn_fwd_qkv_dims.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, i, f, i, i, vp]
    lib.attn_fwd_splitkv.restype = i
    lib.attn_fwd_splitkv.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, f, i, i, i, vp, ctypes.c_size_t, vp]
    lib.attn_fwd_splitkv_workspace_bytes.restype = ctypes.c_size_t
    lib.attn_fwd_splitkv_workspace_bytes.argtypes = [i] * 5
    lib.attn_fwd_fp8.restype = i
    lib.attn_fwd_fp8.argtypes = [vp, vp, vp, vp, vp, i, i, i, i, i, i, f, f, f, f, i, i, vp]
    lib.attn_bwd.restype = i
    lib.attn_bwd.argtypes = [vp] * 9 + [i] * 6 + [f, i, i, vp, ctypes.c_size_t, vp]
    lib.attn_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.attn_bwd_workspace_bytes.argtypes = [i] * 3
    lib.attn_fwd_simt.restype = i
    lib.attn_fwd_simt.argtypes = sig
    lib.attn_fwd_host.restype = i
    lib.attn_fwd_host.argtypes = sig[:-1] + [vp, ctypes.c_size_t, vp]
    lib.attn_fwd_host_workspace_bytes.restype = ctypes.c_size_t
    lib.attn_fwd_host_workspace_bytes.argtypes = [i] * 5
    lib.attn_fwd_host_static.restype = i
    lib.attn_fwd_host_static.argtypes = sig
    lib.attn_fwd_host_static_capacity.restype = ctypes.c_size_t
    lib.attn_fwd_host_static_capacity.argtypes = []
    ll, sz = ctypes.c_longlong, ctypes.c_size_t
    lib.attn_fwd_window.restype = i
    lib.attn_fwd_window.argtypes = [vp] * 5 + [i] * 6 + [f] + [i] * 4 + [vp]
    lib.attn_bwd_window.restype = i
    lib.attn_bwd_window.argtypes = [vp] * 9 + [i] * 6 + [f] + [i] * 4 + [vp, sz, vp]
    lib.attn_bwd_window_workspace_bytes.restype = sz
    lib.attn_bwd_window_workspace_bytes.argtypes = [i] * 9
    lib.attn_qk_norm_rope.restype = i
    lib.attn_qk_norm_rope.argtypes = [vp] * 6 + [i, vp, i, i, i, vp, f, vp, vp, vp] + [i] * 6 + [vp]
    lib.attn_qk_norm_rope_bwd.restype = i
    lib.attn_qk_norm_rope_bwd.argtypes = [vp] * 8 + [i, vp, i, i, i, vp, f] + [vp] * 6 + [i] * 6 + [vp, sz, vp]
    lib.attn_qk_norm_rope_bwd_workspace_bytes.restype = sz
    lib.attn_qk_norm_rope_bwd_workspace_bytes.argtypes = [i]
    lib.attn_paged_append.restype = i
    lib.attn_paged_append.argtypes = [vp] * 6 + [i, vp, i, i, i, f] + [vp] * 4 + [i, i, vp, ll, i, vp, vp] + [i] * 6 + [vp]
    lib.attn_paged_decode.restype = i
    lib.attn_paged_decode.argtypes = [vp] * 4 + [i, i, vp, ll, i] + [vp] * 3 + [i] * 4 + [f, i, i, i, vp, sz, vp]
    lib.attn_paged_decode_workspace_bytes.restype = sz
    lib.attn_paged_decode_workspace_bytes.argtypes = [i] * 3
    lib.attn_query_support.restype = i
    lib.attn_query_support.argtypes = [i, i, i]
    lib.attn_last_device_status.restype = i
    lib.attn_last_device_status.argtypes = [vp]
    lib.attn_status_string.restype = ctypes.c_char_p
    lib.attn_status_string.argtypes = [i]
    _lib = lib
    return lib


# Entry points that _binding marshals in C++, in the order in which its bind() takes their addresses.
_BOUND = ["attn_qk_norm_rope", "attn_qk_norm_rope_bwd", "attn_qk_norm_rope_bwd_workspace_bytes", "attn_paged_append", "attn_paged_decode",
          "attn_paged_decode_workspace_bytes", "attn_fwd_window", "attn_bwd_window", "attn_bwd_window_workspace_bytes"]


def _bind():
    """The _binding extension, or None where it is not built (the calls then take their Python path)."""
    try:
        from . import _binding
    except ImportError:
        return None
    lib = load()
    _binding.bind([ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _BOUND])
    return _binding


_UNBOUND = object()
_binding_module = _UNBOUND


def _fast(name, *args):
    """The call through _binding: its result, or NotImplemented where the Python path has to take it (tensors of another device
    than the current one, anything that needs a message)."""
    global _binding_module
    if _binding_module is _UNBOUND:
        _binding_module = _bind()
    if _binding_module is None:
        return NotImplemented
    result = getattr(_binding_module, name)(*args)
    if type(result) is int:
        raise AttnError(result, name)
    return result


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return DTYPE_FP16
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    raise TypeError("q/k/v must be float16 or bfloat16, got %s" % t.dtype)


# torch's current stream of a device as a plain handle, without building a Stream object (3 us of a call's host time)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


# torch's current stream read and set without the Stream objects of torch.cuda.stream (9 us of a call's host time)
_get_stream, _set_stream = (getattr(torch._C, name, None) for name in ("_cuda_getCurrentStream", "_cuda_setStream"))


def _on_stream(stream, tensor, fn, *args, **kwargs):
    """fn(*args, **kwargs) with `stream` as torch's current stream, on `tensor`'s device.  The outputs and workspaces that the call
    allocates then come from `stream`'s pool: out of another stream's they might still be in use by that stream's earlier work, and a
    workspace, dropped when the call returns, would be handed out there again while the kernels on `stream` use it."""
    if not tensor.is_cuda:
        return fn(*args, **kwargs)      # which says what is wrong
    device, handle = tensor.device, int(stream.cuda_stream)
    if handle == 0:
        stream = torch.cuda.default_stream(device)
    elif not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(handle, device=device)
    if stream.device != device:
        raise ValueError("the stream belongs to %s, the tensors to %s" % (stream.device, device))
    if _get_stream is None or _set_stream is None or device.index != torch.cuda.current_device():
        with torch.cuda.stream(stream):
            return fn(*args, **kwargs)
    before = _get_stream(device.index)
    _set_stream(stream_id=stream.stream_id, device_index=stream.device_index, device_type=stream.device_type)
    try:
        return fn(*args, **kwargs)
    finally:
        _set_stream(stream_id=before[0], device_index=before[1], device_type=before[2])


def _call(name, device, *args):
    """The C entry point `name` with `args` and torch's current stream of `device`; raises AttnError for a status other than ATTN_OK."""
    fn = getattr(_lib or load(), name)
    if device.index == torch.cuda.current_device():
        rc = fn(*args, _stream_ptr(None))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _stream_ptr(None))
    if rc != 0:
        raise AttnError(rc, name)


def _check_qkv(q, k, v):
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v must be [B,H,S,D]")
    B, H, Sq, D = q.shape
    Sk = k.shape[2]
    if tuple(k.shape) != (B, H, Sk, D) or tuple(v.shape) != (B, H, Sk, D):
        raise ValueError("k, v must be [B,H,Sk,D] matching q's B, H, D")
    if not (q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
        raise ValueError("q, k, v must be contiguous")
    if not (q.dtype == k.dtype == v.dtype):
        raise TypeError("q, k, v must share one dtype")
    return B, H, Sq, Sk, D


def _check_grouped(q, k, v, same_v_dim=True):
    """The shared checks of the device entry points with grouped K/V heads: q [B,H,Sq,D], k [B,Hkv,Sk,D],
    v [B,Hkv,Sk,Dv] (Dv == D unless same_v_dim is False), contiguous CUDA tensors of one dtype.
    Returns (B, H, Hkv, Sq, Sk, D, Dv)."""
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q must be [B,H,Sq,D]; k, v must be [B,Hkv,Sk,D]")
    B, H, Sq, D = q.shape
    Hkv, Sk, Dv = k.shape[1], k.shape[2], v.shape[3]
    if tuple(k.shape) != (B, Hkv, Sk, D) or tuple(v.shape) != (B, Hkv, Sk, Dv) or (same_v_dim and Dv != D):
        raise ValueError("k must be [B,Hkv,Sk,D] and v [B,Hkv,Sk,%s] matching q's B and D" % ("D" if same_v_dim else "Dv"))
    if not (q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
        raise ValueError("q, k, v must be contiguous")
    if not q.is_cuda or not (q.device == k.device == v.device) or not (q.dtype == k.dtype == v.dtype):
        raise ValueError("q, k, v must be CUDA tensors of one device and dtype")
    return B, H, Hkv, Sq, Sk, D, Dv


def _outputs(q, B, H, Sq, Dv, out, lse, dtype=None):
    """O [B,H,Sq,Dv] and LSE [B,H,Sq] (fp32), allocated on q's device when not given."""
    if out is None:
        out = torch.empty((B, H, Sq, Dv), dtype=q.dtype if dtype is None else dtype, device=q.device)
    if lse is None:
        lse = torch.empty((B, H, Sq), dtype=torch.float32, device=q.device)
    return out, lse


def _workspace(workspace, bytes, device):
    """The caller's workspace, whose size the entry point checks (its address goes to the kernels as it is), or a new one."""
    if workspace is None:
        return torch.empty(max(bytes, 256), dtype=torch.uint8, device=device)
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on %s" % (device,))
    return workspace


def _bytes(workspace):
    return workspace.numel() * workspace.element_size()


def _call_device(fn_name, q, k, v, scale, causal, out, lse, stream):
    if stream is not None and (out is None or lse is None):
        return _on_stream(stream, q, _call_device, fn_name, q, k, v, scale, causal, out, lse, None)
    B, H, Sq, Sk, D = _check_qkv(q, k, v)
    if not q.is_cuda or not (q.device == k.device == v.device):
        raise ValueError("q, k, v must be CUDA tensors of one device")
    dt = _dtype_code(q)
    out, lse = _outputs(q, B, H, Sq, D, out, lse)
    with torch.cuda.device(q.device):
        rc = getattr(load(), fn_name)(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                      lse.data_ptr(), B, H, Sq, Sk, D, float(scale),
                                      int(bool(causal)), dt, _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, fn_name)
    return out, lse


def attn_fwd(q, k, v, scale: float, causal: bool = False, out=None, lse=None, stream=None):
    """O [B,H,Sq,D] (dtype of q) and LSE [B,H,Sq] (fp32) on the tensor-core kernel.

    Enqueues on `stream` (default: torch's current stream) and returns without synchronising.  As under torch.cuda.stream(stream),
    what a call allocates belongs to its stream; inputs and given outputs are the caller's to order against it.
    """
    return _call_device("attn_fwd", q, k, v, scale, causal, out, lse, stream)


def attn_fwd_gqa(q, k, v, scale: float, causal: bool = False, out=None, lse=None, stream=None):
    """Grouped-query / multi-query attention: q [B,H,Sq,D], k, v [B,Hkv,Sk,D] with H % Hkv == 0."""
    if stream is not None and (out is None or lse is None):
        return _on_stream(stream, q, attn_fwd_gqa, q, k, v, scale, causal, out, lse)
    B, H, Hkv, Sq, Sk, D, _ = _check_grouped(q, k, v)
    dt = _dtype_code(q)
    out, lse = _outputs(q, B, H, Sq, D, out, lse)
    with torch.cuda.device(q.device):
        rc = load().attn_fwd_gqa(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                 B, H, Hkv, Sq, Sk, D, float(scale), int(bool(causal)), dt, _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_fwd_gqa")
    return out, lse


def attn_fwd_partial(q, k, v, scale: float, causal: bool, k_offset: int, out=None, lse=None, stream=None):
    """Attention over one K/V shard whose first key has global index k_offset: q [B,H,Sq,D],
    k, v [B,Hkv,Sk_shard,D].  Returns the shard's normalised O_r and LSE_r (merge with attn_combine)."""
    if stream is not None and (out is None or lse is None):
        return _on_stream(stream, q, attn_fwd_partial, q, k, v, scale, causal, k_offset, out, lse)
    B, H, Hkv, Sq, Sk, D, _ = _check_grouped(q, k, v)
    dt = _dtype_code(q)
    out, lse = _outputs(q, B, H, Sq, D, out, lse)
    with torch.cuda.device(q.device):
        rc = load().attn_fwd_partial(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                     B, H, Hkv, Sq, Sk, D, float(scale), int(bool(causal)), int(k_offset), dt,
                                     _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_fwd_partial")
    return out, lse


def attn_combine(o_parts, lse_parts, out=None, lse=None, stream=None):
    """Merges partial results: o_parts [n,B,H,Sq,D] (16-bit), lse_parts [n,B,H,Sq] (fp32)."""
    if stream is not None and (out is None or lse is None):
        return _on_stream(stream, o_parts, attn_combine, o_parts, lse_parts, out, lse)
    n, B, H, Sq, D = o_parts.shape
    if tuple(lse_parts.shape) != (n, B, H, Sq) or lse_parts.dtype != torch.float32:
        raise ValueError("lse_parts must be fp32 [n,B,H,Sq]")
    if not (o_parts.is_contiguous() and lse_parts.is_contiguous() and o_parts.is_cuda and lse_parts.device == o_parts.device):
        raise ValueError("o_parts, lse_parts must be contiguous CUDA tensors of one device")
    dt = _dtype_code(o_parts)
    if out is None:
        out = torch.empty((B, H, Sq, D), dtype=o_parts.dtype, device=o_parts.device)
    if lse is None:
        lse = torch.empty((B, H, Sq), dtype=torch.float32, device=o_parts.device)
    with torch.cuda.device(o_parts.device):
        rc = load().attn_combine(o_parts.data_ptr(), lse_parts.data_ptr(), n, out.data_ptr(), lse.data_ptr(),
                                 B, H, Sq, D, dt, _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_combine")
    return out, lse


def attn_combine_gather(o_part_ptrs, lse_part_ptrs, shape, dtype, out, lse, row_begin=0, row_count=None, stream=None):
    """Merge of partial results that lie behind separate device pointers (possibly peer GPUs' memory), for the
    rows [row_begin, row_begin + row_count) of the flattened (batch, head, query) axis.  o_part_ptrs, lse_part_ptrs:
    lists of integer device addresses; shape: (B, H, Sq, D); dtype: torch.float16 / torch.bfloat16; out, lse: full-size
    CUDA tensors of which only those rows are written."""
    B, H, Sq, D = shape
    n = len(o_part_ptrs)
    if n != len(lse_part_ptrs):
        raise ValueError("as many O pointers as LSE pointers")
    rows = B * H * Sq
    if row_count is None:
        row_count = rows - row_begin
    o_arr = (ctypes.c_void_p * max(n, 1))(*[int(p) for p in o_part_ptrs])
    l_arr = (ctypes.c_void_p * max(n, 1))(*[int(p) for p in lse_part_ptrs])
    dt = DTYPE_FP16 if dtype == torch.float16 else DTYPE_BF16
    with torch.cuda.device(out.device):
        rc = load().attn_combine_gather(o_arr, l_arr, n, out.data_ptr(), lse.data_ptr(), B, H, Sq, D, dt,
                                        int(row_begin), int(row_count), _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_combine_gather")
    return out, lse


def attn_fwd_qkv_dims(q, k, v, scale: float, causal: bool = False, out=None, lse=None, stream=None):
    """Attention with separate Q/K and V head dims (the 192/128 MLA head shape): q [B,H,Sq,Dqk],
    k [B,Hkv,Sk,Dqk], v [B,Hkv,Sk,Dv]; returns o [B,H,Sq,Dv] and lse [B,H,Sq]."""
    if stream is not None and (out is None or lse is None):
        return _on_stream(stream, q, attn_fwd_qkv_dims, q, k, v, scale, causal, out, lse)
    B, H, Hkv, Sq, Sk, Dqk, Dv = _check_grouped(q, k, v, same_v_dim=False)
    dt = _dtype_code(q)
    out, lse = _outputs(q, B, H, Sq, Dv, out, lse)
    with torch.cuda.device(q.device):
        rc = load().attn_fwd_qkv_dims(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                      B, H, Hkv, Sq, Sk, Dqk, Dv, float(scale), int(bool(causal)), dt,
                                      _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_fwd_qkv_dims")
    return out, lse


def attn_fwd_splitkv_workspace_bytes(B, H, Sq, D, n_splits) -> int:
    return int(load().attn_fwd_splitkv_workspace_bytes(B, H, Sq, D, n_splits))


def attn_fwd_splitkv(q, k, v, scale: float, causal: bool, n_splits: int, workspace=None, out=None, lse=None, stream=None):
    """attn_fwd_gqa with the keys split into n_splits ranges that run concurrently, then merged (split-KV
    decoding).  `workspace`: CUDA uint8 tensor of at least attn_fwd_splitkv_workspace_bytes(...) bytes
    (allocated here when None)."""
    if stream is not None and (out is None or lse is None or workspace is None):
        return _on_stream(stream, q, attn_fwd_splitkv, q, k, v, scale, causal, n_splits, workspace, out, lse)
    B, H, Hkv, Sq, Sk, D, _ = _check_grouped(q, k, v)
    dt = _dtype_code(q)
    workspace = _workspace(workspace, attn_fwd_splitkv_workspace_bytes(B, H, Sq, D, n_splits), q.device)
    out, lse = _outputs(q, B, H, Sq, D, out, lse)
    with torch.cuda.device(q.device):
        rc = load().attn_fwd_splitkv(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                     B, H, Hkv, Sq, Sk, D, float(scale), int(bool(causal)), dt, int(n_splits),
                                     workspace.data_ptr(), _bytes(workspace), _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_fwd_splitkv")
    return out, lse


def attn_fwd_fp8(q, k, v, scale: float, q_factor: float = 1.0, k_factor: float = 1.0, v_factor: float = 1.0,
                 causal: bool = False, out=None, lse=None, stream=None, impl: int = 0):
    """Attention on E4M3 inputs with one dequantisation factor per tensor: q [B,H,Sq,128],
    k, v [B,Hkv,Sk,128] as CUDA uint8 (or torch.float8_e4m3fn) tensors; returns o (bf16) and lse (fp32).
    impl 0: tensor-core kernel; impl 1: CUDA-core cross-check kernel."""
    if stream is not None and (out is None or lse is None):
        return _on_stream(stream, q, attn_fwd_fp8, q, k, v, scale, q_factor, k_factor, v_factor, causal, out, lse, impl=impl)
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v must be [B,H,S,D]")
    for t in (q, k, v):
        if t.dtype not in (torch.uint8, torch.float8_e4m3fn) or not t.is_cuda or t.device != q.device or not t.is_contiguous():
            raise ValueError("q, k, v must be contiguous CUDA tensors of E4M3 bytes on one device")
    B, H, Sq, D = q.shape
    Hkv, Sk = k.shape[1], k.shape[2]
    if tuple(k.shape) != (B, Hkv, Sk, D) or tuple(v.shape) != (B, Hkv, Sk, D):
        raise ValueError("k, v must be [B,Hkv,Sk,D] matching q's B and D")
    if out is None:
        out = torch.empty((B, H, Sq, D), dtype=torch.bfloat16, device=q.device)
    if lse is None:
        lse = torch.empty((B, H, Sq), dtype=torch.float32, device=q.device)
    with torch.cuda.device(q.device):
        rc = load().attn_fwd_fp8(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(),
                                 B, H, Hkv, Sq, Sk, D, float(scale), float(q_factor), float(k_factor),
                                 float(v_factor), int(bool(causal)), int(impl), _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_fwd_fp8")
    return out, lse


def attn_bwd_workspace_bytes(B, H, Sq) -> int:
    return int(load().attn_bwd_workspace_bytes(B, H, Sq))


def attn_bwd(q, k, v, o, lse, dout, scale: float, causal: bool = False, dq=None, dk=None, dv=None, workspace=None,
             stream=None):
    """Gradients (dq, dk, dv) of the attention output for the upstream gradient dout: q, o, dout [B,H,Sq,D];
    k, v [B,Hkv,Sk,D]; lse [B,H,Sq] fp32; o and lse from the forward call on the same inputs.  D in {64, 128}.
    `workspace`: CUDA uint8 tensor of at least attn_bwd_workspace_bytes(B, H, Sq) bytes (allocated here when None)."""
    if stream is not None and (dq is None or dk is None or dv is None or workspace is None):
        return _on_stream(stream, q, attn_bwd, q, k, v, o, lse, dout, scale, causal, dq, dk, dv, workspace)
    B, H, Hkv, Sq, Sk, D, _ = _check_grouped(q, k, v)
    if tuple(o.shape) != tuple(q.shape) or tuple(dout.shape) != tuple(q.shape):
        raise ValueError("o and dout must have q's shape")
    if tuple(lse.shape) != (B, H, Sq) or lse.dtype != torch.float32:
        raise ValueError("lse must be fp32 [B,H,Sq]")
    for t in (o, dout, lse):
        if t.device != q.device or not t.is_contiguous():
            raise ValueError("o, dout, lse must be contiguous CUDA tensors on q's device")
    if not (q.dtype == o.dtype == dout.dtype):
        raise TypeError("q, k, v, o, dout must share one dtype")
    dt = _dtype_code(q)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    workspace = _workspace(workspace, attn_bwd_workspace_bytes(B, H, Sq), q.device)
    with torch.cuda.device(q.device):
        rc = load().attn_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
                             dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Hkv, Sq, Sk, D, float(scale),
                             int(bool(causal)), dt, workspace.data_ptr(), _bytes(workspace), _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_bwd")
    return dq, dk, dv


def attn_fwd_window(q, k, v, scale: float, window: int, sinks: int = 0, q_offset: int = 0, out=None, lse=None, stream=None):
    """Attention under a sliding window: q [B,H,Sq,D] at positions q_offset, q_offset + 1, .., k, v [B,Hkv,Sk,D] (D in {64, 128});
    key j is visible at position p iff j <= p and (j > p - window or j < sinks); window 0: no lower end."""
    if stream is not None:
        return _on_stream(stream, q, attn_fwd_window, q, k, v, scale, window, sinks, q_offset, out, lse)
    result = _fast("attn_fwd_window", q, k, v, scale, window, sinks, q_offset, out, lse)
    if result is not NotImplemented:
        return result
    B, H, Hkv, Sq, Sk, D, _ = _check_grouped(q, k, v)
    dt, dtype, device = _dtype_code(q), q.dtype, q.device
    if out is None:
        out = torch.empty(q.shape, dtype=dtype, device=device)
    else:
        _require(out, "out", (B, H, Sq, D), dtype, device)
    if lse is None:
        lse = torch.empty((B, H, Sq), dtype=torch.float32, device=device)
    else:
        _require(lse, "lse", (B, H, Sq), torch.float32, device)
    _call("attn_fwd_window", device, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), B, H, Hkv, Sq, Sk, D,
          float(scale), int(window), int(sinks), int(q_offset), dt)
    return out, lse


def attn_bwd_window_workspace_bytes(B, H, Hkv, Sq, Sk, D, window, sinks=0, q_offset=0) -> int:
    return int(load().attn_bwd_window_workspace_bytes(B, H, Hkv, Sq, Sk, D, window, sinks, q_offset))


def attn_bwd_window(q, k, v, o, lse, dout, scale: float, window: int, sinks: int = 0, q_offset: int = 0, dq=None, dk=None, dv=None,
                    workspace=None, stream=None):
    """Gradients (dq, dk, dv) of attn_fwd_window's output for the upstream gradient dout; o and lse from the forward call.
    `workspace`: CUDA uint8 tensor of at least attn_bwd_window_workspace_bytes(...) bytes (allocated here when None)."""
    if stream is not None:
        return _on_stream(stream, q, attn_bwd_window, q, k, v, o, lse, dout, scale, window, sinks, q_offset, dq, dk, dv, workspace)
    result = _fast("attn_bwd_window", q, k, v, o, lse, dout, scale, window, sinks, q_offset, dq, dk, dv, workspace)
    if result is not NotImplemented:
        return result
    B, H, Hkv, Sq, Sk, D, _ = _check_grouped(q, k, v)
    dt, dtype, device = _dtype_code(q), q.dtype, q.device
    q_shape, k_shape = (B, H, Sq, D), (B, Hkv, Sk, D)
    _require(o, "o", q_shape, dtype, device)
    _require(dout, "dout", q_shape, dtype, device)
    _require(lse, "lse", (B, H, Sq), torch.float32, device)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    _require(dq, "dq", q_shape, dtype, device)
    _require(dk, "dk", k_shape, dtype, device)
    _require(dv, "dv", k_shape, dtype, device)
    workspace = _workspace(workspace, attn_bwd_window_workspace_bytes(B, H, Hkv, Sq, Sk, D, window, sinks, q_offset), device)
    _call("attn_bwd_window", device, q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), dout.data_ptr(),
          dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), B, H, Hkv, Sq, Sk, D, float(scale), int(window), int(sinks), int(q_offset), dt, workspace.data_ptr(),
          _bytes(workspace))
    return dq, dk, dv


def _ptr(t):
    return None if t is None else t.data_ptr()


_stride_arrays = {}


def _strides(*values):
    """A host array of element strides.  A caller's tensors come with the same strides call after call, so the arrays are
    kept (they are only read)."""
    a = _stride_arrays.get(values)
    if a is None:
        if len(_stride_arrays) >= 1024:
            _stride_arrays.clear()
        a = _stride_arrays[values] = (ctypes.c_longlong * len(values))(*values)
    return a


def _rows3(a, b, c=None):
    """Element strides of axes 0, 1, 2 of two or three tensors (zeros for None)."""
    if c is None:
        return _strides(*a.stride()[:3], *b.stride()[:3], 0, 0, 0)
    return _strides(*a.stride()[:3], *b.stride()[:3], *c.stride()[:3])


def _is(t, shape, dtype, index):
    """Cheap form of _require for the checks that every call makes (whose cost is a good part of a small call): contiguous in the
    last axis, this shape, type and GPU."""
    return t.shape == shape and t.dtype is dtype and t.get_device() == index and (t.stride(-1) == 1 or shape[-1] <= 1)


def _require(t, name, shape, dtype, device, dense=True):
    """t has this shape, type and device; its last axis (dense: all of it) is contiguous."""
    if t.shape != shape:
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.device != device:
        raise ValueError("%s must lie on %s, got %s" % (name, device, t.device))
    if dense:
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
    elif shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("the values of a head of %s must be contiguous" % name)


def _check_rope(dtype, device, D, q_weight, k_weight, cos_sin):
    """Weights [D] of one type (`dtype` or fp32) and the table fp32 [positions, R]: (weights are fp32, table length, R)."""
    index = device.index
    any_weight = q_weight if q_weight is not None else k_weight
    f32 = any_weight is not None and any_weight.dtype is torch.float32
    wanted = torch.float32 if f32 else dtype
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None and not _is(w, (D,), wanted, index):
            _require(w, name, (D,), wanted, device)
    if cos_sin is None:
        return f32, 0, 0
    shape = cos_sin.shape
    if len(shape) != 2:
        raise ValueError("cos_sin must be [positions, R]")
    if not (_is(cos_sin, shape, torch.float32, index) and cos_sin.is_contiguous()):
        _require(cos_sin, "cos_sin", shape, torch.float32, device)
    return f32, shape[0], shape[1]


def attn_qk_norm_rope(q, k, v, q_weight, k_weight, cos_sin, positions=None, eps: float = 1e-6, interleaved: bool = False,
                      q_out=None, k_out=None, v_out=None, stream=None):
    """Per-head normalisation and rotation of q [B,S,H,D] and k [B,S,Hkv,D] (strided views of a projection, each head
    contiguous) into the layout that the attention calls read: q_out [B,H,S,D], k_out [B,Hkv,S,D], and v (may be None)
    copied to v_out [B,Hkv,S,D].  q_weight, k_weight: [D] in q's dtype or float32 (None: not normalised); cos_sin: float32
    [positions, R], R/2 cosines then R/2 sines per position (None: not rotated); positions: int32 [B,S] (None: 0 .. S-1);
    interleaved: pairs (2i, 2i+1) instead of (i, i + R/2)."""
    if stream is not None:
        return _on_stream(stream, q, attn_qk_norm_rope, q, k, v, q_weight, k_weight, cos_sin, positions, eps, interleaved, q_out, k_out, v_out)
    result = _fast("attn_qk_norm_rope", q, k, v, q_weight, k_weight, cos_sin, positions, eps, interleaved, q_out, k_out, v_out)
    if result is not NotImplemented:
        return result
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be [B,S,heads,D]")
    B, S, H, D = q.shape
    Hkv = k.shape[2]
    dt, dtype, device = _dtype_code(q), q.dtype, q.device
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor")
    index = device.index
    if not _is(q, q.shape, dtype, index):
        _require(q, "q", (B, S, H, D), dtype, device, False)
    if not _is(k, (B, S, Hkv, D), dtype, index):
        _require(k, "k", (B, S, Hkv, D), dtype, device, False)
    f32, n_pos, R = _check_rope(dtype, device, D, q_weight, k_weight, cos_sin)
    if positions is not None:
        _require(positions, "positions", (B, S), torch.int32, device)
    if q_out is None:
        q_out = torch.empty((B, H, S, D), dtype=dtype, device=device)
    else:
        _require(q_out, "q_out", (B, H, S, D), dtype, device)
    kv_shape = (B, Hkv, S, D)
    if k_out is None:
        k_out = torch.empty(kv_shape, dtype=dtype, device=device)
    else:
        _require(k_out, "k_out", kv_shape, dtype, device)
    if v is None:
        v_out = None
    else:
        if not _is(v, (B, S, Hkv, D), dtype, index):
            _require(v, "v", (B, S, Hkv, D), dtype, device, False)
        if v_out is None:
            v_out = torch.empty(kv_shape, dtype=dtype, device=device)
        else:
            _require(v_out, "v_out", kv_shape, dtype, device)
    _call("attn_qk_norm_rope", device, q.data_ptr(), k.data_ptr(), _ptr(v), _rows3(q, k, v), _ptr(q_weight), _ptr(k_weight), f32,
          _ptr(cos_sin), n_pos, R, bool(interleaved), _ptr(positions), float(eps), q_out.data_ptr(), k_out.data_ptr(), _ptr(v_out), B, S, H,
          Hkv, D, dt)
    return q_out, k_out, v_out


def attn_qk_norm_rope_bwd_workspace_bytes(D) -> int:
    return int(load().attn_qk_norm_rope_bwd_workspace_bytes(D))


def attn_qk_norm_rope_bwd(dq, dk, dv, q, k, q_weight, k_weight, cos_sin, positions=None, eps: float = 1e-6,
                          interleaved: bool = False, dq_in=None, dk_in=None, dv_in=None, workspace=None, stream=None):
    """Gradients of attn_qk_norm_rope: dq [B,H,S,D], dk, dv [B,Hkv,S,D] (contiguous; dv may be None) are the gradients of its
    outputs, q [B,S,H,D], k [B,S,Hkv,D] its inputs.  Returns (dq_in [B,S,H,D], dk_in, dv_in [B,S,Hkv,D], dq_weight, dk_weight
    (float32 [D], None without a weight)).  dq_in, dk_in, dv_in may be given as strided views of one buffer.
    `workspace`: CUDA uint8 tensor of at least attn_qk_norm_rope_bwd_workspace_bytes(D) bytes (allocated here when None)."""
    if stream is not None:
        return _on_stream(stream, q, attn_qk_norm_rope_bwd, dq, dk, dv, q, k, q_weight, k_weight, cos_sin, positions, eps, interleaved, dq_in, dk_in, dv_in,
                          workspace)
    result = _fast("attn_qk_norm_rope_bwd", dq, dk, dv, q, k, q_weight, k_weight, cos_sin, positions, eps, interleaved, dq_in, dk_in, dv_in,
                   workspace)
    if result is not NotImplemented:
        return result
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q and k must be [B,S,heads,D]")
    B, S, H, D = q.shape
    Hkv = k.shape[2]
    dt, dtype, device = _dtype_code(q), q.dtype, q.device
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor")
    q_shape, k_shape = (B, S, H, D), (B, S, Hkv, D)
    _require(q, "q", q_shape, dtype, device, False)
    _require(k, "k", k_shape, dtype, device, False)
    _require(dq, "dq", (B, H, S, D), dtype, device)
    _require(dk, "dk", (B, Hkv, S, D), dtype, device)
    f32, n_pos, R = _check_rope(dtype, device, D, q_weight, k_weight, cos_sin)
    if positions is not None:
        _require(positions, "positions", (B, S), torch.int32, device)
    if dq_in is None:
        dq_in = torch.empty(q_shape, dtype=dtype, device=device)
    else:
        _require(dq_in, "dq_in", q_shape, dtype, device, False)
    if dk_in is None:
        dk_in = torch.empty(k_shape, dtype=dtype, device=device)
    else:
        _require(dk_in, "dk_in", k_shape, dtype, device, False)
    if dv is None:
        dv_in = None
    else:
        _require(dv, "dv", (B, Hkv, S, D), dtype, device)
        if dv_in is None:
            dv_in = torch.empty(k_shape, dtype=dtype, device=device)
        else:
            _require(dv_in, "dv_in", k_shape, dtype, device, False)
    dqw = None if q_weight is None else torch.empty(D, dtype=torch.float32, device=device)
    dkw = None if k_weight is None else torch.empty(D, dtype=torch.float32, device=device)
    workspace = _workspace(workspace, attn_qk_norm_rope_bwd_workspace_bytes(D), device)
    _call("attn_qk_norm_rope_bwd", device, dq.data_ptr(), dk.data_ptr(), _ptr(dv), q.data_ptr(), k.data_ptr(), _rows3(q, k),
          _ptr(q_weight), _ptr(k_weight), f32, _ptr(cos_sin), n_pos, R, bool(interleaved), _ptr(positions), float(eps), dq_in.data_ptr(),
          dk_in.data_ptr(), _ptr(dv_in), _rows3(dq_in, dk_in, dv_in), _ptr(dqw), _ptr(dkw), B, S, H, Hkv, D, dt, workspace.data_ptr(),
          _bytes(workspace))
    return dq_in, dk_in, dv_in, dqw, dkw


def _check_cache(D, dtype, device, k_cache, v_cache, block_table, seq_lens):
    """Caches [pages, Hkv, page_size, D] (any strides, rows contiguous), block_table int32 [sequences, max_pages], seq_lens
    int32 [sequences].  Returns (pages, Hkv, page_size, the caches' strides, sequences, max_pages)."""
    shape, index = k_cache.shape, device.index
    if len(shape) != 4 or shape[3] != D:
        raise ValueError("k_cache and v_cache must be [pages, Hkv, page_size, %d], got %s" % (D, list(shape)))
    if not (_is(k_cache, shape, dtype, index) and _is(v_cache, shape, dtype, index)):
        _require(k_cache, "k_cache", shape, dtype, device, False)
        _require(v_cache, "v_cache", shape, dtype, device, False)
    if seq_lens.dim() != 1 or block_table.dim() != 2:
        raise ValueError("block_table must be [sequences, max_pages] and seq_lens [sequences]")
    n, width = block_table.shape
    if not (_is(seq_lens, (n,), torch.int32, index) and _is(block_table, (n, width), torch.int32, index)):
        _require(seq_lens, "seq_lens", (n,), torch.int32, device)
        _require(block_table, "block_table", (n, width), torch.int32, device, False)
    return shape[0], shape[1], shape[2], _strides(*k_cache.stride()[:3], *v_cache.stride()[:3]), n, width


def attn_paged_append(q, k, v, k_cache, v_cache, block_table, seq_lens, q_weight=None, k_weight=None, cos_sin=None, cu_seqlens=None,
                      eps: float = 1e-6, interleaved: bool = False, q_out=None, stream=None):
    """Appends new tokens to a paged cache: q [T,H,D] (may be None) and k [T,Hkv,D] normalised and rotated as by
    attn_qk_norm_rope at each token's position in its sequence, k and v [T,Hkv,D] written into the pages of k_cache, v_cache
    ([pages, Hkv, page_size, D], any strides).  seq_lens int32 [B]: lengths with the new tokens; block_table int32 [B, max_pages];
    cu_seqlens int32 [B+1]: first new token of each sequence and the end (None: one token per sequence, T == B).  Tokens
    before the first and behind the end, and of sequences of length 0, are padding: nothing is written for them.  Returns
    q_out [T,H,D]."""
    if stream is not None:
        return _on_stream(stream, k, attn_paged_append, q, k, v, k_cache, v_cache, block_table, seq_lens, q_weight, k_weight, cos_sin, cu_seqlens, eps, interleaved,
                          q_out)
    result = _fast("attn_paged_append", q, k, v, k_cache, v_cache, block_table, seq_lens, q_weight, k_weight, cos_sin, cu_seqlens, eps,
                   interleaved, q_out)
    if result is not NotImplemented:
        return result
    if k.dim() != 3 or (q is not None and q.dim() != 3):
        raise ValueError("q must be [tokens,H,D]; k and v [tokens,Hkv,D]")
    T, Hkv, D = kv_shape = k.shape
    dt, dtype, device = _dtype_code(k), k.dtype, k.device
    if not k.is_cuda:
        raise ValueError("k must be a CUDA tensor")
    index = device.index
    if not (_is(k, kv_shape, dtype, index) and _is(v, kv_shape, dtype, index)):
        _require(k, "k", kv_shape, dtype, device, False)
        _require(v, "v", kv_shape, dtype, device, False)
    H, qs = 0, (0, 0)
    if q is not None:
        H = q.shape[1]
        q_shape = (T, H, D)
        if not _is(q, q_shape, dtype, index):
            _require(q, "q", q_shape, dtype, device, False)
        qs = q.stride()
        if q_out is None:
            q_out = torch.empty(q_shape, dtype=dtype, device=device)
        elif not (_is(q_out, q_shape, dtype, index) and q_out.is_contiguous()):
            _require(q_out, "q_out", q_shape, dtype, device)
    elif q_out is not None:
        raise ValueError("q_out without q")
    f32, n_pos, R = _check_rope(dtype, device, D, q_weight, k_weight, cos_sin)
    pages, heads, page_size, cache_strides, n_seqs, width = _check_cache(D, dtype, device, k_cache, v_cache, block_table, seq_lens)
    if heads != Hkv:
        raise ValueError("the caches hold %d heads, k has %d" % (heads, Hkv))
    if cu_seqlens is not None:
        if not _is(cu_seqlens, (n_seqs + 1,), torch.int32, index):
            _require(cu_seqlens, "cu_seqlens", (n_seqs + 1,), torch.int32, device)
    elif T != n_seqs:
        raise ValueError("without cu_seqlens there is one token per sequence: %d tokens, %d sequences" % (T, n_seqs))
    ks, vs = k.stride(), v.stride()
    _call("attn_paged_append", device, _ptr(q), k.data_ptr(), v.data_ptr(), _strides(qs[0], qs[1], ks[0], ks[1], vs[0], vs[1]),
          _ptr(q_weight), _ptr(k_weight), f32, _ptr(cos_sin), n_pos, R, bool(interleaved), float(eps), _ptr(q_out), k_cache.data_ptr(),
          v_cache.data_ptr(), cache_strides, pages, page_size, block_table.data_ptr(), block_table.stride(0), width,
          seq_lens.data_ptr(), _ptr(cu_seqlens), n_seqs, T, H, Hkv, D, dt)
    return q_out


def attn_paged_decode_workspace_bytes(H, Hkv, D) -> int:
    return int((_lib or load()).attn_paged_decode_workspace_bytes(H, Hkv, D))


def attn_paged_decode(q, k_cache, v_cache, block_table, seq_lens, scale: float, window: int = 0, sinks: int = 0, out=None,
                      lse=None, workspace=None, stream=None):
    """Attention of one new token per sequence, q [B,H,D], over a paged cache (see attn_paged_append): keys below seq_lens[b],
    and with window > 0 only the last `window` of them and the first `sinks`.  Returns o [B,H,D] and lse [B,H] (float32).
    `workspace`: CUDA uint8 tensor of at least attn_paged_decode_workspace_bytes(H, Hkv, D) bytes (allocated here when None)."""
    if stream is not None:
        return _on_stream(stream, q, attn_paged_decode, q, k_cache, v_cache, block_table, seq_lens, scale, window, sinks, out, lse, workspace)
    result = _fast("attn_paged_decode", q, k_cache, v_cache, block_table, seq_lens, scale, window, sinks, out, lse, workspace)
    if result is not NotImplemented:
        return result
    if q.dim() != 3:
        raise ValueError("q must be [B,H,D]")
    B, H, D = q_shape = q.shape
    dt, dtype, device = _dtype_code(q), q.dtype, q.device
    if not q.is_cuda:
        raise ValueError("q must be a CUDA tensor")
    if not q.is_contiguous():
        raise ValueError("q must be contiguous")
    pages, Hkv, page_size, cache_strides, n_seqs, width = _check_cache(D, dtype, device, k_cache, v_cache, block_table, seq_lens)
    if n_seqs != B:
        raise ValueError("q has %d rows, seq_lens %d" % (B, n_seqs))
    if out is None:
        out = torch.empty(q_shape, dtype=dtype, device=device)
    else:
        _require(out, "out", q_shape, dtype, device)
    if lse is None:
        lse = torch.empty((B, H), dtype=torch.float32, device=device)
    else:
        _require(lse, "lse", (B, H), torch.float32, device)
    workspace = _workspace(workspace, attn_paged_decode_workspace_bytes(H, Hkv, D), device)
    _call("attn_paged_decode", device, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), cache_strides, pages, page_size,
          block_table.data_ptr(), block_table.stride(0), width, seq_lens.data_ptr(), out.data_ptr(), lse.data_ptr(), B, H,
          Hkv, D, float(scale), int(window), int(sinks), dt, workspace.data_ptr(), _bytes(workspace))
    return out, lse


def attn_fwd_simt(q, k, v, scale: float, causal: bool = False, out=None, lse=None, stream=None):
    """Same operator on the slow CUDA-core cross-check kernel."""
    return _call_device("attn_fwd_simt", q, k, v, scale, causal, out, lse, stream)


def attn_fwd_host_workspace_bytes(B, H, Sq, Sk, D) -> int:
    return int(load().attn_fwd_host_workspace_bytes(B, H, Sq, Sk, D))


def attn_fwd_host(q, k, v, scale: float, causal: bool, out, lse, workspace, stream=None):
    """attn_fwd for HOST tensors (pinned for asynchronous copies); `workspace` is a CUDA uint8
    tensor of at least attn_fwd_host_workspace_bytes(...) bytes.  Results are valid after the
    stream has been synchronised."""
    B, H, Sq, Sk, D = _check_qkv(q, k, v)
    dt = _dtype_code(q)
    with torch.cuda.device(workspace.device):
        rc = load().attn_fwd_host(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                  lse.data_ptr(), B, H, Sq, Sk, D, float(scale), int(bool(causal)),
                                  dt, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                  _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_fwd_host")
    return out, lse


def attn_fwd_host_static_capacity() -> int:
    return int(load().attn_fwd_host_static_capacity())


def attn_fwd_host_static(q, k, v, scale: float, causal: bool, out, lse, stream=None, device=None):
    """attn_fwd_host for callers that cannot allocate device memory: Q, K, V, O and LSE are staged in
    the 16 MiB buffer built into the library image, so no workspace is passed and nothing is
    allocated.  Host tensors in, host tensors out; valid after the stream has been synchronised.
    Problems that need more staging than attn_fwd_host_static_capacity() raise
    AttnError(ATTN_ERR_STATIC_CAPACITY).  All calls on a device share the one buffer: keep them on
    one stream (overlapping calls race).  The first call on a device resolves the buffer's address
    and should come before any stream capture."""
    B, H, Sq, Sk, D = _check_qkv(q, k, v)
    dt = _dtype_code(q)
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(dev):
        rc = load().attn_fwd_host_static(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                         lse.data_ptr(), B, H, Sq, Sk, D, float(scale),
                                         int(bool(causal)), dt, _stream_ptr(stream))
    if rc != 0:
        raise AttnError(rc, "attn_fwd_host_static")
    return out, lse


def attn_query_support(D: int, dtype: int, causal: bool) -> int:
    return int(load().attn_query_support(int(D), int(dtype), int(bool(causal))))


def attn_last_device_status(stream=None) -> int:
    return int(load().attn_last_device_status(_stream_ptr(stream)))


def attn_status_string(status: int) -> str:
    return load().attn_status_string(int(status)).decode()
