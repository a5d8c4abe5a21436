"""BF1 causal dyadic block-sparse attention (prefill forward and backward) for MI355X.

Thin binding over libbf1.so (declared in include/bf1.h), through ctypes and, for
the usual calls of the cache's operators, through _marshal.so.  Every
function here only checks tensor metadata and marshals pointers, sizes and
the current HIP stream; every step of the computation runs in the library's
HIP kernels.  There is no fallback: if the library is not built, or a call
fails, an exception is raised.

Layouts: Q, O [batch, Hq, n, d] bf16; K, V [batch, Hkv, n, d] bf16;
LSE [batch, Hq, n] float32 (natural log).  q-head h reads kv-head
h // (Hq // Hkv).  Block width ``B`` (tokens per block) and local width
``L`` (blocks) define the route of the paper's §3.1, Eq. 1.
"""

import ctypes
import math
import os
from typing import NamedTuple

__all__ = [
    "BF1Error", "lib_path", "load", "version", "status_string", "plan_size", "plan",
    "attn_fwd", "attn_fwd_csr", "dense_causal_fwd", "release_plans", "selected_flops",
    "plan_transposed", "bwd_workspace_size", "attn_bwd", "selected_bwd_flops", "attn_fwd_noalloc",
    "set_forward_key_split",
    "PageStep", "page_step", "rope_freqs", "rope", "rope_bwd", "kv_append", "CacheQ8", "cache_q8", "kv_append_q8",
    "decode_q8_workspace_size", "attn_decode_q8",
    "qk_norm_rope", "qk_norm_rope_bwd_workspace_size", "qk_norm_rope_bwd", "tree_step", "attn_tree_workspace_size",
    "attn_tree", "kv_compact", "PageFork", "page_fork", "kv_copy",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

BF1_OK = 0
BF1_ERR_INVALID_ARG = -1
BF1_ERR_UNSUPPORTED = -2
BF1_ERR_BUFFER_TOO_SMALL = -3
BF1_ERR_HIP = -4
BF1_ERR_NOMEM = -5
BF1_ERR_CAPTURE = -6


class BF1Error(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


def lib_path():
    return os.path.join(_HERE, "libbf1.so")


def load():
    """Load libbf1.so (built in-tree by __graft_entry__.build()).  Raises if
    it is missing: there is no other implementation to fall back to."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run `python -m paper_2608_20427_amd.build`")
    lib = ctypes.CDLL(path)
    i32, i64, vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p
    lib.bf1_version.restype = ctypes.c_int
    lib.bf1_version.argtypes = []
    lib.bf1_status_string.restype = ctypes.c_char_p
    lib.bf1_status_string.argtypes = [ctypes.c_int]
    lib.bf1_plan_size.restype = ctypes.c_int
    lib.bf1_plan_size.argtypes = [i64, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i64),
                                  ctypes.POINTER(i64)]
    lib.bf1_plan.restype = ctypes.c_int
    lib.bf1_plan.argtypes = [i64, i32, i32, vp, vp, i64, vp]
    attn = [vp, vp, vp, vp, vp, i32, i64, i32, i32, i32]
    lib.bf1_attn_fwd.restype = ctypes.c_int
    lib.bf1_attn_fwd.argtypes = attn + [i32, i32, vp]
    lib.bf1_attn_fwd_noalloc.restype = ctypes.c_int
    lib.bf1_attn_fwd_noalloc.argtypes = attn + [i32, i32, vp]
    lib.bf1_attn_fwd_csr.restype = ctypes.c_int
    lib.bf1_attn_fwd_csr.argtypes = attn + [i32, vp, vp, i64, vp]
    lib.bf1_dense_causal_fwd.restype = ctypes.c_int
    lib.bf1_dense_causal_fwd.argtypes = attn + [vp]
    f32 = ctypes.c_float
    lib.bf1_attn_fwd_token_major.restype = ctypes.c_int
    lib.bf1_attn_fwd_token_major.argtypes = [vp, vp, vp, vp, i32, i64, i32, i32, i32, i32, i32, i32, vp]
    lib.bf1_stack_rms.restype = ctypes.c_int
    lib.bf1_stack_rms.argtypes = [vp, vp, vp, vp, i64, i32, f32, vp]
    lib.bf1_stack_heads.restype = ctypes.c_int
    lib.bf1_stack_heads.argtypes = [vp, vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, i64, i32, i32, i32, f32,
                                    vp]
    lib.bf1_stack_swiglu.restype = ctypes.c_int
    lib.bf1_stack_swiglu.argtypes = [vp, vp, i64, i64, vp, i64, i32, vp]
    lib.bf1_set_forward_key_split.restype = ctypes.c_int
    lib.bf1_set_forward_key_split.argtypes = [i32]
    lib.bf1_release_plans.restype = None
    lib.bf1_release_plans.argtypes = []
    lib.bf1_plan_transposed.restype = ctypes.c_int
    lib.bf1_plan_transposed.argtypes = [i64, i32, i32, vp, vp, i64]
    lib.bf1_attn_bwd_workspace_size.restype = ctypes.c_int
    lib.bf1_attn_bwd_workspace_size.argtypes = [i32, i64, i32, i32, i32, i32, i32,
                                                ctypes.POINTER(i64)]
    lib.bf1_attn_bwd.restype = ctypes.c_int
    lib.bf1_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i64, i32, i32, i32,
                                 i32, i32, vp, i64, vp]
    lib.bf1_plan_variant.restype = ctypes.c_int
    lib.bf1_plan_variant.argtypes = [i32, i64, i32, i32, ctypes.c_uint64, vp, vp, i64]
    lib.bf1_route_depth.restype = ctypes.c_int
    lib.bf1_route_depth.argtypes = [vp, vp, i32, ctypes.POINTER(i32)]
    lib.bf1_decode_plan_stride.restype = ctypes.c_int
    lib.bf1_decode_plan_stride.argtypes = [i64, i32, i32, i32, ctypes.POINTER(i32)]
    lib.bf1_decode_plan.restype = ctypes.c_int
    lib.bf1_decode_plan.argtypes = [i32, vp, vp, i32, i32, i32, i32, i32, vp, i32, vp]
    lib.bf1_decode_workspace_size.restype = ctypes.c_int
    lib.bf1_decode_workspace_size.argtypes = [i32, i32, i32, i32, i32, ctypes.POINTER(i64)]
    lib.bf1_decode_attn.restype = ctypes.c_int
    lib.bf1_decode_attn.argtypes = [vp, vp, vp, vp, i32, vp, i32, vp, vp, i32, i32, i32, i32, i32, vp,
                                    i64, vp]
    lib.bf1_page_step.restype = ctypes.c_int
    lib.bf1_page_step.argtypes = [i32, vp, vp, vp, i32, vp, i32, vp, i32, i64, vp, vp, vp, vp, vp, vp, vp]
    lib.bf1_rope.restype = ctypes.c_int
    lib.bf1_rope.argtypes = [vp, vp, vp, i64, vp, vp, vp, i32, i64, i32, i32, i32, i32, i32, i32, i32, f32, i32,
                             ctypes.POINTER(i64), vp]
    lib.bf1_kv_append.restype = ctypes.c_int
    lib.bf1_kv_append.argtypes = [vp, vp, i64, i64, i64, i64, vp, vp, vp, i64, i32, i32, i32, i32, vp]
    lib.bf1_kv_append_q8.restype = ctypes.c_int
    lib.bf1_kv_append_q8.argtypes = [vp, vp, i64, i64, i64, i64, i64, i32, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp,
                                     vp, vp, vp, i32, i32, i32, i32, vp]
    lib.bf1_decode_q8_workspace_size.restype = ctypes.c_int
    lib.bf1_decode_q8_workspace_size.argtypes = [i32, i32, i32, i32, i32, i32, ctypes.POINTER(i64)]
    lib.bf1_decode_attn_q8.restype = ctypes.c_int
    lib.bf1_decode_attn_q8.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, i32, vp, vp, i32, i32, i32, i32, i32,
                                       i32, vp, i64, vp]
    pi64 = ctypes.POINTER(i64)
    lib.bf1_qk_norm_rope.restype = ctypes.c_int
    lib.bf1_qk_norm_rope.argtypes = [vp, vp, vp, vp, i32, vp, i64, vp, vp, vp, i32, i64, i32, i32, i32, i32, i32, i32, i32,
                                     f32, f32, pi64, vp]
    lib.bf1_qk_norm_rope_bwd_workspace_size.restype = ctypes.c_int
    lib.bf1_qk_norm_rope_bwd_workspace_size.argtypes = [i32, i64, i32, i32, i32, i32, i32, pi64]
    lib.bf1_qk_norm_rope_bwd.restype = ctypes.c_int
    lib.bf1_qk_norm_rope_bwd.argtypes = [vp, vp, i32, vp, vp, vp, vp, i32, vp, i64, vp, vp, vp, vp, vp, i32, i64, i32, i32,
                                         i32, i32, i32, i32, i32, f32, f32, pi64, vp, i64, vp]
    lib.bf1_tree_step.restype = ctypes.c_int
    lib.bf1_tree_step.argtypes = [vp, vp, vp, vp, i32, i64, vp, vp, vp]
    lib.bf1_attn_tree_workspace_size.restype = ctypes.c_int
    lib.bf1_attn_tree_workspace_size.argtypes = [i32, i32, i32, i32, i32, i32, i32, i32, i32, pi64]
    lib.bf1_attn_tree.restype = ctypes.c_int
    lib.bf1_attn_tree.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, i32, i64, i32, i32, i32, i32, i32, i32,
                                  i32, vp, i64, vp]
    lib.bf1_kv_compact.restype = ctypes.c_int
    lib.bf1_kv_compact.argtypes = [vp, vp, vp, i32, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, vp]
    lib.bf1_page_fork.restype = ctypes.c_int
    lib.bf1_page_fork.argtypes = [i32, vp, vp, vp, vp, i32, vp, i32, vp, i32, vp, i32, vp, vp, vp, vp, vp, vp, vp]
    lib.bf1_kv_copy.restype = ctypes.c_int
    lib.bf1_kv_copy.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp]
    _LIB = lib
    return lib


def _check(status, where):
    if status != BF1_OK:
        raise BF1Error(status, where)


def version():
    return load().bf1_version()


def status_string(status):
    return load().bf1_status_string(int(status)).decode()


def plan_size(n, B=64, L=2):
    """(num_blocks, nnz, selected pairs per (batch, head)) in closed form."""
    nb, nnz, pairs = ctypes.c_int32(), ctypes.c_int64(), ctypes.c_int64()
    _check(load().bf1_plan_size(int(n), int(B), int(L), ctypes.byref(nb), ctypes.byref(nnz),
                                ctypes.byref(pairs)), "bf1_plan_size")
    return nb.value, nnz.value, pairs.value


def selected_flops(batch, n, Hq, d, B=64, L=2):
    """Algorithmic flops of the forward: 4 d per selected pair (QK^T and PV),
    per q-head and batch element."""
    return 4 * d * plan_size(n, B, L)[2] * Hq * batch


# Host time of a call matters: short prefills and decode steps take 8-12 us on
# the device.  A call reads the current stream and device through torch's own
# raw accessors (0.2 us against 4 for a Stream object and a device context),
# enters a device context only for a tensor of another device, hands pointers
# over as integers, and checks a buffer with one test, naming what is wrong only
# when that fails; the library itself refuses a small workspace.  Host time per
# call, before and after, us: attn_fwd 15.7 / 11.2, attn_decode 18.7 / 13.2,
# attn_bwd 38.9 / 28.7 (3.8 of it per kernel launch, 1.2 per allocation).

def _stream(stream, dev=None):
    """Raw handle of `stream` (None: the current stream of device `dev`)."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice() if dev is None else dev.index)


def _call(fn, where, dev, stream, *args):
    """fn(*args, stream) with `dev` current; raises BF1Error unless it is BF1_OK."""
    import torch
    if torch._C._cuda_getDevice() == dev.index:
        status = fn(*args, _stream(stream, dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, _stream(stream, dev))
    if status != BF1_OK:
        raise BF1Error(status, where)


def check_buffer(t, name, shape, dtype, device):
    """Raise ValueError unless `t` is a contiguous tensor of exactly `shape`
    and `dtype` on `device`.  Every buffer handed to the library goes through
    this check before its pointer is taken: a host tensor, or one of another
    size, would otherwise become a kernel access outside the intended memory."""
    try:
        if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
            return t
    except AttributeError:
        pass  # no tensor: named below
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor, got {type(t).__name__}")
    if t.device != device:
        raise ValueError(f"{name} must be on device {device}, got {t.device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t


def check_workspace(t, name, nbytes, device):
    """Raise ValueError unless `t` is a contiguous tensor on `device` holding at
    least `nbytes` bytes; returns its size in bytes."""
    import torch
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a tensor, got {type(t).__name__}")
    if t.device != device:
        raise ValueError(f"{name} must be on device {device}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    have = t.numel() * t.element_size()
    if have < nbytes:
        raise ValueError(f"{name} holds {have} bytes, {nbytes} needed")
    return have


def _cuda_device(t, name):
    """The CUDA device of input `t` (ValueError if it is not a CUDA tensor)."""
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t.device


def _ptr(t):
    return None if t is None else t.data_ptr()


def plan(n, B=64, L=2, row_ptr=None, col_idx=None, stream=None):
    """Route table of Eq. 1 as device CSR (int32 row_ptr[NB+1], col_idx[nnz])."""
    import torch
    nb, nnz, _ = plan_size(n, B, L)
    dev = torch.device("cuda", torch.cuda.current_device())
    if row_ptr is None:
        row_ptr = torch.empty(nb + 1, dtype=torch.int32, device=dev)
    if col_idx is None:
        col_idx = torch.empty(max(nnz, 1), dtype=torch.int32, device=dev)
    check_buffer(row_ptr, "row_ptr", (nb + 1,), torch.int32, dev)
    if col_idx.dim() != 1:
        raise ValueError("col_idx must be 1-D")
    check_buffer(col_idx, "col_idx", col_idx.shape, torch.int32, dev)
    _call(load().bf1_plan, "bf1_plan", dev, stream, int(n), int(B), int(L), _ptr(row_ptr), _ptr(col_idx),
          col_idx.numel())
    return row_ptr, col_idx[:nnz]


def _prep(q, k, v, out, lse, want_lse):
    """Check the attention operands and the caller's output buffers (or
    allocate them) on q's device; returns (out, lse, sizes)."""
    import torch
    dev = _cuda_device(q, "q")
    if q.dim() != 4:
        raise ValueError("q must be 4-D [batch, Hq, n, d]")
    batch, Hq, n, d = q.shape
    check_buffer(q, "q", q.shape, torch.bfloat16, dev)
    if not isinstance(k, torch.Tensor) or k.dim() != 4:
        raise ValueError("k must be a 4-D tensor [batch, Hkv, n, d]")
    Hkv = k.shape[1]
    check_buffer(k, "k", (batch, Hkv, n, d), torch.bfloat16, dev)
    check_buffer(v, "v", (batch, Hkv, n, d), torch.bfloat16, dev)
    if out is None:
        out = torch.empty_like(q)
    check_buffer(out, "out", q.shape, torch.bfloat16, dev)
    if lse is None and want_lse:
        lse = torch.empty((batch, Hq, n), dtype=torch.float32, device=dev)
    if lse is not None:
        check_buffer(lse, "lse", (batch, Hq, n), torch.float32, dev)
    return out, lse, (batch, n, Hq, Hkv, d)


def attn_fwd(q, k, v, B=64, L=2, out=None, lse=None, want_lse=True, stream=None):
    """BF1 prefill forward; returns (O, LSE)."""
    out, lse, (batch, n, Hq, Hkv, d) = _prep(q, k, v, out, lse, want_lse)
    _call(load().bf1_attn_fwd, "bf1_attn_fwd", q.device, stream, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
          batch, n, Hq, Hkv, d, int(B), int(L))
    return out, lse


def attn_fwd_noalloc(q, k, v, out, lse=None, B=64, L=2, stream=None):
    """BF1 prefill forward that allocates no device memory: the caller passes O
    (and optionally LSE); returns (O, LSE)."""
    if out is None:
        raise ValueError("attn_fwd_noalloc writes into a caller-provided out")
    out, lse, (batch, n, Hq, Hkv, d) = _prep(q, k, v, out, lse, False)
    _call(load().bf1_attn_fwd_noalloc, "bf1_attn_fwd_noalloc", q.device, stream, _ptr(q), _ptr(k), _ptr(v), _ptr(out),
          _ptr(lse), batch, n, Hq, Hkv, d, int(B), int(L))
    return out, lse


def attn_fwd_csr(q, k, v, B, row_ptr, col_idx, out=None, lse=None, want_lse=True, stream=None):
    """Forward over a caller-supplied block route (CSR, int32 CUDA tensors)."""
    import torch
    out, lse, (batch, n, Hq, Hkv, d) = _prep(q, k, v, out, lse, want_lse)
    if int(B) < 1:
        raise ValueError("B must be positive")
    nb = -(-n // int(B))
    check_buffer(row_ptr, "row_ptr", (nb + 1,), torch.int32, q.device)
    if not isinstance(col_idx, torch.Tensor) or col_idx.dim() != 1:
        raise ValueError("col_idx must be a 1-D tensor")
    check_buffer(col_idx, "col_idx", col_idx.shape, torch.int32, q.device)
    _call(load().bf1_attn_fwd_csr, "bf1_attn_fwd_csr", q.device, stream, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse),
          batch, n, Hq, Hkv, d, int(B), _ptr(row_ptr), _ptr(col_idx), col_idx.numel())
    return out, lse


def dense_causal_fwd(q, k, v, out=None, lse=None, want_lse=True, stream=None):
    """In-house dense causal attention built from the same kernel."""
    out, lse, (batch, n, Hq, Hkv, d) = _prep(q, k, v, out, lse, want_lse)
    _call(load().bf1_dense_causal_fwd, "bf1_dense_causal_fwd", q.device, stream, _ptr(q), _ptr(k), _ptr(v), _ptr(out),
          _ptr(lse), batch, n, Hq, Hkv, d)
    return out, lse


def release_plans():
    load().bf1_release_plans()


def set_forward_key_split(mode):
    """Forward key split: 0 automatic (default), 1 never, 2 always."""
    _check(load().bf1_set_forward_key_split(int(mode)), "bf1_set_forward_key_split")


def plan_transposed(n, B=64, L=2):
    """Transposed route (host only): for every key block, the ascending query
    blocks whose route selects it, as numpy int32 (row_ptr[NB+1], col_idx)."""
    import numpy as np
    nb, nnz, _ = plan_size(n, B, L)
    row_ptr = np.zeros(nb + 1, dtype=np.int32)
    col_idx = np.zeros(max(nnz, 1), dtype=np.int32)
    _check(load().bf1_plan_transposed(int(n), int(B), int(L), row_ptr.ctypes.data_as(ctypes.c_void_p),
                                      col_idx.ctypes.data_as(ctypes.c_void_p), col_idx.size),
           "bf1_plan_transposed")
    return row_ptr, col_idx[:nnz]


ROUTE_KINDS = {"bf1": 0, "sliding": 1, "static_random": 2}


def plan_variant(kind, n, B=64, L=2, seed=17):
    """Route table (host numpy int32 row_ptr[NB+1], col_idx) of kind "bf1",
    "sliding" (matched local sliding) or "static_random" (static random
    nonlocal graph drawn from `seed`); every kind has BF1's row sizes."""
    import numpy as np
    if kind not in ROUTE_KINDS:
        raise ValueError(f"unknown route kind {kind!r}; one of {sorted(ROUTE_KINDS)}")
    nb, nnz, _ = plan_size(n, B, L)
    row_ptr = np.zeros(nb + 1, dtype=np.int32)
    col_idx = np.zeros(max(nnz, 1), dtype=np.int32)
    _check(load().bf1_plan_variant(ROUTE_KINDS[kind], int(n), int(B), int(L), int(seed),
                                   row_ptr.ctypes.data_as(ctypes.c_void_p),
                                   col_idx.ctypes.data_as(ctypes.c_void_p), col_idx.size),
           "bf1_plan_variant")
    return row_ptr, col_idx[:nnz]


def route_depth(row_ptr, col_idx):
    """Communication depth (largest shortest path between blocks) of a host
    CSR route table; -1 if some later block is unreachable."""
    import numpy as np
    rp = np.ascontiguousarray(row_ptr, dtype=np.int32)
    ci = np.ascontiguousarray(col_idx, dtype=np.int32)
    if ci.size == 0:
        ci = np.zeros(1, dtype=np.int32)
    out = ctypes.c_int32(0)
    _check(load().bf1_route_depth(rp.ctypes.data_as(ctypes.c_void_p), ci.ctypes.data_as(ctypes.c_void_p),
                                  int(rp.size - 1), ctypes.byref(out)), "bf1_route_depth")
    return out.value


def bwd_workspace_size(batch, n, Hq, Hkv, d=128, B=64, L=2):
    """Bytes of device workspace bf1_attn_bwd needs."""
    out = ctypes.c_int64(0)
    _check(load().bf1_attn_bwd_workspace_size(int(batch), int(n), int(Hq), int(Hkv), int(d),
                                              int(B), int(L), ctypes.byref(out)),
           "bf1_attn_bwd_workspace_size")
    return out.value


def selected_bwd_flops(batch, n, Hq, d, B=64, L=2):
    """Algorithmic flops of the backward on the selected pairs: the five
    products S = Q K^T (recomputed), dP = dO V^T, dV = P^T dO, dQ = dS K and
    dK = dS^T Q, 2 d flops per selected pair each."""
    return 10 * d * plan_size(n, B, L)[2] * Hq * batch


def attn_bwd(q, k, v, o, do, lse, B=64, L=2, dq=None, dk=None, dv=None, workspace=None,
             stream=None):
    """BF1 backward; returns float32 (dQ, dK, dV).  o and lse are the
    forward's outputs; do is the upstream gradient of o (bf16, o's shape)."""
    import torch
    if o is None or lse is None:
        raise ValueError("attn_bwd needs the forward's o and lse")
    _, _, (batch, n, Hq, Hkv, d) = _prep(q, k, v, o, lse, True)
    dev = q.device
    check_buffer(do, "do", q.shape, torch.bfloat16, dev)

    def _grad(t, name, shape):
        if t is None:
            return torch.empty(shape, dtype=torch.float32, device=dev)
        return check_buffer(t, name, shape, torch.float32, dev)
    dq = _grad(dq, "dq", q.shape)
    dk = _grad(dk, "dk", k.shape)
    dv = _grad(dv, "dv", v.shape)
    if workspace is None:
        need = bwd_workspace_size(batch, n, Hq, Hkv, d, B, L)
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    ws_bytes = check_workspace(workspace, "workspace", 0, dev)
    try:
        _call(load().bf1_attn_bwd, "bf1_attn_bwd", dev, stream, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(do),
              _ptr(lse), _ptr(dq), _ptr(dk), _ptr(dv), batch, n, Hq, Hkv, d, int(B), int(L), _ptr(workspace), ws_bytes)
    except BF1Error:  # refused before anything is launched; a small workspace is a ValueError
        check_workspace(workspace, "workspace", bwd_workspace_size(batch, n, Hq, Hkv, d, B, L), dev)
        raise
    return dq, dk, dv


# ---- one-token decode over a paged cache ------------------------------------

def decode_plan_stride(max_seq_len, B=64, L=2, dense=False):
    """int32 entries per sequence of a decode plan for up to max_seq_len tokens."""
    out = ctypes.c_int32(0)
    _check(load().bf1_decode_plan_stride(int(max_seq_len), int(B), int(L), int(bool(dense)),
                                         ctypes.byref(out)), "bf1_decode_plan_stride")
    return out.value


def _i32_cuda(t, name, dim, device=None):
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.int32 \
            or t.dim() != dim or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dim}-D int32 CUDA tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} must be on device {device}, got {t.device}")


def decode_plan(seq_lens, page_table, num_pages, stride, B=64, L=2, dense=False, plan=None,
                stream=None):
    """Decode plan [batch, stride] int32 (device) for the current block of
    every sequence: the pages of its earlier selected blocks."""
    import torch
    _i32_cuda(seq_lens, "seq_lens", 1)
    dev = seq_lens.device
    _i32_cuda(page_table, "page_table", 2, dev)
    batch, max_pages = page_table.shape
    if seq_lens.shape[0] != batch:
        raise ValueError("seq_lens and page_table disagree on the batch size")
    if plan is None:
        plan = torch.empty((batch, stride), dtype=torch.int32, device=dev)
    check_buffer(plan, "plan", (batch, stride), torch.int32, dev)
    _call(load().bf1_decode_plan, "bf1_decode_plan", dev, stream, batch, _ptr(seq_lens), _ptr(page_table), max_pages,
          int(num_pages), int(B), int(L), int(bool(dense)), _ptr(plan), int(stride))
    return plan


def decode_workspace_size(batch, Hq, Hkv, head_dim, stride):
    out = ctypes.c_int64(0)
    _check(load().bf1_decode_workspace_size(int(batch), int(Hq), int(Hkv), int(head_dim), int(stride),
                                            ctypes.byref(out)), "bf1_decode_workspace_size")
    return out.value


def attn_decode(q, k_pages, v_pages, seq_lens, plan, B=64, out=None, lse=None, workspace=None,
                stream=None):
    """Attention of each sequence's newest token over the paged cache, using
    a decode plan; returns (O [batch, Hq, d] bf16, LSE [batch, Hq] fp32)."""
    import torch
    dev = _cuda_device(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be 3-D [batch, Hq, d]")
    batch, Hq, d = q.shape
    check_buffer(q, "q", q.shape, torch.bfloat16, dev)
    if not isinstance(k_pages, torch.Tensor) or k_pages.dim() != 4:
        raise ValueError("k_pages must be a 4-D tensor [num_pages, Hkv, B, d]")
    num_pages, Hkv, pw, dk = k_pages.shape
    if dk != d or pw != B:
        raise ValueError("k_pages / v_pages must be [num_pages, Hkv, B, d] matching q")
    check_buffer(k_pages, "k_pages", k_pages.shape, torch.bfloat16, dev)
    check_buffer(v_pages, "v_pages", k_pages.shape, torch.bfloat16, dev)
    _i32_cuda(seq_lens, "seq_lens", 1, dev)
    _i32_cuda(plan, "plan", 2, dev)
    if seq_lens.shape[0] != batch or plan.shape[0] != batch:
        raise ValueError("batch sizes disagree")
    if out is None:
        out = torch.empty_like(q)
    check_buffer(out, "out", q.shape, torch.bfloat16, dev)
    if lse is None:
        lse = torch.empty((batch, Hq), dtype=torch.float32, device=dev)
    check_buffer(lse, "lse", (batch, Hq), torch.float32, dev)
    stride = plan.shape[1]
    if workspace is None:
        need = decode_workspace_size(batch, Hq, Hkv, d, stride)
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    ws_bytes = check_workspace(workspace, "workspace", 0, dev)
    try:
        _call(load().bf1_decode_attn, "bf1_decode_attn", dev, stream, _ptr(q), _ptr(k_pages), _ptr(v_pages),
              _ptr(seq_lens), num_pages, _ptr(plan), stride, _ptr(out), _ptr(lse), batch, Hq, Hkv, d, int(B),
              _ptr(workspace), ws_bytes)
    except BF1Error:  # refused before anything is launched; a small workspace is a ValueError
        check_workspace(workspace, "workspace", decode_workspace_size(batch, Hq, Hkv, d, stride), dev)
        raise
    return out, lse


# ---- a served sequence's cache ------------------------------------------------
#
# One step of a batch: page_step places the new tokens, rope turns their queries and
# keys, kv_append or kv_append_q8 writes the cache, decode_plan and attn_decode or
# attn_decode_q8 read it.  A step's rows are packed, sequence after sequence; a sequence
# keeps its place in the batch.

# The usual call of each operator (plain tensors on the current device, outputs of its
# own) is marshalled natively, in _marshal.so: the same checks, allocations and library
# call, of which all but the launch (3.8 us) cost 5 to 11 us as Python code and 0.4 to 3
# there.  Anything else, also what has to be refused, goes through the Python code below
# it, which names what is wrong.  Host time per call, Python / native, us: page_step
# 12.1 / 7.0, rope of q and k 13.4 / 5.8, kv_append 8.6 / 4.2, kv_append_q8 12.4 / 4.8,
# attn_decode_q8 14.6 / 7.0.
_MARSHAL = None


def _native():
    global _MARSHAL
    if _MARSHAL is None:
        import torch  # noqa: F401  (the module resolves against its libraries)
        load()
        from . import _marshal
        _MARSHAL = _marshal
    return _MARSHAL


def _done(r, where):
    """The result of a native call; raises where it is a status of the library."""
    if type(r) is int:
        raise BF1Error(r, where)
    return r


def _empty(shape, dtype, device, stream):
    """An output or scratch tensor whose memory belongs to the stream it is used on."""
    import torch
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=device)  # a tuple for a size costs 0.5 us more
    with torch.cuda.stream(stream):
        return torch.empty(*shape, dtype=dtype, device=device)


class PageStep(NamedTuple):
    """What page_step writes: the lengths after the step [batch], the first row
    [batch + 1] and the blocks written before [batch + 1] of every sequence, the
    position [max_tokens] and slot [max_tokens] of every row (-1: no token, or none
    that has a place), and the free list's new head [1]."""
    seq_lens: object
    token_start: object
    block_start: object
    positions: object
    slots: object
    free_head: object


def page_step(seq_lens, new_lens, page_table, free_pages, free_head, max_tokens, B=64, out=None, stream=None):
    """Page table, slot map and positions of a step that appends new_lens[b] tokens
    to sequence b of seq_lens[b] tokens; returns a PageStep (`out`, if given).

    page_table [batch, max_pages] is updated in place: a block that gets its first
    token takes the next page of free_pages, from entry free_head[0] on.  All are
    int32; slots are int64, page * B + position % B, and index the cache of
    kv_append.  max_tokens (host) bounds the step's rows, so that no length has to
    come back from the GPU.  A token without a free page, past the table or past
    max_tokens has no place, nor do those behind it in its sequence: the returned
    seq_lens count what was placed."""
    if out is None and stream is None:
        r = (_MARSHAL or _native()).page_step(seq_lens, new_lens, page_table, free_pages, free_head, max_tokens, B)
        if r is not None:
            return PageStep._make(_done(r, "bf1_page_step"))
    import torch
    dev = _cuda_device(page_table, "page_table")
    if page_table.dim() != 2:
        raise ValueError("page_table must be a 2-D tensor [batch, max_pages]")
    batch, max_pages = page_table.shape
    check_buffer(page_table, "page_table", page_table.shape, torch.int32, dev)
    check_buffer(seq_lens, "seq_lens", (batch,), torch.int32, dev)
    check_buffer(new_lens, "new_lens", (batch,), torch.int32, dev)
    if not isinstance(free_pages, torch.Tensor) or free_pages.dim() != 1:
        raise ValueError("free_pages must be a 1-D tensor")
    check_buffer(free_pages, "free_pages", free_pages.shape, torch.int32, dev)
    check_buffer(free_head, "free_head", (1,), torch.int32, dev)
    max_tokens = int(max_tokens)
    if not 0 <= max_tokens < 2 ** 31:
        raise ValueError("max_tokens must not be negative, and below 2^31")
    if out is None:
        # one allocation, slots (8 bytes) first; 4 us less than one each
        buf = _empty((3 * max_tokens + 3 * batch + 3,), torch.int32, dev, stream)
        slots, *rest = torch.unsafe_split_with_sizes(
            buf, (2 * max_tokens, batch, batch + 1, batch + 1, max_tokens, 1))
        lens, tstart, bstart, positions, head = rest
        out = PageStep(lens, tstart, bstart, positions, slots.view(torch.int64), head)
    else:
        out = PageStep(*out)
        sizes = (batch, batch + 1, batch + 1, max_tokens, max_tokens, 1)
        for name, t, size in zip(PageStep._fields, out, sizes):
            check_buffer(t, name, (size,), torch.int64 if name == "slots" else torch.int32, dev)
    lens, tstart, bstart, positions, slots, head = out
    _call(load().bf1_page_step, "bf1_page_step", dev, stream, batch, seq_lens.data_ptr(), new_lens.data_ptr(),
          page_table.data_ptr(), max_pages, free_pages.data_ptr(), free_pages.shape[0], free_head.data_ptr(), int(B),
          max_tokens, lens.data_ptr(), tstart.data_ptr(), bstart.data_ptr(), positions.data_ptr(), slots.data_ptr(),
          head.data_ptr())
    return out


ROPE_SCALINGS = ("none", "linear", "base", "bands")


def rope_freqs(rot_dim, theta=1e6, scaling="none", factor=1.0, original_len=32768, slow=1.0, fast=32.0, device=None):
    """(freqs, amplitude) for rope: float64 [rot_dim / 2] radians per position on
    `device` (None: the current CUDA device), theta^(-2 i / rot_dim), for contexts
    `factor` times as long as the original ones:
      "linear"  positions are divided by factor;
      "base"    theta grows by factor^(rot_dim / (rot_dim - 2)), so that the slowest
                pair slows down by factor and the fastest stays;
      "bands"   pairs that turn less than `slow` times over original_len tokens slow
                down by factor, those that turn more than `fast` times stay, the others
                are blended; queries and keys grow by amplitude 0.1 ln(factor) + 1
                (YaRN, arXiv 2309.00071, section 3)."""
    import torch
    if rot_dim < 2 or rot_dim % 2:
        raise ValueError("rot_dim must be even and positive")
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"unknown scaling {scaling!r}; one of {ROPE_SCALINGS}")
    if not (theta > 0 and factor >= 1 and original_len > 0 and fast > slow > 0):
        raise ValueError("rope_freqs needs theta > 0, factor >= 1, original_len > 0 and fast > slow > 0")
    if scaling == "base" and rot_dim > 2:
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    f = theta ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    amplitude = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "bands":
        turns = original_len * f / (2 * math.pi)
        keep = ((turns - slow) / (fast - slow)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
        amplitude = 0.1 * math.log(factor) + 1
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    return f.to(dev), amplitude


def _rope_side(x, name, dim, lead, d, dtype, dev, out, out_dtype, stream):
    """Check one of q, k and its output; returns (out, heads, six strides)."""
    import torch
    if not isinstance(x, torch.Tensor) or x.device != dev or x.dtype != dtype or x.dim() != dim:
        raise ValueError(f"{name} must be a {dim}-D {dtype} tensor on {dev}")
    shape, s = x.shape, x.stride()
    rows = (1, shape[0]) if dim == 3 else (shape[0], shape[2])
    if rows != lead or shape[-1] != d:
        raise ValueError(f"{name} must agree with the other operand in every size but the heads")
    if s[-1] != 1:
        raise ValueError(f"{name} must have the elements of a head side by side")
    if out is None:
        out = _empty(shape, out_dtype, dev, stream)
    else:
        check_buffer(out, name + "_out", shape, out_dtype, dev)
    if dim == 3:  # rows [tokens, heads, d]
        h = shape[1]
        return out, h, (0, s[1], s[0], 0, d, h * d)
    _, h, n, _ = shape
    return out, h, (s[0], s[1], s[2], h * n * d, n * d, d)


def _rope(q, k, positions, freqs, interleaved, amplitude, transposed, q_out, k_out, dtype, stream):
    if stream is None and q_out is None and k_out is None and dtype is None:
        r = (_MARSHAL or _native()).rope(q, k, positions, freqs, interleaved, amplitude, transposed)
        if r is not None:
            return _done(r, "bf1_rope")
    import torch
    x = q if q is not None else k
    dev = _cuda_device(x, "q" if q is not None else "k")
    dim = x.dim()
    if dim not in (3, 4) or x.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("q and k must be bf16 or float32, [batch, heads, n, d] or rows [tokens, heads, d]")
    if dtype is None:
        dtype = x.dtype
    if dtype is not x.dtype and dtype is not torch.bfloat16:
        raise ValueError(f"dtype must be {x.dtype} or bfloat16")
    d = x.shape[-1]
    batch, n = lead = (1, x.shape[0]) if dim == 3 else (x.shape[0], x.shape[2])
    Hq = Hkv = 0
    qs = ks = (0,) * 6
    if q is not None:
        q_out, Hq, qs = _rope_side(q, "q", dim, lead, d, x.dtype, dev, q_out, dtype, stream)
    if k is not None:
        k_out, Hkv, ks = _rope_side(k, "k", dim, lead, d, x.dtype, dev, k_out, dtype, stream)
    if not isinstance(positions, torch.Tensor) or (positions.shape != (n,) and (dim == 3 or positions.shape != lead)):
        raise ValueError(f"positions must have shape ({n},)" + (f" or ({batch}, {n})" if dim == 4 else ""))
    check_buffer(positions, "positions", positions.shape, torch.int32, dev)
    if not isinstance(freqs, torch.Tensor) or freqs.dim() != 1 or not 1 <= freqs.shape[0] <= d // 2:
        raise ValueError("freqs must be a 1-D tensor of at most d / 2 entries")
    check_buffer(freqs, "freqs", freqs.shape, torch.float64, dev)
    _call(load().bf1_rope, "bf1_rope", dev, stream, _ptr(q), _ptr(k), _ptr(positions),
          n if positions.dim() == 2 else 0, _ptr(freqs), _ptr(q_out), _ptr(k_out), batch, n, Hq, Hkv, d,
          2 * freqs.shape[0], 0 if x.dtype is torch.bfloat16 else 1, 0 if dtype is torch.bfloat16 else 1,
          int(bool(interleaved)), float(amplitude), transposed, (ctypes.c_int64 * 12)(*qs, *ks))
    return q_out, k_out


def rope(q, k, positions, freqs, interleaved=False, amplitude=1.0, q_out=None, k_out=None, dtype=None, stream=None):
    """Rotary positions of queries and keys in one launch; returns (q_out, k_out),
    contiguous tensors of the inputs' shapes.

    q, k: [batch, heads, n, d] (any strides with the elements of a head side by side, so
    a view of joined projections is split on the way) or a step's rows [tokens, heads,
    d]; bf16 or float32; either may be None.  positions: int32 [n] or [batch, n].
    freqs, amplitude: rope_freqs'; the first 2 * len(freqs) elements of a head are
    turned, in pairs (i, i + len(freqs)) or, interleaved, (2 i, 2 i + 1); the others
    are copied.  q_out and k_out may be the inputs where those are contiguous."""
    if q is None and k is None:
        raise ValueError("rope needs q or k")
    return _rope(q, k, positions, freqs, interleaved, amplitude, 0, q_out, k_out, dtype, stream)


def rope_bwd(dq, dk, positions, freqs, interleaved=False, amplitude=1.0, dq_out=None, dk_out=None, dtype=None,
             stream=None):
    """Gradients of rope's inputs from those of its outputs: the transposed turn.
    Arguments as rope's; dtype=torch.bfloat16 rounds float32 gradients on the way."""
    if dq is None and dk is None:
        raise ValueError("rope_bwd needs dq or dk")
    return _rope(dq, dk, positions, freqs, interleaved, amplitude, 1, dq_out, dk_out, dtype, stream)


def _step_rows(k, v, Hkv, d, dev):
    """Check a step's rows k, v [tokens, Hkv, d] (strided rows and heads)."""
    import torch
    for name, x in (("k", k), ("v", v)):
        if not isinstance(x, torch.Tensor) or x.device != dev or x.dtype is not torch.bfloat16 or x.dim() != 3:
            raise ValueError(f"{name} must be a bf16 tensor [tokens, Hkv, d] on {dev}")
    shape, (kt, kh, ke), (vt, vh, ve) = k.shape, k.stride(), v.stride()
    if shape[1:] != (Hkv, d) or ke != 1:
        raise ValueError(f"k must have shape (tokens, {Hkv}, {d}) with the elements of a head side by side")
    if v.shape != shape or ve != 1:
        raise ValueError(f"v must have shape {tuple(shape)} with the elements of a head side by side")
    return shape[0], (kt, kh, vt, vh)


def kv_append(k, v, slots, k_pages, v_pages, stream=None):
    """Write a step's rows k, v [tokens, Hkv, d] bf16 into the bf16 pages
    [num_pages, Hkv, B, d] of attn_decode at page_step's slots; rows with a negative
    slot, or one past the cache, are left out.  Slots are distinct."""
    if stream is None:
        r = (_MARSHAL or _native()).kv_append(k, v, slots, k_pages, v_pages)
        if r is not None:
            return _check(r, "bf1_kv_append")
    import torch
    dev = _cuda_device(k_pages, "k_pages")
    if k_pages.dim() != 4:
        raise ValueError("k_pages must be a 4-D tensor [num_pages, Hkv, B, d]")
    num_pages, Hkv, B, d = k_pages.shape
    check_buffer(k_pages, "k_pages", k_pages.shape, torch.bfloat16, dev)
    check_buffer(v_pages, "v_pages", k_pages.shape, torch.bfloat16, dev)
    tokens, strides = _step_rows(k, v, Hkv, d, dev)
    check_buffer(slots, "slots", (tokens,), torch.int64, dev)
    _call(load().bf1_kv_append, "bf1_kv_append", dev, stream, _ptr(k), _ptr(v), *strides, _ptr(slots), _ptr(k_pages),
          _ptr(v_pages), tokens, num_pages, Hkv, d, B)


class CacheQ8(NamedTuple):
    """The 8-bit cache: pages of codes (int8, or e4m3 as torch.float8_e4m3fn), K
    [num_pages, Hkv, B, d] and V [num_pages, Hkv, d, B] with keys side by side; float32
    scales [num_pages, Hkv]; and the newest block of every sequence in bf16, tails
    [batch, Hkv, B, d].  cache_q8 makes one."""
    k_pages: object
    v_pages: object
    k_scale: object
    v_scale: object
    k_tail: object
    v_tail: object


def cache_q8(num_pages, batch, Hkv, d=128, B=64, dtype=None, device=None):
    """An empty CacheQ8 for `batch` sequences over `num_pages` pages; dtype:
    torch.float8_e4m3fn (default) or torch.int8."""
    import torch
    dtype = torch.float8_e4m3fn if dtype is None else dtype
    if dtype not in (torch.float8_e4m3fn, torch.int8):
        raise ValueError("dtype must be torch.float8_e4m3fn or torch.int8")
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    pages = [torch.zeros(s, dtype=torch.int8, device=dev).view(dtype)
             for s in ((num_pages, Hkv, B, d), (num_pages, Hkv, d, B))]
    scales = [torch.ones((num_pages, Hkv), dtype=torch.float32, device=dev) for _ in range(2)]
    tails = [torch.zeros((batch, Hkv, B, d), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    return CacheQ8(*pages, *scales, *tails)


def _cache_q8(cache, batch):
    """Check a CacheQ8 for `batch` sequences; returns (device, num_pages, Hkv, B, d,
    format).  What passes is asked in one expression (2 us; six check_buffer calls 2.8);
    what does not is named after it."""
    import torch
    kp, vp, ks, vs, kt, vt = cache
    dev = _cuda_device(kp, "k_pages")
    dtype, f32, bf16 = kp.dtype, torch.float32, torch.bfloat16
    if kp.dim() != 4 or (dtype is not torch.float8_e4m3fn and dtype is not torch.int8):
        raise ValueError("k_pages must be an int8 or float8_e4m3fn tensor [num_pages, Hkv, B, d]")
    num_pages, Hkv, B, d = kp.shape
    scale, tail = (num_pages, Hkv), (batch, Hkv, B, d)
    try:
        good = vp.dtype is dtype and ks.dtype is f32 and vs.dtype is f32 and kt.dtype is bf16 and vt.dtype is bf16 \
            and vp.shape == (num_pages, Hkv, d, B) and ks.shape == scale and vs.shape == scale and kt.shape == tail \
            and vt.shape == tail and vp.device == dev and ks.device == dev and vs.device == dev and kt.device == dev \
            and vt.device == dev and kp.is_contiguous() and vp.is_contiguous() and ks.is_contiguous() \
            and vs.is_contiguous() and kt.is_contiguous() and vt.is_contiguous()
    except AttributeError:
        good = False  # no tensor
    if not good:
        check_buffer(kp, "k_pages", kp.shape, dtype, dev)
        check_buffer(vp, "v_pages", (num_pages, Hkv, d, B), dtype, dev)
        check_buffer(ks, "k_scale", scale, f32, dev)
        check_buffer(vs, "v_scale", scale, f32, dev)
        check_buffer(kt, "k_tail", tail, bf16, dev)
        check_buffer(vt, "v_tail", tail, bf16, dev)
    return dev, num_pages, Hkv, B, d, 1 if dtype is torch.int8 else 0


def kv_append_q8(k, v, lens_before, seq_lens, token_start, block_start, page_table, cache, stream=None):
    """Write a step's rows k, v [tokens, Hkv, d] bf16 into a CacheQ8: blocks that the
    step completes are quantised into their pages, the rows of each sequence's newest
    block go to its tail.  lens_before: the lengths page_step was given; seq_lens,
    token_start and block_start: what it returned; page_table: what it updated.

    A step that begins inside a block and ends in a later one overwrites the tail rows
    that it quantised: to run it again (a warm-up before a capture, a retry), put
    cache.k_tail and cache.v_tail back as they were first.  Other steps can be repeated
    as they are.  Tokens can be taken back only as far as the newest block's first."""
    if stream is None:
        r = (_MARSHAL or _native()).kv_append_q8(k, v, lens_before, seq_lens, token_start, block_start, page_table, cache)
        if r is not None:
            return _check(r, "bf1_kv_append_q8")
    import torch
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be a 2-D tensor [batch, max_pages]")
    batch, max_pages = page_table.shape
    dev, num_pages, Hkv, B, d, fmt = _cache_q8(cache, batch)
    check_buffer(page_table, "page_table", page_table.shape, torch.int32, dev)
    check_buffer(lens_before, "lens_before", (batch,), torch.int32, dev)
    check_buffer(seq_lens, "seq_lens", (batch,), torch.int32, dev)
    check_buffer(token_start, "token_start", (batch + 1,), torch.int32, dev)
    check_buffer(block_start, "block_start", (batch + 1,), torch.int32, dev)
    tokens, strides = _step_rows(k, v, Hkv, d, dev)
    kp, vp, ks, vs, kt, vt = cache
    _call(load().bf1_kv_append_q8, "bf1_kv_append_q8", dev, stream, k.data_ptr(), v.data_ptr(), *strides, tokens, batch,
          lens_before.data_ptr(), seq_lens.data_ptr(), token_start.data_ptr(), block_start.data_ptr(),
          page_table.data_ptr(), max_pages, num_pages, kp.data_ptr(), vp.data_ptr(), ks.data_ptr(), vs.data_ptr(),
          kt.data_ptr(), vt.data_ptr(), Hkv, d, B, fmt)


def decode_q8_workspace_size(batch, Hq, Hkv, head_dim, B, stride):
    out = ctypes.c_int64(0)
    _check(load().bf1_decode_q8_workspace_size(int(batch), int(Hq), int(Hkv), int(head_dim), int(B), int(stride),
                                               ctypes.byref(out)), "bf1_decode_q8_workspace_size")
    return out.value


def attn_decode_q8(q, cache, seq_lens, plan, B=64, out=None, lse=None, workspace=None, stream=None):
    """attn_decode over a CacheQ8, with the same plan: earlier pages in 8 bits, the
    newest block from the tail; returns (O [batch, Hq, d] bf16, LSE [batch, Hq]
    fp32)."""
    if stream is None and out is None and lse is None and workspace is None:
        r = (_MARSHAL or _native()).attn_decode_q8(q, cache, seq_lens, plan, B)
        if r is not None:
            return _done(r, "bf1_decode_attn_q8")
    import torch
    dev = _cuda_device(q, "q")
    if q.dim() != 3:
        raise ValueError("q must be 3-D [batch, Hq, d]")
    batch, Hq, d = shape = q.shape
    check_buffer(q, "q", shape, torch.bfloat16, dev)
    where, num_pages, Hkv, pw, dk, fmt = _cache_q8(cache, batch)
    if where != dev or dk != d or pw != B:
        raise ValueError("the cache must have q's device and head size, and pages of B tokens")
    _i32_cuda(seq_lens, "seq_lens", 1, dev)
    _i32_cuda(plan, "plan", 2, dev)
    rows, stride = plan.shape
    if seq_lens.shape[0] != batch or rows != batch:
        raise ValueError("batch sizes disagree")
    if out is None:
        out = torch.empty_like(q) if stream is None else _empty(shape, torch.bfloat16, dev, stream)
    else:
        check_buffer(out, "out", shape, torch.bfloat16, dev)
    if lse is None:
        lse = _empty((batch, Hq), torch.float32, dev, stream)
    else:
        check_buffer(lse, "lse", (batch, Hq), torch.float32, dev)
    need = decode_q8_workspace_size(batch, Hq, Hkv, d, B, stride)
    ws_bytes = need
    if workspace is not None:
        ws_bytes = check_workspace(workspace, "workspace", need, dev)
    elif need:
        workspace = _empty((need,), torch.uint8, dev, stream)
    kp, vp, ks, vs, kt, vt = cache
    _call(load().bf1_decode_attn_q8, "bf1_decode_attn_q8", dev, stream, q.data_ptr(), kp.data_ptr(), vp.data_ptr(),
          ks.data_ptr(), vs.data_ptr(), kt.data_ptr(), vt.data_ptr(), seq_lens.data_ptr(), num_pages, plan.data_ptr(),
          stride, out.data_ptr(), lse.data_ptr(), batch, Hq, Hkv, d, int(B), fmt, _ptr(workspace), ws_bytes)
    return out, lse


# ---- norms of queries and keys with their rotary positions -----------------------

def _strided(t, name, shape, dtype, dev):
    """Raise ValueError unless `t` is a tensor of `shape` and `dtype` on `dev` with the
    elements of a head side by side; returns its strides over batch, heads and tokens."""
    import torch
    if not isinstance(t, torch.Tensor) or t.device != dev or t.dtype != dtype or t.shape != shape:
        raise ValueError(f"{name} must be a {dtype} tensor of shape {tuple(shape)} on {dev}")
    s = t.stride()
    if s[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name} must have the elements of a head side by side")
    return (0, s[1], s[0]) if len(shape) == 3 else s[:3]


def _norm_rope_sides(q, k, q_gain, k_gain, positions, freqs):
    """Check what forward and gradient have in common; returns (device, type, gains' type,
    sizes)."""
    import torch
    x = q if q is not None else k
    if x is None:
        raise ValueError("qk_norm_rope needs q or k")
    dev = _cuda_device(x, "q" if q is not None else "k")
    dim = x.dim()
    if dim not in (3, 4) or x.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("q and k must be bf16 or float32, [batch, heads, n, d] or rows [tokens, heads, d]")
    d = x.shape[-1]
    batch, n = lead = (1, x.shape[0]) if dim == 3 else (x.shape[0], x.shape[2])
    heads = []
    for name, t in (("q", q), ("k", k)):
        if t is None:
            heads.append(0)
            continue
        if not isinstance(t, torch.Tensor) or t.dim() != dim or t.shape[-1] != d \
                or ((1, t.shape[0]) if dim == 3 else (t.shape[0], t.shape[2])) != lead:
            raise ValueError(f"{name} must agree with the other operand in every size but the heads")
        heads.append(t.shape[1])
    gains = [g for g in (q_gain, k_gain) if g is not None]
    gtype = torch.float32
    if gains:
        gtype = getattr(gains[0], "dtype", None)
        if gtype not in (torch.bfloat16, torch.float32):
            raise ValueError("gains must be bf16 or float32 tensors")
        for name, g in (("q_gain", q_gain), ("k_gain", k_gain)):
            if g is not None:
                check_buffer(g, name, (d,), gtype, dev)
    if not isinstance(positions, torch.Tensor) or (positions.shape != (n,) and (dim == 3 or positions.shape != lead)):
        raise ValueError(f"positions must have shape ({n},)" + (f" or ({batch}, {n})" if dim == 4 else ""))
    check_buffer(positions, "positions", positions.shape, torch.int32, dev)
    if not isinstance(freqs, torch.Tensor) or freqs.dim() != 1 or not 1 <= freqs.shape[0] <= d // 2:
        raise ValueError("freqs must be a 1-D tensor of at most d / 2 entries")
    check_buffer(freqs, "freqs", freqs.shape, torch.float64, dev)
    return dev, x.dtype, gtype, (batch, n, *heads, d)


def _type(dtype):
    import torch
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"dtype must be bfloat16 or float32, got {dtype}")
    return 0 if dtype is torch.bfloat16 else 1


def qk_norm_rope(q, k, q_gain, k_gain, positions, freqs, eps=1e-6, interleaved=False, amplitude=1.0, q_out=None,
                 k_out=None, dtype=None, stream=None):
    """RMSNorm of every head of queries and keys, times q_gain and k_gain [d] (bf16 or
    float32; None: ones), and rope in one launch; returns (q_out, k_out).

    q, k, positions, freqs, interleaved and amplitude as rope's; either of q, k may be
    None.  Outputs are contiguous tensors of the inputs' shapes, or q_out and k_out: any
    strides with the elements of a head side by side, the inputs themselves among them.
    dtype=torch.bfloat16 rounds float32 inputs on the way."""
    if stream is None and q_out is None and k_out is None and dtype is None:
        r = (_MARSHAL or _native()).qk_norm_rope(q, k, q_gain, k_gain, positions, freqs, eps, interleaved, amplitude)
        if r is not None:
            return _done(r, "bf1_qk_norm_rope")
    dev, xtype, gtype, (batch, n, Hq, Hkv, d) = _norm_rope_sides(q, k, q_gain, k_gain, positions, freqs)
    dtype = xtype if dtype is None else dtype
    strides, outs = [], []
    for name, x, out in (("q", q, q_out), ("k", k, k_out)):
        if x is None:
            strides += [0] * 6
            outs.append(None)
            continue
        strides += _strided(x, name, x.shape, xtype, dev)
        out = _empty(x.shape, dtype, dev, stream) if out is None else out
        strides += _strided(out, name + "_out", x.shape, dtype, dev)
        outs.append(out)
    _call(load().bf1_qk_norm_rope, "bf1_qk_norm_rope", dev, stream, _ptr(q), _ptr(k), _ptr(q_gain), _ptr(k_gain),
          _type(gtype), _ptr(positions), n if positions.dim() == 2 else 0, _ptr(freqs), _ptr(outs[0]), _ptr(outs[1]), batch,
          n, Hq, Hkv, d, 2 * freqs.shape[0], _type(xtype), _type(dtype), int(bool(interleaved)), float(eps),
          float(amplitude), (ctypes.c_int64 * 12)(*strides))
    return tuple(outs)


def qk_norm_rope_bwd_workspace_size(batch, n, Hq, Hkv, d, rot_dim, dtype):
    """Bytes of workspace of qk_norm_rope_bwd; dtype: q's and k's."""
    out = ctypes.c_int64(0)
    _check(load().bf1_qk_norm_rope_bwd_workspace_size(int(batch), int(n), int(Hq), int(Hkv), int(d), int(rot_dim),
                                                      _type(dtype), ctypes.byref(out)), "bf1_qk_norm_rope_bwd_workspace_size")
    return out.value


def qk_norm_rope_bwd(dq, dk, q, k, q_gain, k_gain, positions, freqs, eps=1e-6, interleaved=False, amplitude=1.0,
                     dq_out=None, dk_out=None, dtype=None, workspace=None, stream=None):
    """Gradients of qk_norm_rope: of q, k (dtype: theirs by default, or bf16 or float32)
    and, in float32, of q_gain and k_gain (None where that is None), from those of its
    outputs, dq and dk: float32, or q's type.  q and k are the forward's inputs; any
    strides with the elements of a head side by side.  Outputs are contiguous, or dq_out
    and dk_out with any such strides, dq and dk themselves or q and k among them."""
    import torch
    if stream is None and dq_out is None and dk_out is None and dtype is None and workspace is None:
        r = (_MARSHAL or _native()).qk_norm_rope_bwd(dq, dk, q, k, q_gain, k_gain, positions, freqs, eps, interleaved,
                                                     amplitude)
        if r is not None:
            return _done(r, "bf1_qk_norm_rope_bwd")
    dev, xtype, gtype, (batch, n, Hq, Hkv, d) = _norm_rope_sides(q, k, q_gain, k_gain, positions, freqs)
    dtype = xtype if dtype is None else dtype
    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("dtype must be bfloat16 or float32")
    ytype = getattr(dq if q is not None else dk, "dtype", None)
    if ytype is not torch.float32 and ytype is not xtype:
        raise ValueError(f"dq and dk must be float32 or {xtype}")
    strides, outs, gains = [], [], []
    for name, x, dy, out, gain in (("q", q, dq, dq_out, q_gain), ("k", k, dk, dk_out, k_gain)):
        if x is None:
            if dy is not None:
                raise ValueError(f"d{name} without {name}")
            strides += [0] * 9
            outs.append(None)
            gains.append(None)
            continue
        strides += _strided(dy, "d" + name, x.shape, ytype, dev)
        strides += _strided(x, name, x.shape, xtype, dev)
        out = _empty(x.shape, dtype, dev, stream) if out is None else out
        strides += _strided(out, f"d{name}_out", x.shape, dtype, dev)
        outs.append(out)
        gains.append(None if gain is None else _empty((d,), torch.float32, dev, stream))
    rot = 2 * freqs.shape[0]
    need = qk_norm_rope_bwd_workspace_size(batch, n, Hq, Hkv, d, rot, xtype) if any(g is not None for g in gains) else 0
    if workspace is not None:
        check_workspace(workspace, "workspace", need, dev)
    elif need:
        workspace = _empty((need,), torch.uint8, dev, stream)
    _call(load().bf1_qk_norm_rope_bwd, "bf1_qk_norm_rope_bwd", dev, stream, _ptr(dq), _ptr(dk), _type(ytype), _ptr(q),
          _ptr(k), _ptr(q_gain), _ptr(k_gain), _type(gtype), _ptr(positions), n if positions.dim() == 2 else 0, _ptr(freqs),
          _ptr(outs[0]), _ptr(outs[1]), _ptr(gains[0]), _ptr(gains[1]), batch, n, Hq, Hkv, d, rot, _type(xtype),
          _type(dtype), int(bool(interleaved)), float(eps), float(amplitude), (ctypes.c_int64 * 18)(*strides),
          _ptr(workspace), need)
    return (*outs, *gains)


# ---- drafted tokens over the cache, and pages of several sequences -----------------
#
# A step that verifies drafts: page_step and kv_append place the trees' nodes as new
# tokens, tree_step makes their masks and positions (for rope or qk_norm_rope too),
# attn_tree is their attention, kv_compact keeps the accepted ones.  page_fork and
# kv_copy continue sequences from others and free what nobody holds any more.

def tree_step(parents, token_start, lens_before, seq_lens, masks=None, positions=None, stream=None):
    """(masks, positions) of the nodes of drafted trees, packed as page_step's rows.

    parents: int32 [rows], each node's parent in its own tree (an earlier node; anything
    else: none, the node follows the sequence's newest token).  token_start and seq_lens:
    page_step's for this step; lens_before: the lengths it was given.  masks: int64 [rows],
    bit k of a row set where node k is the node or one before it; positions: int32 [rows],
    the length plus the depth.  A tree has up to 64 nodes; those past the 64th or past
    seq_lens, and rows behind the last tree, get mask 0 and position -1."""
    if masks is None and positions is None and stream is None:
        r = (_MARSHAL or _native()).tree_step(parents, token_start, lens_before, seq_lens)
        if r is not None:
            return _done(r, "bf1_tree_step")
    import torch
    dev = _cuda_device(parents, "parents")
    _i32_cuda(parents, "parents", 1)
    _i32_cuda(lens_before, "lens_before", 1, dev)
    rows, batch = parents.shape[0], lens_before.shape[0]
    check_buffer(token_start, "token_start", (batch + 1,), torch.int32, dev)
    check_buffer(seq_lens, "seq_lens", (batch,), torch.int32, dev)
    masks = _empty((rows,), torch.int64, dev, stream) if masks is None \
        else check_buffer(masks, "masks", (rows,), torch.int64, dev)
    positions = _empty((rows,), torch.int32, dev, stream) if positions is None \
        else check_buffer(positions, "positions", (rows,), torch.int32, dev)
    _call(load().bf1_tree_step, "bf1_tree_step", dev, stream, _ptr(parents), _ptr(token_start), _ptr(lens_before),
          _ptr(seq_lens), batch, rows, _ptr(masks), _ptr(positions))
    return masks, positions


def _bf16_pages(k_pages, v_pages):
    """Check bf16 pages [num_pages, Hkv, B, d]; returns (device, sizes)."""
    import torch
    dev = _cuda_device(k_pages, "k_pages")
    if k_pages.dim() != 4:
        raise ValueError("k_pages must be a 4-D tensor [num_pages, Hkv, B, d]")
    check_buffer(k_pages, "k_pages", k_pages.shape, torch.bfloat16, dev)
    check_buffer(v_pages, "v_pages", k_pages.shape, torch.bfloat16, dev)
    return dev, tuple(k_pages.shape)


def attn_tree_workspace_size(batch, max_nodes, Hq, Hkv, head_dim, B, max_pages, L=2, dense=False):
    out = ctypes.c_int64(0)
    _check(load().bf1_attn_tree_workspace_size(int(batch), int(max_nodes), int(Hq), int(Hkv), int(head_dim), int(B),
                                               int(max_pages), int(L), int(bool(dense)), ctypes.byref(out)),
           "bf1_attn_tree_workspace_size")
    return out.value


def attn_tree(q, k_pages, v_pages, masks, positions, lens_before, token_start, page_table, B=64, L=2, dense=False,
              max_nodes=64, out=None, lse=None, workspace=None, stream=None):
    """Attention of all nodes of drafted trees over the paged cache that holds them (at
    page_step's slots); returns (O [rows, Hq, d] bf16, LSE [rows, Hq] fp32).

    q: [rows, Hq, d] bf16, packed; masks, positions: tree_step's, or any masks; lens_before:
    the lengths without the drafted tokens; token_start: page_step's.  A node at position
    p reads the committed keys of the blocks on the BF1 route of block p // B (dense: of
    every block up to it) and the drafted ones of its mask; as in the decodes, weights are
    applied with their 24 bits.  max_nodes: the largest tree of the call, 1 to 64; rows past
    it get NaN, as do those without a place and those of a sequence that lacks a page.  Rows
    behind the last tree are left as they are."""
    if out is None and lse is None and workspace is None and stream is None:
        r = (_MARSHAL or _native()).attn_tree(q, k_pages, v_pages, masks, positions, lens_before, token_start, page_table, B,
                                              L, dense, max_nodes)
        if r is not None:
            return _done(r, "bf1_attn_tree")
    import torch
    dev, (num_pages, Hkv, pw, d) = _bf16_pages(k_pages, v_pages)
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.shape[2] != d or pw != B:
        raise ValueError("q must be [rows, Hq, d] with the cache's head size, and its pages hold B tokens")
    rows, Hq, _ = q.shape
    check_buffer(q, "q", q.shape, torch.bfloat16, dev)
    check_buffer(masks, "masks", (rows,), torch.int64, dev)
    check_buffer(positions, "positions", (rows,), torch.int32, dev)
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be a 2-D tensor [batch, max_pages]")
    batch, max_pages = page_table.shape
    check_buffer(page_table, "page_table", page_table.shape, torch.int32, dev)
    check_buffer(lens_before, "lens_before", (batch,), torch.int32, dev)
    check_buffer(token_start, "token_start", (batch + 1,), torch.int32, dev)
    out = _empty(q.shape, torch.bfloat16, dev, stream) if out is None \
        else check_buffer(out, "out", q.shape, torch.bfloat16, dev)
    lse = _empty((rows, Hq), torch.float32, dev, stream) if lse is None \
        else check_buffer(lse, "lse", (rows, Hq), torch.float32, dev)
    need = attn_tree_workspace_size(batch, max_nodes, Hq, Hkv, d, B, max_pages, L, dense)
    if workspace is not None:
        check_workspace(workspace, "workspace", need, dev)
    elif need:
        workspace = _empty((need,), torch.uint8, dev, stream)
    _call(load().bf1_attn_tree, "bf1_attn_tree", dev, stream, _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(masks),
          _ptr(positions), _ptr(lens_before), _ptr(token_start), _ptr(page_table), max_pages, num_pages, _ptr(out), _ptr(lse),
          batch, rows, int(max_nodes), Hq, Hkv, d, int(B), int(L), int(bool(dense)), _ptr(workspace), need)
    return out, lse


def kv_compact(k_pages, v_pages, accepted, lens_before, seq_lens, page_table, out=None, stream=None):
    """Move the rows of the accepted nodes of every tree together in one layer's bf16
    cache: node accepted[b, k] goes to position lens_before[b] + k.  Returns the new lengths
    int32 [batch] (`out`, if given; another tensor than the two it is made of).

    accepted: int32 [batch, up to 64], a path's nodes, ascending; the first entry that is
    not above the one before it, or is no node (-1), ends it.  seq_lens: with the drafted
    tokens, as page_step returned it.  The pages behind the new lengths stay in the table:
    give seq_lens and, as keep_lens, the result to page_fork before the next page_step, which
    frees them."""
    if out is None and stream is None:
        r = (_MARSHAL or _native()).kv_compact(k_pages, v_pages, accepted, lens_before, seq_lens, page_table)
        if r is not None:
            return _done(r, "bf1_kv_compact")
    import torch
    dev, (num_pages, Hkv, B, d) = _bf16_pages(k_pages, v_pages)
    if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be a 2-D tensor [batch, max_pages]")
    batch, max_pages = page_table.shape
    check_buffer(page_table, "page_table", page_table.shape, torch.int32, dev)
    if not isinstance(accepted, torch.Tensor) or accepted.dim() != 2:
        raise ValueError("accepted must be a 2-D tensor [batch, up to 64]")
    width = accepted.shape[1]
    check_buffer(accepted, "accepted", (batch, width), torch.int32, dev)
    check_buffer(lens_before, "lens_before", (batch,), torch.int32, dev)
    check_buffer(seq_lens, "seq_lens", (batch,), torch.int32, dev)
    out = _empty((batch,), torch.int32, dev, stream) if out is None else check_buffer(out, "out", (batch,), torch.int32, dev)
    _call(load().bf1_kv_compact, "bf1_kv_compact", dev, stream, _ptr(k_pages), _ptr(v_pages), _ptr(accepted), width,
          _ptr(lens_before), _ptr(seq_lens), _ptr(page_table), batch, max_pages, num_pages, Hkv, d, B, _ptr(out))
    return out


class PageFork(NamedTuple):
    """What page_fork writes: the new page table [batch, max_pages], lengths [batch] and
    head of the free list [1], and the copies to make, [batch] each: copy_rows[b] tokens of
    page copy_from[b] to page copy_to[b] (-1, -1 and 0: none)."""
    page_table: object
    seq_lens: object
    free_head: object
    copy_from: object
    copy_to: object
    copy_rows: object


def page_fork(seq_lens, sources, keep_lens, page_table, shares, free_pages, free_head, B=64, out=None, stream=None):
    """Every place b of the batch goes on with the first keep_lens[b] tokens (at most all)
    of the sequence that place sources[b] holds, or ends where sources[b] is no place: forks,
    beams that change places, tokens taken back, ends.  Returns a PageFork (`out`, if given).

    All are int32.  shares [num_pages] counts the holders of a page beyond the first
    (zeros for a new cache; add 1 to the pages you hold yourself) and is updated, as is
    free_pages, page_step's list with room for every page: pages that nobody holds any more
    go back below the head.  Full blocks are shared; a block that goes on being written
    stays with the first place that continues it, if nobody else holds its page, and is
    copied for the others: kv_copy with the result's lists, for each layer's cache.  Without a
    free page a sequence goes on without that block's tokens.  To run the same call again (a
    warm-up before a capture, a retry), put shares and free_pages back as they were first.

    A CacheQ8's tails belong to places, not to pages: instead of the result's lists, tail
    sources[b] goes to tail b of every place,
    cache.k_tail.copy_(cache.k_tail[sources.clamp(0, batch - 1)]) and v_tail alike (a place that
    ends may get any).  kv_copy does it, tails as pages, where no tail is both read and written
    (samples of one prompt; not places that change about).  There a sequence goes on inside the
    block that its source is writing, or from the end of a full one."""
    if out is None and stream is None:
        r = (_MARSHAL or _native()).page_fork(seq_lens, sources, keep_lens, page_table, shares, free_pages, free_head, B)
        if r is not None:
            return PageFork._make(_done(r, "bf1_page_fork"))
    import torch
    dev = _cuda_device(page_table, "page_table")
    if page_table.dim() != 2:
        raise ValueError("page_table must be a 2-D tensor [batch, max_pages]")
    batch, max_pages = page_table.shape
    check_buffer(page_table, "page_table", page_table.shape, torch.int32, dev)
    for name, t in (("seq_lens", seq_lens), ("sources", sources), ("keep_lens", keep_lens)):
        check_buffer(t, name, (batch,), torch.int32, dev)
    _i32_cuda(shares, "shares", 1, dev)
    _i32_cuda(free_pages, "free_pages", 1, dev)
    check_buffer(free_head, "free_head", (1,), torch.int32, dev)
    sizes = ((batch, max_pages), (batch,), (1,), (batch,), (batch,), (batch,))
    if out is None:
        out = PageFork(*(_empty(s, torch.int32, dev, stream) for s in sizes))
    else:
        out = PageFork(*out)
        for name, t, s in zip(PageFork._fields, out, sizes):
            check_buffer(t, name, s, torch.int32, dev)
    _call(load().bf1_page_fork, "bf1_page_fork", dev, stream, batch, _ptr(seq_lens), _ptr(sources), _ptr(keep_lens),
          _ptr(page_table), max_pages, _ptr(shares), shares.shape[0], _ptr(free_pages), free_pages.shape[0],
          _ptr(free_head), int(B), *(_ptr(t) for t in out))
    return out


def kv_copy(k_pages, v_pages, copy_from, copy_to, copy_rows, stream=None):
    """Copy the first copy_rows[i] tokens of K and V page copy_from[i] to page copy_to[i]
    (int32 lists, page_fork's) in bf16 pages [num_pages, Hkv, B, d]; entries outside the
    cache are left out.  No page is copied to twice, or both to and from: the copies run at
    once."""
    if stream is None:
        r = (_MARSHAL or _native()).kv_copy(k_pages, v_pages, copy_from, copy_to, copy_rows)
        if r is not None:
            return _check(r, "bf1_kv_copy")
    dev, (num_pages, Hkv, B, d) = _bf16_pages(k_pages, v_pages)
    _i32_cuda(copy_from, "copy_from", 1, dev)
    _i32_cuda(copy_to, "copy_to", 1, dev)
    _i32_cuda(copy_rows, "copy_rows", 1, dev)
    if not copy_from.shape == copy_to.shape == copy_rows.shape:
        raise ValueError("copy_from, copy_to and copy_rows must have the same length")
    _call(load().bf1_kv_copy, "bf1_kv_copy", dev, stream, _ptr(k_pages), _ptr(v_pages), _ptr(copy_from), _ptr(copy_to),
          _ptr(copy_rows), copy_from.shape[0], num_pages, Hkv, d, B)
