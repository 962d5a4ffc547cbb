"""BinaryPC decode hot path on AMD Instinct MI355X (gfx950).

A thin ctypes binding over libbpc.so (see include/bpc.h): it only checks
tensor metadata and marshals pointers, strides and the current HIP stream.
Every step of the computation runs in the library's HIP kernels; there is
no Python or CPU fallback.  Importing the package fails loudly when the
library has not been built (``python -m paper_2608_04405_amd.build_lib``).
"""

from __future__ import annotations

import contextlib
import ctypes
import functools
import math
import os
from typing import Optional, Sequence

import torch

__all__ = [
    "BPCError",
    "append_kv",
    "append_kv_paged",
    "attention_cut",
    "chunk_attention",
    "chunk_cut",
    "chunk_workspace_bytes",
    "LIB_PATH",
    "build_hash",
    "build_workspace_bytes",
    "build_checkpoint_workspace_bytes",
    "hash_keys",
    "hash_keys_mm",
    "decode_attention",
    "decode_workspace_bytes",
    "decode_attention_per_head",
    "decode_attention_noalloc",
    "decode_noalloc_max_bytes",
    "decode_per_head_workspace_bytes",
    "dense_attention",
    "evict_kv",
    "evict_workspace_bytes",
    "key_weights",
    "prefill_attention",
    "prefill_workspace_bytes",
    "qk_norm_rope",
    "select_hard",
    "select_hard_workspace_bytes",
    "tree_attention",
    "tree_workspace_bytes",
    "DECODE_STAGES",
    "DECODE_STAGE_NAMES",
    "version",
    "set_decode_path",
    "decode_path_taken",
    "decode_slice_keys",
    "DECODE_ZEROED_BYTES",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbpc.so")
if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2608_04405_amd.build_lib`")

_lib = ctypes.CDLL(LIB_PATH)

_p = ctypes.c_void_p
_i64 = ctypes.c_int64
_i = ctypes.c_int
_sz = ctypes.c_size_t

_lib.bpc_status_string.restype = ctypes.c_char_p
_lib.bpc_status_string.argtypes = [_i]
_lib.bpc_last_error.restype = ctypes.c_char_p
_lib.bpc_last_error.argtypes = []
_lib.bpc_version.restype = _i
_lib.bpc_build_workspace_bytes.restype = _sz
_lib.bpc_build_workspace_bytes.argtypes = [_i, _i, _i, _i, _i]
_lib.bpc_build_checkpoint_workspace_bytes.restype = _sz
_lib.bpc_build_checkpoint_workspace_bytes.argtypes = [_i, _i, _i, _i, _i]
_lib.bpc_build_hash.restype = _i
_lib.bpc_build_hash.argtypes = [_p, _i64, _i64, _i64, _i, _i, _i, _i, _i, _p, _p, _p, _i64, _i64, _p, _p, _p, _sz, _p]
_lib.bpc_hash_keys.restype = _i
_lib.bpc_hash_keys.argtypes = [_p, _i64, _i64, _i64, _i, _i, _i, _i, _i, _p, _i64, _i64, _p, _i64, _i64, _p, _p, _p]
_lib.bpc_hash_keys_mm.restype = _i
_lib.bpc_hash_keys_mm.argtypes = [_p, _i64, _i64, _i64, _i, _i, _i, _i, _i, _p, _i64, _i64, _p, _i64, _i64, _p, _p, _p]
_lib.bpc_decode_workspace_bytes.restype = _sz
_lib.bpc_decode_workspace_bytes.argtypes = [_i, _i, _i, _i, _i, _i, _i]
_DECODE_ARGS = [_p, _p, _i64, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _i64, _p, _i64, _i64,
                _i, _i, _i, _i, _i, _i, _i, ctypes.c_float, _p, _p, _p, _p, _p, _sz, _p]
_lib.bpc_decode_attention.restype = _i
_lib.bpc_decode_attention.argtypes = _DECODE_ARGS
_lib.bpc_decode_per_head_workspace_bytes.restype = _sz
_lib.bpc_decode_per_head_workspace_bytes.argtypes = [_i, _i, _i, _i, _i, _i, _i]
_lib.bpc_decode_attention_per_head.restype = _i
_lib.bpc_decode_attention_per_head.argtypes = _DECODE_ARGS
_lib.bpc_decode_attention_eas.restype = _i
_lib.bpc_decode_attention_eas.argtypes = [_p, _p, _i64, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _i64, _p, _i64, _i64,
                                          _i, _i, _i, _i, _i, _i, _i, ctypes.c_float, _p, _i64, _i64, _i, _p, _p, _p,
                                          _p, _sz, _p]
_lib.bpc_append_kv.restype = _i
_lib.bpc_append_kv.argtypes = [_p, _i64, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64, _i64, _i64,
                               _p, _i64, _i64, _p, _i64, _i64, _i, _i, _i, _i, _i, _i, _i, _p, _p, _p]
_lib.bpc_dense_workspace_bytes.restype = _sz
_lib.bpc_dense_workspace_bytes.argtypes = [_i, _i, _i, _i, _i]
_lib.bpc_dense_attention.restype = _i
_lib.bpc_dense_attention.argtypes = [_p, _p, _i64, _i64, _i64, _p, _i64, _i64, _i64, _i, _i, _i, _i, _i,
                                     ctypes.c_float, _p, _p, _sz, _p]
_lib.bpc_select_hard.restype = _i
_lib.bpc_select_hard.argtypes = [_p, _i64, _i64, _i, _i, _i, _i, _p, _p]
_lib.bpc_select_hard_workspace_bytes.restype = _sz
_lib.bpc_select_hard_workspace_bytes.argtypes = [_i, _i, _i, _i]
_lib.bpc_select_hard_ws.restype = _i
_lib.bpc_select_hard_ws.argtypes = [_p, _i64, _i64, _i, _i, _i, _i, _p, _p, _sz, _p]
_lib.bpc_set_decode_path.restype = _i
_lib.bpc_set_decode_path.argtypes = [_i]
_lib.bpc_decode_slice_keys.restype = _i
_lib.bpc_decode_slice_keys.argtypes = [_i, _i, _i, _i, _i]
_lib.bpc_decode_path_taken.restype = _i
_lib.bpc_decode_path_taken.argtypes = [_i, _i, _i, _i, _i]
_lib.bpc_decode_noalloc_max_bytes.restype = _sz
_lib.bpc_decode_noalloc_max_bytes.argtypes = []
_lib.bpc_decode_attention_noalloc.restype = _i
_lib.bpc_decode_attention_noalloc.argtypes = _DECODE_ARGS[:-3] + [_p]
_lib.bpc_decode_attention_profiled.restype = _i
_lib.bpc_decode_attention_profiled.argtypes = _DECODE_ARGS + [ctypes.POINTER(_p), _i]

_f = ctypes.c_float
_lib.bpc_qk_norm_rope.restype = _i
_ROPE_TENSOR = [_p, _i64, _i64, _i64, _p, _i64, _i64, _i64, _p, _i64]
_lib.bpc_qk_norm_rope.argtypes = _ROPE_TENSOR * 2 + [_i, _i, _i, _i, _i, _f, _p, _i, _i, _i, _p, _i64, _p]
_lib.bpc_append_kv_paged.restype = _i
_lib.bpc_append_kv_paged.argtypes = [_p, _i64, _i64, _i64] * 4 + [_p, _i64, _i, _i, _i, _p, _p, _i, _i, _i, _i,
                                                                  _p, _i64, _f, _p, _i, _i, _i, _p, _i64, _p]
_lib.bpc_prefill_workspace_bytes.restype = _sz
_lib.bpc_prefill_workspace_bytes.argtypes = [_i] * 6
_lib.bpc_prefill_attention.restype = _i
_lib.bpc_prefill_attention.argtypes = [_p, _i64, _i64, _i64] * 3 + [_i] * 7 + [_f, _f, _p, _p, _i64, _p, _i64,
                                                                             _p, _i64, _i64, _i64, _p, _sz, _p]
_lib.bpc_tree_workspace_bytes.restype = _sz
_lib.bpc_tree_workspace_bytes.argtypes = [_i] * 6
_lib.bpc_tree_attention.restype = _i
_lib.bpc_tree_attention.argtypes = [_p, _i64, _i64, _i64] * 3 + [_p, _i64, _i, _i, _p, _p, _i64] + [_i] * 6 + \
    [_f, _f, _p, _p, _i64, _i64, _i64, _p, _sz, _p]

_lib.bpc_chunk_workspace_bytes.restype = _sz
_lib.bpc_chunk_workspace_bytes.argtypes = [_i] * 8
_lib.bpc_chunk_attention.restype = _i
_lib.bpc_chunk_attention.argtypes = [_p, _i64, _i64, _i64] * 3 + [_p, _i64, _i, _i, _p, _p] + [_i] * 6 + \
    [_f, _f, _p, _i, _i, _p, _i64, _i64, _i64, _p, _i64, _i64, _p, _sz, _p]
_lib.bpc_chunk_cut.restype = _i
_lib.bpc_chunk_cut.argtypes = [_i] * 8 + [ctypes.POINTER(_i)] * 3
_lib.bpc_key_weights.restype = _i
_lib.bpc_key_weights.argtypes = [_p, _i64, _i64, _i64] * 2 + [_p, _i64, _i64] * 2 + [_p, _i64, _i, _i, _p, _p] + [_i] * 6 + \
    [_f, _f, _p, _i, _i, _f, _p]
_lib.bpc_evict_workspace_bytes.restype = _sz
_lib.bpc_evict_workspace_bytes.argtypes = [_i] * 4
_lib.bpc_evict_kv.restype = _i
_lib.bpc_evict_kv.argtypes = [_p, _i64, _i64, _i64] * 2 + [_p, _i64, _i, _i, _p, _i64, _i64, _p] + [_i] * 7 + \
    [_p, _i64, _i64, _i64] * 2 + [_p, _i64, _i, _i] + [_p, _i64, _i64] * 2 + [_i, _p, _i64, _i64, _i, _p, _p, _sz, _p]
_lib.bpc_attention_cut.restype = _i
_lib.bpc_attention_cut.argtypes = [_i] * 7 + [ctypes.POINTER(_i)] * 3

DECODE_STAGES = 3
DECODE_STAGE_NAMES = ("score", "attend", "merge")
# a decode workspace's leading bytes that must be zero before its first use
# (the fused path's arrival counters; every call leaves them zero)
DECODE_ZEROED_BYTES = 1088 * 1024


class BPCError(RuntimeError):
    def __init__(self, status: int, where: str):
        msg = _lib.bpc_status_string(status).decode()
        detail = _lib.bpc_last_error().decode()
        super().__init__(f"{where}: {msg} ({status}): {detail}")
        self.status = status


def _check(status: int, where: str) -> None:
    if status != 0:
        raise BPCError(status, where)


def version() -> int:
    return _lib.bpc_version()


def set_decode_path(path: int) -> None:
    """0: a decode step runs as one fused launch whenever its workgroups fit
    on the GPU at once (the default; slices of 2048 to 8192 keys where
    16384-key ones would leave the GPU mostly idle); 1: always the three
    launches; 2: the fused launch on 16384-key slices only."""
    _check(_lib.bpc_set_decode_path(int(path)), "bpc_set_decode_path")


def decode_path_taken(B: int, Hq: int, Hkv: int, N: int, L: int) -> int:
    """0 if a decode step of this shape runs as one fused launch on the
    current device, 1 if as three launches (needs a GPU)."""
    return int(_lib.bpc_decode_path_taken(B, Hq, Hkv, N, L))


def decode_slice_keys(B: int, Hq: int, Hkv: int, N: int, L: int) -> int:
    """Keys per slice (16384, 8192, 4096 or 2048) of a decode step of this shape on the
    current device (needs a GPU)."""
    return int(_lib.bpc_decode_slice_keys(B, Hq, Hkv, N, L))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice()) or None
    return stream.cuda_stream or None


def _need(t: torch.Tensor, name: str, dtype, dim: int) -> None:
    """dtype, number of dims and a contiguous innermost dimension; the device
    is checked separately (`_on_gpu`), after every shape check, so that a
    shape mistake is reported as such wherever the tensors live."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dims, got shape {tuple(t.shape)}")
    if t.numel() and t.stride(-1) != 1:
        raise ValueError(f"{name}: innermost dimension must be contiguous")


def _extent(t: torch.Tensor, name: str, spec) -> None:
    """Check every extent of t against spec: an int is an exact size, ("ge",
    n) a lower bound (a cache with room for more rows), None anything."""
    shape = tuple(t.shape)
    if len(shape) != len(spec):
        raise ValueError(f"{name} must have {len(spec)} dims, got shape {shape}")
    for i, (got, want) in enumerate(zip(shape, spec)):
        if want is None:
            continue
        if isinstance(want, tuple):
            if got < want[1]:
                raise ValueError(f"{name}: dim {i} is {got}, needs at least {want[1]} (shape {shape})")
        elif got != want:
            raise ValueError(f"{name}: dim {i} is {got}, expected {want} (shape {shape})")


def _exact_out(t: Optional[torch.Tensor], name: str, dtype, shape) -> None:
    """An optional output the kernels address as a dense array of `shape`."""
    if t is None:
        return
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of shape {tuple(shape)}, got {tuple(t.shape)}")


def _on_gpu(*tensors) -> None:
    """Every given tensor (None entries skipped) on one GPU."""
    devices = {t.get_device() for t in tensors if t is not None}
    if len(devices) == 1 and -1 not in devices:
        return
    if -1 in devices:
        raise ValueError("every tensor must be on a GPU")
    if devices:
        raise ValueError("tensors on different devices: " + " and ".join(f"cuda:{d}" for d in sorted(devices)))


def _budget(k: int, N: int, Ncap: int) -> None:
    if not 1 <= N <= Ncap:
        raise ValueError(f"N={N} must satisfy 1 <= N <= {Ncap} (the rows the cache holds)")
    if not 1 <= k <= N:
        raise ValueError(f"k={k} must satisfy 1 <= k <= N={N}")


def _kv_strides(t: torch.Tensor):
    return t.stride(0), t.stride(1), t.stride(2)


def _proj(P: torch.Tensor, D: int = 128, B: Optional[int] = None, Hkv: Optional[int] = None):
    """(L, sP_b, sP_h) of a projection given as [B, Hkv, L, D] (one per
    (sequence, KV head)), [Hkv, L, D] (one per KV head, shared by the batch:
    offline calibration) or [L, D] (one for everything).  When B and Hkv are
    given, the leading dims must match them."""
    if not isinstance(P, torch.Tensor) or P.dtype != torch.float32:
        raise TypeError("P must be a float32 tensor")
    if P.dim() not in (2, 3, 4):
        raise ValueError("P must be [B, Hkv, L, 128], [Hkv, L, 128] or [L, 128]")
    if P.stride(-1) != 1 or P.shape[-1] != D or (P.shape[-2] > 1 and P.stride(-2) != D):
        raise ValueError("P rows must be contiguous [.., L, 128]")
    L = P.shape[-2]
    if L not in (32, 64, 128):
        raise ValueError(f"P has {L} rows: the code length must be 32, 64 or 128")
    if P.dim() == 3 and Hkv is not None and P.shape[0] != Hkv:
        raise ValueError(f"P is [Hkv, L, 128] with {P.shape[0]} heads, expected Hkv={Hkv}")
    if P.dim() == 4 and B is not None and (P.shape[0], P.shape[1]) != (B, Hkv):
        raise ValueError(f"P is {tuple(P.shape)}, expected [{B}, {Hkv}, L, 128]")
    if P.dim() == 2:
        return L, 0, 0
    if P.dim() == 3:
        return L, 0, P.stride(0)
    return L, P.stride(0), P.stride(1)


def build_workspace_bytes(B: int, Hkv: int, N: int, L: int, D: int = 128) -> int:
    return int(_lib.bpc_build_workspace_bytes(B, Hkv, N, D, L))


def build_checkpoint_workspace_bytes(B: int, Hkv: int, N: int, L: int, D: int = 128) -> int:
    return int(_lib.bpc_build_checkpoint_workspace_bytes(B, Hkv, N, D, L))


def decode_workspace_bytes(B: int, Hq: int, Hkv: int, N: int, L: int, k: int, D: int = 128) -> int:
    return int(_lib.bpc_decode_workspace_bytes(B, Hq, Hkv, N, D, L, k))


def decode_per_head_workspace_bytes(B: int, Hq: int, Hkv: int, N: int, L: int, k: int, D: int = 128) -> int:
    return int(_lib.bpc_decode_per_head_workspace_bytes(B, Hq, Hkv, N, D, L, k))


def _u32_codes(codes: torch.Tensor, name: str = "codes") -> torch.Tensor:
    # torch has no uint32 arithmetic on every build; int32 storage is used and
    # reinterpreted by the library.
    if not isinstance(codes, torch.Tensor) or codes.dtype not in (torch.int32, torch.uint32):
        raise TypeError(f"{name} must be int32/uint32 storage")
    if codes.dim() != 4 or (codes.numel() and codes.stride(-1) != 1) or (codes.shape[2] > 1 and codes.stride(2) != codes.shape[3]):
        raise ValueError(f"{name} must be [B, Hkv, Ncap, L/32] with the words of a key and the keys of a head contiguous")
    return codes


def _fragile(fragile: Optional[torch.Tensor]) -> None:
    if fragile is not None and (fragile.dtype != torch.int64 or fragile.numel() < 1):
        raise ValueError("fragile must be an int64 tensor with at least one element")


def build_hash(K: torch.Tensor, G: torch.Tensor, N: Optional[int] = None, *,
               P_out: Optional[torch.Tensor] = None, codes_out: Optional[torch.Tensor] = None,
               err_out: Optional[torch.Tensor] = None, fragile: Optional[torch.Tensor] = None,
               workspace: Optional[torch.Tensor] = None, checkpoint: bool = False, stream=None):
    """Binary principal components of every (b, h): returns (P, codes, err).

    K [B, Hkv, >=N, 128] bf16; G [L, 128] fp32 Gaussian directions.  codes
    are int32 storage [B, Hkv, Ncap, L/32] holding the packed bits; err_out,
    when given, is a contiguous [B, Hkv, N] fp32 tensor.  When `fragile` (a
    1-element int64 GPU tensor) is given, the number of fragile sign
    decisions is added to it.  With `checkpoint` the workspace allocated
    here also holds, where that is the faster way (few keys), a checkpoint of
    the fp64 residuals (1 KiB per key); a given workspace enables it by its
    size alone.  Results are the same."""
    _need(K, "K", torch.bfloat16, 4)
    B, Hkv, Ncap, D = K.shape
    N = Ncap if N is None else N
    if not 1 <= N <= Ncap:
        raise ValueError(f"N={N} must satisfy 1 <= N <= {Ncap}")
    _need(G, "G", torch.float32, 2)
    L = G.shape[0]
    _extent(G, "G", (L, D))
    if L not in (32, 64, 128):
        raise ValueError(f"G has {L} rows: the code length must be 32, 64 or 128")
    G = G.contiguous()
    W = L // 32
    if P_out is not None:
        _exact_out(P_out, "P_out", torch.float32, (B, Hkv, L, D))
    if codes_out is not None:
        _u32_codes(codes_out, "codes_out")
        _extent(codes_out, "codes_out", (B, Hkv, ("ge", N), W))
    _exact_out(err_out, "err_out", torch.float32, (B, Hkv, N))
    _fragile(fragile)
    _on_gpu(K, G, P_out, codes_out, err_out, fragile, workspace)
    dev = K.device
    if P_out is None:
        P_out = torch.empty(B, Hkv, L, D, dtype=torch.float32, device=dev)
    if codes_out is None:
        codes_out = torch.zeros(B, Hkv, Ncap, W, dtype=torch.int32, device=dev)
    ws_bytes = (build_checkpoint_workspace_bytes if checkpoint else build_workspace_bytes)(B, Hkv, N, L, D)
    if workspace is None:
        workspace = torch.empty(max(ws_bytes, 1), dtype=torch.uint8, device=dev)
    _check(_lib.bpc_build_hash(_ptr(K), *_kv_strides(K), B, Hkv, N, D, L, _ptr(G), _ptr(P_out),
                               _ptr(codes_out), codes_out.stride(0), codes_out.stride(1), _ptr(err_out),
                               _ptr(fragile), _ptr(workspace), workspace.numel(), _stream(stream)),
           "bpc_build_hash")
    return P_out, codes_out, err_out


def hash_keys(K: torch.Tensor, P: torch.Tensor, N: Optional[int] = None, *,
              codes_out: Optional[torch.Tensor] = None, err_out: Optional[torch.Tensor] = None,
              fragile: Optional[torch.Tensor] = None, stream=None):
    """Hash keys against P (Algorithm 2).  P is [B, Hkv, L, 128], or
    [Hkv, L, 128] / [L, 128] shared across the batch (offline calibration).
    err_out, when given, is a contiguous [B, Hkv, N] fp32 tensor.  Returns
    (codes, err)."""
    _need(K, "K", torch.bfloat16, 4)
    B, Hkv, Ncap, D = K.shape
    N = Ncap if N is None else N
    if not 1 <= N <= Ncap:
        raise ValueError(f"N={N} must satisfy 1 <= N <= {Ncap}")
    L, sPb, sPh = _proj(P, D, B, Hkv)
    if codes_out is not None:
        _u32_codes(codes_out, "codes_out")
        _extent(codes_out, "codes_out", (B, Hkv, ("ge", N), L // 32))
    _exact_out(err_out, "err_out", torch.float32, (B, Hkv, N))
    _fragile(fragile)
    _on_gpu(K, P, codes_out, err_out, fragile)
    if codes_out is None:
        codes_out = torch.zeros(B, Hkv, Ncap, L // 32, dtype=torch.int32, device=K.device)
    _check(_lib.bpc_hash_keys(_ptr(K), *_kv_strides(K), B, Hkv, N, D, L, _ptr(P), sPb, sPh, _ptr(codes_out),
                              codes_out.stride(0), codes_out.stride(1), _ptr(err_out), _ptr(fragile),
                              _stream(stream)),
           "bpc_hash_keys")
    return codes_out, err_out


def hash_keys_mm(K: torch.Tensor, P: torch.Tensor, N: Optional[int] = None, *,
                 codes_out: Optional[torch.Tensor] = None, fragile: Optional[torch.Tensor] = None,
                 fallbacks: Optional[torch.Tensor] = None, stream=None):
    """The codes of hash_keys (Algorithm 2), bit for bit, with the
    projections on the matrix cores and certified signs.  fragile and
    fallbacks are device uint64 accumulators ([1] int64 tensors).  Returns
    codes."""
    _need(K, "K", torch.bfloat16, 4)
    B, Hkv, Ncap, D = K.shape
    N = Ncap if N is None else N
    if not 1 <= N <= Ncap:
        raise ValueError(f"N={N} must satisfy 1 <= N <= {Ncap}")
    L, sPb, sPh = _proj(P, D, B, Hkv)
    if codes_out is not None:
        _u32_codes(codes_out, "codes_out")
        _extent(codes_out, "codes_out", (B, Hkv, ("ge", N), L // 32))
    _fragile(fragile)
    _fragile(fallbacks)
    _on_gpu(K, P, codes_out, fragile, fallbacks)
    if codes_out is None:
        codes_out = torch.zeros(B, Hkv, Ncap, L // 32, dtype=torch.int32, device=K.device)
    _check(_lib.bpc_hash_keys_mm(_ptr(K), *_kv_strides(K), B, Hkv, N, D, L, _ptr(P), sPb, sPh, _ptr(codes_out),
                                 codes_out.stride(0), codes_out.stride(1), _ptr(fragile), _ptr(fallbacks),
                                 _stream(stream)),
           "bpc_hash_keys_mm")
    return codes_out


def _decode_inputs(q, K, V, codes, P, k, N):
    """Shape checks shared by the decode entry points; returns the sizes."""
    _need(q, "q", torch.bfloat16, 3)
    _need(K, "K", torch.bfloat16, 4)
    _need(V, "V", torch.bfloat16, 4)
    if not q.is_contiguous():
        raise ValueError("q must be contiguous")
    B, Hq, D = q.shape
    _, Hkv, Ncap, _ = K.shape
    N = Ncap if N is None else N
    _extent(K, "K", (B, Hkv, ("ge", 1), D))
    _budget(k, N, Ncap)
    _extent(V, "V", (B, Hkv, ("ge", N), D))
    if Hq % Hkv:
        raise ValueError(f"Hq={Hq} must be a multiple of Hkv={Hkv}")
    L, sPb, sPh = _proj(P, D, B, Hkv)
    _u32_codes(codes)
    _extent(codes, "codes", (B, Hkv, ("ge", N), L // 32))
    return B, Hq, Hkv, D, N, L, sPb, sPh


def decode_attention(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, codes: torch.Tensor,
                     P: torch.Tensor, k: int, sm_scale: Optional[float] = None, N: Optional[int] = None, *,
                     out: Optional[torch.Tensor] = None, idx_out: Optional[torch.Tensor] = None,
                     score_out: Optional[torch.Tensor] = None, qcode_out: Optional[torch.Tensor] = None,
                     serr: Optional[torch.Tensor] = None, added_out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None, stream=None,
                     events: Optional[Sequence] = None) -> torch.Tensor:
    """One BinaryPC decode step; returns out [B, Hq, 128] fp32.

    q [B, Hq, 128] bf16 contiguous; K, V [B, Hkv, >=N, 128] bf16; codes
    int32 storage [B, Hkv, >=N, L/32]; P [B, Hkv, L, 128] fp32, or shared
    across the batch as [Hkv, L, 128] (offline calibration) or [L, 128].
    Optional debug outputs (contiguous): idx_out [B, Hkv, k] int32,
    score_out [B, Hkv, N] int32, qcode_out [B, Hkv, 8, L/32] int32.
    `events`: BPC_DECODE_STAGES + 1 torch.cuda.Event objects recorded at the
    stage boundaries (for measurement).

    With `serr` [B, Hkv, m] int32 (the hard-to-hash set from select_hard),
    attention runs over the union of the k hash-selected keys and serr (the
    error-aware safeguard); added_out [B, Hkv, m] int32 then marks the
    entries of serr that the hash selection had not taken."""
    B, Hq, Hkv, D, N, L, sPb, sPh = _decode_inputs(q, K, V, codes, P, k, N)
    _exact_out(out, "out", torch.float32, (B, Hq, D))
    _exact_out(idx_out, "idx_out", torch.int32, (B, Hkv, k))
    _exact_out(score_out, "score_out", torch.int32, (B, Hkv, N))
    _exact_out(qcode_out, "qcode_out", torch.int32, (B, Hkv, 8, L // 32))
    m = 0
    if serr is not None:
        if events is not None or score_out is not None or qcode_out is not None:
            raise ValueError("serr cannot be combined with events, score_out or qcode_out")
        if not isinstance(serr, torch.Tensor) or serr.dtype != torch.int32 or serr.dim() != 3 or \
                (serr.numel() and serr.stride(-1) != 1):
            raise ValueError("serr must be a [B, Hkv, m] int32 tensor, innermost dimension contiguous")
        _extent(serr, "serr", (B, Hkv, None))
        m = serr.shape[-1]
        if m > N:
            raise ValueError(f"serr holds m={m} keys per head, more than N={N}")
        _exact_out(added_out, "added_out", torch.int32, (B, Hkv, m))
    elif added_out is not None:
        raise ValueError("added_out needs serr")
    if workspace is not None and (workspace.dtype != torch.uint8 or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor")
    _on_gpu(q, K, V, codes, P, out, idx_out, score_out, qcode_out, serr, added_out, workspace)
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty(B, Hq, D, dtype=torch.float32, device=q.device)
    ws_bytes = decode_workspace_bytes(B, Hq, Hkv, N, L, k, D)
    if workspace is None:
        workspace = torch.zeros(max(ws_bytes, 1), dtype=torch.uint8, device=q.device)
    args = [_ptr(q), _ptr(K), *_kv_strides(K), _ptr(V), *_kv_strides(V), _ptr(codes), codes.stride(0),
            codes.stride(1), _ptr(P), sPb, sPh, B, Hq, Hkv, N, D, L, k, float(sm_scale), _ptr(out),
            _ptr(idx_out), _ptr(score_out), _ptr(qcode_out), _ptr(workspace), workspace.numel(),
            _stream(stream)]
    if serr is not None:
        _check(_lib.bpc_decode_attention_eas(*args[:23], _ptr(serr), serr.stride(0), serr.stride(1), m, _ptr(out),
                                             _ptr(idx_out), _ptr(added_out), _ptr(workspace), workspace.numel(),
                                             _stream(stream)),
               "bpc_decode_attention_eas")
    elif events is None:
        _check(_lib.bpc_decode_attention(*args), "bpc_decode_attention")
    else:
        handles = (_p * len(events))()
        st = torch.cuda.current_stream() if stream is None else stream
        for i, ev in enumerate(events):
            if ev.cuda_event == 0:  # torch creates the event lazily on first record
                ev.record(st)
            handles[i] = ev.cuda_event
        _check(_lib.bpc_decode_attention_profiled(*args, handles, len(events)), "bpc_decode_attention_profiled")
    return out


def decode_noalloc_max_bytes() -> int:
    """Size of the library's static decode scratch (the limit of
    decode_attention_noalloc)."""
    return int(_lib.bpc_decode_noalloc_max_bytes())


def decode_attention_noalloc(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, codes: torch.Tensor,
                             P: torch.Tensor, k: int, out: torch.Tensor, sm_scale: Optional[float] = None,
                             N: Optional[int] = None, *, idx_out: Optional[torch.Tensor] = None,
                             score_out: Optional[torch.Tensor] = None, qcode_out: Optional[torch.Tensor] = None,
                             stream=None) -> torch.Tensor:
    """decode_attention with the library's static scratch as the workspace:
    the call allocates no device memory (the caller passes `out`).  Calls on
    one GPU share the scratch, so calls that overlap in time race."""
    B, Hq, Hkv, D, N, L, sPb, sPh = _decode_inputs(q, K, V, codes, P, k, N)
    if out is None:
        raise ValueError("out is required (the call allocates nothing)")
    _exact_out(out, "out", torch.float32, (B, Hq, D))
    _exact_out(idx_out, "idx_out", torch.int32, (B, Hkv, k))
    _exact_out(score_out, "score_out", torch.int32, (B, Hkv, N))
    _exact_out(qcode_out, "qcode_out", torch.int32, (B, Hkv, 8, L // 32))
    _on_gpu(q, K, V, codes, P, out, idx_out, score_out, qcode_out)
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(D)
    _check(_lib.bpc_decode_attention_noalloc(
        _ptr(q), _ptr(K), *_kv_strides(K), _ptr(V), *_kv_strides(V), _ptr(codes), codes.stride(0), codes.stride(1),
        _ptr(P), sPb, sPh, B, Hq, Hkv, N, D, L, k, float(sm_scale), _ptr(out), _ptr(idx_out), _ptr(score_out),
        _ptr(qcode_out), _stream(stream)), "bpc_decode_attention_noalloc")
    return out


def decode_attention_per_head(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, codes: torch.Tensor,
                              P: torch.Tensor, k: int, sm_scale: Optional[float] = None, N: Optional[int] = None, *,
                              out: Optional[torch.Tensor] = None, idx_out: Optional[torch.Tensor] = None,
                              score_out: Optional[torch.Tensor] = None, qcode_out: Optional[torch.Tensor] = None,
                              workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The decode step with one selection per query head: query head j
    quantises its own projection, scores the codes of KV head j // G, takes
    its own top-k and attends over it.  Shapes as decode_attention, except
    idx_out [B, Hq, k], score_out [B, Hq, N], qcode_out [B, Hq, 8, L/32]."""
    B, Hq, Hkv, D, N, L, sPb, sPh = _decode_inputs(q, K, V, codes, P, k, N)
    _exact_out(out, "out", torch.float32, (B, Hq, D))
    _exact_out(idx_out, "idx_out", torch.int32, (B, Hq, k))
    _exact_out(score_out, "score_out", torch.int32, (B, Hq, N))
    _exact_out(qcode_out, "qcode_out", torch.int32, (B, Hq, 8, L // 32))
    if workspace is not None and (workspace.dtype != torch.uint8 or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor")
    _on_gpu(q, K, V, codes, P, out, idx_out, score_out, qcode_out, workspace)
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty(B, Hq, D, dtype=torch.float32, device=q.device)
    ws_bytes = decode_per_head_workspace_bytes(B, Hq, Hkv, N, L, k, D)
    if workspace is None:
        workspace = torch.zeros(max(ws_bytes, 1), dtype=torch.uint8, device=q.device)
    _check(_lib.bpc_decode_attention_per_head(
        _ptr(q), _ptr(K), *_kv_strides(K), _ptr(V), *_kv_strides(V), _ptr(codes), codes.stride(0), codes.stride(1),
        _ptr(P), sPb, sPh, B, Hq, Hkv, N, D, L, k, float(sm_scale), _ptr(out), _ptr(idx_out), _ptr(score_out),
        _ptr(qcode_out), _ptr(workspace), workspace.numel(), _stream(stream)), "bpc_decode_attention_per_head")
    return out


def select_hard_workspace_bytes(B: int, Hkv: int, N: int, m: int) -> int:
    """Bytes of workspace with which select_hard reads its errors only once
    (0 where that would not help)."""
    return int(_lib.bpc_select_hard_workspace_bytes(B, Hkv, N, m))


def select_hard(err: torch.Tensor, m: int, N: Optional[int] = None, *, serr_out: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The error-aware safeguard's hard-to-hash set: per (b, KV head), the m
    keys with the largest reconstruction errors (err [B, Hkv, >=N] fp32, as
    written by build_hash / hash_keys), ascending; returns [B, Hkv, m] int32.
    `workspace` (uint8, select_hard_workspace_bytes) is allocated here where it
    helps and is not given; not while a stream is being captured, whose graph
    would outlive it: there the selection without a workspace runs, the same
    set in more passes."""
    _need(err, "err", torch.float32, 3)
    B, Hkv, Ncap = err.shape
    N = Ncap if N is None else N
    if not 1 <= N <= Ncap:
        raise ValueError(f"N={N} must satisfy 1 <= N <= {Ncap}")
    if not 0 <= m <= N:
        raise ValueError(f"m={m} must satisfy 0 <= m <= N={N}")
    _exact_out(serr_out, "serr_out", torch.int32, (B, Hkv, m))
    _on_gpu(err, serr_out, workspace)
    if serr_out is None:
        serr_out = torch.empty(B, Hkv, m, dtype=torch.int32, device=err.device)
    size = select_hard_workspace_bytes(B, Hkv, N, m)
    if size and workspace is None and (stream is None or isinstance(stream, torch.cuda.Stream)):
        # allocated on the stream that uses it, so that its memory is not
        # reused elsewhere while the kernels run
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            if not torch.cuda.is_current_stream_capturing():
                workspace = torch.empty(size, dtype=torch.uint8, device=err.device)
    args = (_ptr(err), err.stride(0), err.stride(1), B, Hkv, N, m, _ptr(serr_out))
    if size and workspace is not None:
        _check(_lib.bpc_select_hard_ws(*args, _ptr(workspace), workspace.numel(), _stream(stream)), "bpc_select_hard")
    else:
        _check(_lib.bpc_select_hard(*args, _stream(stream)), "bpc_select_hard")
    return serr_out


def append_kv(k_new: torch.Tensor, v_new: torch.Tensor, K: torch.Tensor, V: torch.Tensor, codes: torch.Tensor,
              P: torch.Tensor, pos: int, *, err_out: Optional[torch.Tensor] = None,
              fragile: Optional[torch.Tensor] = None, stream=None) -> None:
    """Decode-time append: store k_new, v_new [B, Hkv, T, 128] bf16 at rows
    [pos, pos + T) of the caches K, V [B, Hkv, Ncap, 128] and their codes
    (Algorithm 2 against P, [B, Hkv, L, 128] or a shared [L, 128]) at the same
    rows of codes [B, Hkv, Ncap, L/32].  err_out, when given, is a
    contiguous [B, Hkv, T] fp32 tensor."""
    for t, nm in ((k_new, "k_new"), (v_new, "v_new"), (K, "K"), (V, "V")):
        _need(t, nm, torch.bfloat16, 4)
    B, Hkv, T, D = k_new.shape
    _extent(v_new, "v_new", (B, Hkv, T, D))
    Ncap = K.shape[2]
    _extent(K, "K", (B, Hkv, Ncap, D))
    _extent(V, "V", (B, Hkv, ("ge", Ncap), D))
    if T < 1 or pos < 0 or pos + T > Ncap:
        raise ValueError(f"pos={pos}, T={T}: the new rows must lie within the {Ncap} cache rows")
    L, sPb, sPh = _proj(P, D, B, Hkv)
    _u32_codes(codes)
    _extent(codes, "codes", (B, Hkv, ("ge", pos + T), L // 32))
    _exact_out(err_out, "err_out", torch.float32, (B, Hkv, T))
    _fragile(fragile)
    _on_gpu(k_new, v_new, K, V, codes, P, err_out, fragile)
    _check(_lib.bpc_append_kv(_ptr(k_new), *_kv_strides(k_new), _ptr(v_new), *_kv_strides(v_new), _ptr(K),
                              *_kv_strides(K), _ptr(V), *_kv_strides(V), _ptr(codes), codes.stride(0),
                              codes.stride(1), _ptr(P), sPb, sPh, B, Hkv, Ncap, pos, T, D, L, _ptr(err_out),
                              _ptr(fragile), _stream(stream)),
           "bpc_append_kv")


def dense_attention(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, sm_scale: Optional[float] = None,
                    N: Optional[int] = None, *, out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense decode attention over all N cached keys (the comparison point
    for the sparse step); returns out [B, Hq, 128] fp32."""
    _need(q, "q", torch.bfloat16, 3)
    _need(K, "K", torch.bfloat16, 4)
    _need(V, "V", torch.bfloat16, 4)
    if not q.is_contiguous():
        raise ValueError("q must be contiguous")
    B, Hq, D = q.shape
    _, Hkv, Ncap, _ = K.shape
    N = Ncap if N is None else N
    _extent(K, "K", (B, Hkv, ("ge", N), D))
    _extent(V, "V", (B, Hkv, ("ge", N), D))
    if not 1 <= N or Hq % Hkv:
        raise ValueError(f"N={N} must be >= 1 and Hq={Hq} a multiple of Hkv={Hkv}")
    _exact_out(out, "out", torch.float32, (B, Hq, D))
    _on_gpu(q, K, V, out, workspace)
    if sm_scale is None:
        sm_scale = 1.0 / math.sqrt(D)
    if out is None:
        out = torch.empty(B, Hq, D, dtype=torch.float32, device=q.device)
    need = int(_lib.bpc_dense_workspace_bytes(B, Hq, Hkv, N, D))
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=q.device)
    _check(_lib.bpc_dense_attention(_ptr(q), _ptr(K), *_kv_strides(K), _ptr(V), *_kv_strides(V), B, Hq, Hkv, N, D,
                                    float(sm_scale), _ptr(out), _ptr(workspace), workspace.numel(), _stream(stream)),
           "bpc_dense_attention")
    return out


# ---------------------------------------------------------------------------
# Rows on their way into the cache, and attention of many query rows
# ---------------------------------------------------------------------------
def _rows(t: torch.Tensor, name: str):
    """(B, H, T, their strides) of a bf16 [B, H, T, 128] tensor with contiguous
    rows; the stride of an extent of one, which torch leaves open, as 0."""
    if type(t) is torch.Tensor and t.dtype is torch.bfloat16 and t.dim() == 4:
        a, b, c, d = t.shape
        x, y, z, one = t.stride()
        if d == 128 and one == 1 and a and b and c:
            return a, b, c, x if a > 1 else 0, y if b > 1 else 0, z if c > 1 else 0
    _need(t, name, torch.bfloat16, 4)
    _extent(t, name, (("ge", 1), ("ge", 1), ("ge", 1), 128))
    (a, b, c, _), (x, y, z, _) = t.shape, t.stride()
    return a, b, c, x if a > 1 else 0, y if b > 1 else 0, z if c > 1 else 0


def _indices(t: Optional[torch.Tensor], name: str, shape, dtype=torch.int32) -> int:
    """Checks an index array (1 or 2 dims, innermost contiguous); returns its
    batch stride.  An expanded batch dimension (stride 0) shares one row."""
    if t is None:
        return 0
    if type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return shape[-1] if len(shape) == 2 else 0
    _need(t, name, dtype, len(shape))
    _extent(t, name, shape)
    return t.stride(0) if len(shape) == 2 and shape[0] > 1 else 0


def _cache(t: torch.Tensor, name: str):
    """As _rows, with the strides that the C entries take a cache's to be."""
    a, b, c, x, y, z = _rows(t, name)
    return a, b, c, (x, y, z if c > 1 else 128)


def _written(t: torch.Tensor, name: str, B: Optional[int] = None, H: Optional[int] = None, T: Optional[int] = None):
    """The strides of a [B, H, T, 128] tensor whose rows a call writes, behind its
    extents where these are not given."""
    a, b, c, x, y, z = _rows(t, name)
    if B is not None and (a != B or b != H or c != T):
        _extent(t, name, (B, H, T, 128))
    if (z < 128 or y < z * c or x < y * b) and not t.is_contiguous():
        span = 128  # a stride is no smaller than what those below it span
        for stride, extent in sorted(((x, a), (y, b), (z, c))):
            if extent > 1:
                if stride < span:
                    raise ValueError(f"{name}: its rows must not overlap (strides {tuple(t.stride())})")
                span += stride * (extent - 1)
    return (x, y, z) if B is not None else (a, b, c, (x, y, z))


def _dense(B: int, H: int, T: int):
    """The strides of a contiguous [B, H, T, 128] tensor."""
    return H * T * 128, T * 128, 128


def _norm_weight(w: Optional[torch.Tensor], name: str, H: int) -> int:
    """Head stride of norm weights given as [128] (one row for all heads) or [H, 128]."""
    if w is None:
        return 0
    if type(w) is torch.Tensor and w.dtype is torch.bfloat16 and w.shape == (128,) and w.is_contiguous():
        return 0
    if isinstance(w, torch.Tensor) and w.dim() == 1:
        _need(w, name, torch.bfloat16, 1)
        _extent(w, name, (128,))
        return 0
    _need(w, name, torch.bfloat16, 2)
    _extent(w, name, (H, 128))
    return w.stride(0) if H > 1 else 0


def _table(cos_sin: Optional[torch.Tensor]):
    """(rows, R) of a rotation table [positions, R]; (0, 0) without one."""
    if cos_sin is None:
        return 0, 0
    if type(cos_sin) is not torch.Tensor or cos_sin.dtype is not torch.float32 or cos_sin.dim() != 2:
        _need(cos_sin, "cos_sin", torch.float32, 2)
    rows, R = cos_sin.shape
    if rows < 1 or R % 16 or not 16 <= R <= 128 or not cos_sin.is_contiguous():
        raise ValueError(f"cos_sin must be a contiguous [positions, R] tensor, R a multiple of 16 up to 128, got {(rows, R)}")
    return rows, R


def _block_table(t: torch.Tensor, B: int):
    """(batch stride, pages of a sequence) of a page table [B, pages]."""
    if type(t) is not torch.Tensor or t.dtype is not torch.int32 or t.dim() != 2 or t.stride(1) != 1:
        _need(t, "block_table", torch.int32, 2)
    b, n = t.shape
    if b != B or n < 1:
        _extent(t, "block_table", (B, ("ge", 1)))
    return t.stride(0) if B > 1 else 0, n


def _page_rows(page: int) -> None:
    if page < 16 or page > 1 << 20 or page & (page - 1):
        raise ValueError(f"K: pages of {page} rows, must be a power of two, 16 to 2^20")


@contextlib.contextmanager
def _place(t: torch.Tensor, stream):
    """t's device and, when given, `stream` as the current ones: what a call
    allocates then belongs to the stream that uses it, and its memory is not
    reused elsewhere while the kernels run."""
    if stream is not None:
        if not isinstance(stream, torch.cuda.Stream):
            raise TypeError("stream must be a torch.cuda.Stream")
        if stream.device != t.device:
            raise ValueError(f"the stream is on {stream.device}, the tensors are on {t.device}")
    with torch.cuda.device(t.device):
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            yield


_current_device = torch._C._cuda_getDevice
_current_stream = torch._C._cuda_getCurrentRawStream


_NO_ROWS = (None, 0, 0, 0, None, 0, 0, 0, None, 0)


def qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], pos: Optional[torch.Tensor],
                 cos_sin: Optional[torch.Tensor], *, wq: Optional[torch.Tensor] = None,
                 wk: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
    """RMS norm of each head's queries and keys and their rotation by position,
    in one pass; returns (q_out, k_out), allocated where not given.

    q [B, Hq, T, 128] and k [B, Hkv, T, 128] bf16, any strides over contiguous
    rows (views of a fused projection, say); either may be None.  wq, wk: norm
    weights [128] or [H, 128] bf16; None: no norm.  cos_sin [positions, R] fp32:
    R/2 cosines, then R/2 sines of each position, rotating the first R
    coordinates (R a multiple of 16, up to 128) in pairs (i, i + R/2), or
    (2i, 2i + 1) with `interleaved`; None: no rotation.  pos [B, T] int32; the
    rows of a token whose position is not in the table are not written.
    q_out, k_out may be q and k themselves, or the rows of a cache, but overlap
    neither input otherwise, nor one another."""
    if q is None and k is None:
        raise ValueError("q and k cannot both be None")
    Hq = Hkv = 0
    if q is not None:
        B, Hq, T, *sq = _rows(q, "q")
    if k is not None:
        kB, Hkv, kT, *sk = _rows(k, "k")
        if q is None:
            B, T = kB, kT
        elif kB != B or kT != T:
            _extent(k, "k", (B, Hkv, T, 128))
    for t, src, nm in ((q_out, q, "q_out"), (k_out, k, "k_out")):
        if t is not None and src is None:
            raise ValueError(f"{nm} is given without its input")
    sqo = _dense(B, Hq, T) if q_out is None else _written(q_out, "q_out", B, Hq, T)
    sko = _dense(B, Hkv, T) if k_out is None else _written(k_out, "k_out", B, Hkv, T)
    rows, R = _table(cos_sin)
    sp = 0
    if not R:
        pos = None
    elif pos is None:
        raise ValueError("pos is required with cos_sin")
    else:
        sp = _indices(pos, "pos", (B, T))
    swq, swk = _norm_weight(wq, "wq", Hq), _norm_weight(wk, "wk", Hkv)
    _on_gpu(q, k, pos, cos_sin, wq, wk, q_out, k_out)
    some = k if q is None else q
    dev = some.get_device()
    if stream is not None or dev != _current_device():
        with _place(some, stream):
            return qk_norm_rope(q, k, pos, cos_sin, wq=wq, wk=wk, eps=eps, interleaved=interleaved, q_out=q_out, k_out=k_out)
    if q is not None and q_out is None:
        q_out = q.new_empty((B, Hq, T, 128))
    if k is not None and k_out is None:
        k_out = k.new_empty((B, Hkv, T, 128))
    status = _lib.bpc_qk_norm_rope(
        *(_NO_ROWS if q is None else (q.data_ptr(), *sq, q_out.data_ptr(), *sqo, _ptr(wq), swq)),
        *(_NO_ROWS if k is None else (k.data_ptr(), *sk, k_out.data_ptr(), *sko, _ptr(wk), swk)),
        B, Hq, Hkv, T, 128, eps, _ptr(cos_sin), rows, R, interleaved, _ptr(pos), sp, _current_stream(dev))
    if status:
        _check(status, "bpc_qk_norm_rope")
    return q_out, k_out


def append_kv_paged(k_new: torch.Tensor, v_new: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                    block_table: torch.Tensor, pos: torch.Tensor, *, count: Optional[torch.Tensor] = None,
                    cos_sin: Optional[torch.Tensor] = None, rope_pos: Optional[torch.Tensor] = None,
                    wk: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                    stream=None) -> None:
    """Append to a paged cache, each sequence at its own length: token t of
    k_new, v_new [B, Hkv, T, 128] bf16 (t < count[b], int32 [B], default T) goes
    to slot pos[b] + t, that is row slot % page of page block_table[b, slot //
    page] of the pools K, V [pages, Hkv, page, 128] (page a power of two from 16
    on), its key normed with wk and rotated as by qk_norm_rope on the way, by
    its slot or by rope_pos [B, T].  Tokens without a page, or without a row of
    cos_sin, are not stored."""
    B, Hkv, T, *skn = _rows(k_new, "k_new")
    vB, vH, vT, *svn = _rows(v_new, "v_new")
    if vB != B or vH != Hkv or vT != T:
        _extent(v_new, "v_new", (B, Hkv, T, 128))
    pages, Hk, page, *_ = _rows(K, "K")
    sK, sV = _written(K, "K", pages, Hkv, page), _written(V, "V", pages, Hkv, page)
    _page_rows(page)
    st, max_pages = _block_table(block_table, B)
    _indices(pos, "pos", (B,))
    _indices(count, "count", (B,))
    rows, R = _table(cos_sin)
    if rope_pos is not None and not R:
        raise ValueError("rope_pos needs cos_sin")
    sr = _indices(rope_pos, "rope_pos", (B, T))
    sw = _norm_weight(wk, "wk", Hkv)
    _on_gpu(k_new, v_new, K, V, block_table, pos, count, cos_sin, rope_pos, wk)
    dev = K.get_device()
    if stream is not None or dev != _current_device():
        with _place(K, stream):
            return append_kv_paged(k_new, v_new, K, V, block_table, pos, count=count, cos_sin=cos_sin, rope_pos=rope_pos,
                                   wk=wk, eps=eps, interleaved=interleaved)
    status = _lib.bpc_append_kv_paged(
        k_new.data_ptr(), *skn, v_new.data_ptr(), *svn, K.data_ptr(), *sK, V.data_ptr(), *sV, block_table.data_ptr(), st,
        max_pages, pages, page, pos.data_ptr(), _ptr(count), B, Hkv, T, 128, _ptr(wk), sw, eps, _ptr(cos_sin), rows, R,
        interleaved, _ptr(rope_pos), sr, _current_stream(dev))
    if status:
        _check(status, "bpc_append_kv_paged")


@functools.lru_cache(maxsize=4096)  # (sizes alone decide it)
def prefill_workspace_bytes(B: int, Hq: int, Hkv: int, T: int, N: int, D: int = 128) -> int:
    return int(_lib.bpc_prefill_workspace_bytes(B, Hq, Hkv, T, N, D))


@functools.lru_cache(maxsize=4096)
def tree_workspace_bytes(B: int, Hq: int, Hkv: int, T: int, N: int, D: int = 128) -> int:
    return int(_lib.bpc_tree_workspace_bytes(B, Hq, Hkv, T, N, D))


def attention_cut(B: int, Hq: int, Hkv: int, T: int, N: int, D: int = 128, tree: bool = False):
    """(row_blocks, pieces, streamed): the blocks of 32 rows (1, 4 or 8) of a
    workgroup, the pieces of the key axis, and whether keys and values pass the
    last-level cache by, in prefill_attention or (tree) tree_attention of these
    sizes."""
    row_blocks, pieces, streamed = _i(), _i(), _i()
    _check(_lib.bpc_attention_cut(B, Hq, Hkv, T, N, D, tree, row_blocks, pieces, streamed), "bpc_attention_cut")
    return row_blocks.value, pieces.value, bool(streamed.value)


_SM_SCALE = 1.0 / math.sqrt(128)


def _attn_inputs(q, K, V, slopes, out, workspace):
    """Checks shared by prefill_attention and tree_attention; returns the sizes
    and strides of q and out, and those of K and V."""
    B, Hq, T, *sq = _rows(q, "q")
    Kb, Hkv, Kn, sK = _cache(K, "K")
    Vb, Vh, Vn, sV = _cache(V, "V")
    if Hq % Hkv:
        raise ValueError(f"Hq={Hq} must be a multiple of Hkv={Hkv}")
    if slopes is not None:
        _need(slopes, "slopes", torch.float32, 1)
        _extent(slopes, "slopes", (Hq,))
    so = _dense(B, Hq, T) if out is None else _written(out, "out", B, Hq, T)
    if workspace is not None and (workspace.dtype != torch.uint8 or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor")
    return B, Hq, Hkv, T, sq, so, Kb, Kn, sK, Vb, Vh, Vn, sV


def _cache_rows(K, V, B, Hkv, N) -> None:
    _extent(K, "K", (B, Hkv, ("ge", N), 128))
    _extent(V, "V", (B, Hkv, ("ge", N), 128))


def prefill_attention(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, sm_scale: Optional[float] = None,
                      N: Optional[int] = None, *, pos0: Optional[int] = None, softcap: float = 0.0,
                      slopes: Optional[torch.Tensor] = None, key_begin: Optional[torch.Tensor] = None,
                      key_end: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense attention of a prefill: q [B, Hq, T, 128] bf16 over the first N of
    the cached keys K, V [B, Hkv, >=N, 128]; returns out [B, Hq, T, 128] bf16.

    Query t has position pos0 + t (default: the queries are the last T of the N
    tokens) and sees keys key_begin[b, t] <= n < key_end[b, t] (int32 [B, T];
    default: from 0, to its own position, both clipped to [0, N)): begin at each
    document's first token for a document mask, end at the prefix's end for a
    prefix mask.  Scores are capped to softcap * tanh(s / softcap) when softcap
    > 0, then lowered by slopes[head] * distance.  A token that sees nothing
    gets zeros.  `out` overlaps no input."""
    B, Hq, Hkv, T, sq, so, Kb, Kn, sK, Vb, Vh, Vn, sV = _attn_inputs(q, K, V, slopes, out, workspace)
    N = Kn if N is None else N
    if N < 1:
        raise ValueError(f"N={N} must be >= 1")
    if Kb != B or Vb != B or Vh != Hkv or Kn < N or Vn < N:
        _cache_rows(K, V, B, Hkv, N)
    if pos0 is None:
        if T > N:
            raise ValueError(f"{T} queries are more than the N={N} tokens: pos0 must be given")
        pos0 = N - T
    if not 0 <= pos0 <= 1 << 30:
        raise ValueError(f"pos0={pos0} must be in [0, 2^30]")
    sb = _indices(key_begin, "key_begin", (B, T))
    se = _indices(key_end, "key_end", (B, T))
    _on_gpu(q, K, V, slopes, key_begin, key_end, out, workspace)
    dev = q.get_device()
    if stream is not None or dev != _current_device():
        with _place(q, stream):
            return prefill_attention(q, K, V, sm_scale, N, pos0=pos0, softcap=softcap, slopes=slopes, key_begin=key_begin,
                                     key_end=key_end, out=out, workspace=workspace)
    if out is None:
        out = q.new_empty((B, Hq, T, 128))
    if workspace is None:
        need = prefill_workspace_bytes(B, Hq, Hkv, T, N)
        if need:
            workspace = q.new_empty(need, dtype=torch.uint8)
    status = _lib.bpc_prefill_attention(
        q.data_ptr(), *sq, K.data_ptr(), *sK, V.data_ptr(), *sV, B, Hq, Hkv, T, N, pos0, 128,
        _SM_SCALE if sm_scale is None else sm_scale, softcap, _ptr(slopes), _ptr(key_begin), sb, _ptr(key_end), se,
        out.data_ptr(), *so, _ptr(workspace), 0 if workspace is None else workspace.numel(), _current_stream(dev))
    if status:
        _check(status, "bpc_prefill_attention")
    return out


def tree_attention(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, lens: torch.Tensor,
                   tree: Optional[torch.Tensor] = None, sm_scale: Optional[float] = None, N: Optional[int] = None, *,
                   block_table: Optional[torch.Tensor] = None, softcap: float = 0.0,
                   slopes: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense attention of T <= 64 drafted tokens q [B, Hq, T, 128] bf16 over the
    cache that holds them, sequence b's at slots lens[b] .. lens[b] + T - 1 (lens
    int32 [B]); returns out [B, Hq, T, 128] bf16.

    Draft t sees the slots below lens[b] and the drafts j whose bit is set in
    tree[b, t] (int64 [B, T]; None: a chain, drafts 0..t).  K, V are the
    contiguous cache [B, Hkv, >=N, 128], or with block_table (int32 [B, pages of
    a sequence]) pools of pages [pages, Hkv, page, 128] as append_kv_paged writes
    them.  N: slots that any sequence may use (default: what the cache or the
    table holds); one near the longest sequence cuts the work best.  softcap and slopes as in prefill_attention, a draft's position
    being lens[b] plus its depth.  A sequence whose lens[b] is not in [0, N - T]
    is skipped: its rows of `out` stay as they are (undefined where `out` is
    allocated here)."""
    B, Hq, Hkv, T, sq, so, Kb, Kn, sK, Vb, Vh, Vn, sV = _attn_inputs(q, K, V, slopes, out, workspace)
    pages = page = st = 0
    if block_table is None:
        N = Kn if N is None else N
        if Kb != B or Vb != B or Vh != Hkv or Kn < N or Vn < N:
            _cache_rows(K, V, B, Hkv, N)
    else:
        pages, page = Kb, Kn
        if Vb != pages or Vh != Hkv or Vn != page:
            _extent(V, "V", (pages, Hkv, page, 128))
        _page_rows(page)
        st, most = _block_table(block_table, B)
        most *= page
        N = min(most, 1 << 30) if N is None else N
        if N > most:
            raise ValueError(f"N={N}: the block_table holds {most} slots per sequence")
    if not 1 <= T <= min(64, N):
        raise ValueError(f"T={T} drafted tokens: must be 1 to 64, and at most N={N}")
    _indices(lens, "lens", (B,))
    sm = _indices(tree, "tree", (B, T), torch.int64)
    _on_gpu(q, K, V, lens, tree, block_table, slopes, out, workspace)
    dev = q.get_device()
    if stream is not None or dev != _current_device():
        with _place(q, stream):
            return tree_attention(q, K, V, lens, tree, sm_scale, N, block_table=block_table, softcap=softcap, slopes=slopes,
                                  out=out, workspace=workspace)
    if out is None:
        out = q.new_empty((B, Hq, T, 128))
    if workspace is None:
        need = tree_workspace_bytes(B, Hq, Hkv, T, N)
        if need:
            workspace = q.new_empty(need, dtype=torch.uint8)
    status = _lib.bpc_tree_attention(
        q.data_ptr(), *sq, K.data_ptr(), *sK, V.data_ptr(), *sV, _ptr(block_table), st, pages,
        page, lens.data_ptr(), _ptr(tree), sm, B, Hq, Hkv, T, N, 128, _SM_SCALE if sm_scale is None else sm_scale,
        softcap, _ptr(slopes), out.data_ptr(), *so, _ptr(workspace), 0 if workspace is None else workspace.numel(),
        _current_stream(dev))
    if status:
        _check(status, "bpc_tree_attention")
    return out


def _slots(n: int) -> int:
    """A window or a number of first slots, as the C entries take it: slots are below 2^30."""
    return max(-1, min(n, 1 << 30))


@functools.lru_cache(maxsize=4096)
def chunk_workspace_bytes(B: int, Hq: int, Hkv: int, T: int, N: int, window: int = 0, sinks: int = 0, D: int = 128) -> int:
    return int(_lib.bpc_chunk_workspace_bytes(B, Hq, Hkv, T, N, D, _slots(window), _slots(sinks)))


def chunk_cut(B: int, Hq: int, Hkv: int, T: int, N: int, window: int = 0, sinks: int = 0, D: int = 128):
    """(row_blocks, pieces, streamed) of chunk_attention, as attention_cut."""
    row_blocks, pieces, streamed = _i(), _i(), _i()
    _check(_lib.bpc_chunk_cut(B, Hq, Hkv, T, N, D, _slots(window), _slots(sinks), row_blocks, pieces, streamed), "bpc_chunk_cut")
    return row_blocks.value, pieces.value, bool(streamed.value)


def _paged_or_not(K, B, Hkv, Kb, Kn, N, block_table, V=None, Vs=None, weights=None):
    """(N, pages, page, table stride) of a call over a contiguous cache or pools
    of pages, whose extents (Vs: V's first three) it checks; N: by default what they
    and the weights hold."""
    most_weights = weights.shape[2] if isinstance(weights, torch.Tensor) and weights.dim() == 3 else 1 << 30
    if block_table is None:
        N = min(Kn, most_weights) if N is None else N
        if Kb != B or Kn < N:
            _extent(K, "K", (B, Hkv, ("ge", N), 128))
        if V is not None and (Vs[0] != B or Vs[1] != Hkv or Vs[2] < N):
            _extent(V, "V", (B, Hkv, ("ge", N), 128))
        pages = page = st = 0
    else:
        pages, page = Kb, Kn
        if V is not None and Vs != (pages, Hkv, page):
            _extent(V, "V", (pages, Hkv, page, 128))
        _page_rows(page)
        st, most = _block_table(block_table, B)
        most *= page
        N = min(most, most_weights) if N is None else N
        if N > most:
            raise ValueError(f"N={N}: the block_table holds {most} slots per sequence")
    if N < 1:
        raise ValueError(f"N={N} must be >= 1")
    return N, pages, page, st


def _float_rows(t: torch.Tensor, name: str, B: int, H: int, n: int, more: bool, written: bool):
    """(batch, head) strides of an fp32 [B, H, n] tensor (or wider, with `more`)
    with contiguous rows; rows that are written must not overlap."""
    fits = False
    if type(t) is torch.Tensor and t.dtype is torch.float32 and t.dim() == 3:
        (b, h, m), (x, y, one) = t.shape, t.stride()
        fits = b == B and h == H and one == 1 and (m == n or more and m > n)
    if not fits:
        _need(t, name, torch.float32, 3)
        _extent(t, name, (B, H, ("ge", n) if more else n))
        (_, _, m), (x, y, _) = t.shape, t.stride()
    if written and (y < m or x < y * H) and not t.is_contiguous():
        span = m
        for stride, extent in sorted(((x, B), (y, H))):
            if extent > 1:
                if stride < span:
                    raise ValueError(f"{name}: its rows must not overlap (strides {tuple(t.stride())})")
                span += stride * (extent - 1)
    return x if B > 1 else 0, y if H > 1 else 0


def _window(window: int, sinks: int):
    """Both, as the C entries take them."""
    if window < 0 or sinks < 0:
        raise ValueError(f"window={window} and sinks={sinks} must be >= 0")
    return _slots(window), _slots(sinks)


def chunk_attention(q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, pos: torch.Tensor, sm_scale: Optional[float] = None,
                    N: Optional[int] = None, *, count: Optional[torch.Tensor] = None,
                    block_table: Optional[torch.Tensor] = None, softcap: float = 0.0,
                    slopes: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0,
                    out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense attention of a chunk of new tokens q [B, Hq, T, 128] bf16 over the
    cache that holds them, token t < count[b] (int32 [B], default T) of sequence b
    at slot pos[b] + t (int32 [B]), where append_kv_paged stores it; returns out
    [B, Hq, T, 128] bf16.

    A token sees the slots up to its own; with `window` the last so many of them
    and the first `sinks` of the cache.  K, V are the contiguous cache [B, Hkv,
    >=N, 128], or with block_table (int32 [B, pages of a sequence]) pools of pages
    [pages, Hkv, page, 128].  N: slots that any sequence may use (default: what the
    cache or the table holds); one near the longest sequence cuts the work best.
    softcap and slopes as in prefill_attention.  lse_out [B, Hq, T] fp32, when
    given, gets the logarithm of each row's sum of exponentials.  Rows of tokens
    from count[b] on, and of a sequence whose slots are not all in [0, N), stay as
    they are (undefined where `out` is allocated here)."""
    B, Hq, Hkv, T, sq, so, Kb, Kn, sK, Vb, Vh, Vn, sV = _attn_inputs(q, K, V, slopes, out, workspace)
    N, pages, page, st = _paged_or_not(K, B, Hkv, Kb, Kn, N, block_table, V, (Vb, Vh, Vn))
    if window or sinks:
        window, sinks = _window(window, sinks)
    _indices(pos, "pos", (B,))
    if count is not None:
        _indices(count, "count", (B,))
    l_b = l_h = 0
    if lse_out is not None:
        l_b, l_h = _float_rows(lse_out, "lse_out", B, Hq, T, False, True)
    _on_gpu(q, K, V, pos, count, block_table, slopes, out, lse_out, workspace)
    dev = q.get_device()
    if stream is not None or dev != _current_device():
        with _place(q, stream):
            return chunk_attention(q, K, V, pos, sm_scale, N, count=count, block_table=block_table, softcap=softcap,
                                   slopes=slopes, window=window, sinks=sinks, out=out, lse_out=lse_out, workspace=workspace)
    if out is None:
        out = q.new_empty((B, Hq, T, 128))
    if workspace is None:
        need = chunk_workspace_bytes(B, Hq, Hkv, T, N, window, sinks)
        if need:
            workspace = q.new_empty(need, dtype=torch.uint8)
    status = _lib.bpc_chunk_attention(
        q.data_ptr(), *sq, K.data_ptr(), *sK, V.data_ptr(), *sV, _ptr(block_table), st, pages, page, pos.data_ptr(),
        _ptr(count), B, Hq, Hkv, T, N, 128, _SM_SCALE if sm_scale is None else sm_scale, softcap, _ptr(slopes),
        window, sinks, out.data_ptr(), *so, _ptr(lse_out), l_b, l_h, _ptr(workspace),
        0 if workspace is None else workspace.numel(), _current_stream(dev))
    if status:
        _check(status, "bpc_chunk_attention")
    return out


def key_weights(q: torch.Tensor, K: torch.Tensor, lse: torch.Tensor, weights: torch.Tensor, pos: torch.Tensor,
                sm_scale: Optional[float] = None, N: Optional[int] = None, *, count: Optional[torch.Tensor] = None,
                block_table: Optional[torch.Tensor] = None, softcap: float = 0.0,
                slopes: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0, decay: float = 1.0,
                stream=None) -> torch.Tensor:
    """Adds to `weights` [B, Hkv, >=N] fp32 the attention weight that each cached
    slot gathers from the tokens of a chunk_attention call: the sum over its
    tokens and the query heads of a KV head of exp(score - lse), lse [B, Hq, T]
    fp32 being that call's lse_out; the other arguments are that call's.  What was
    there is multiplied by `decay` first (0: not even read).  Slots from pos[b] +
    count[b] on, and sequences whose slots are not all in [0, N), stay as they are
    (N: by default what the cache or the table, and the weights, hold).  Returns
    weights."""
    B, Hq, T, q_b, q_h, q_t = _rows(q, "q")
    Kb, Hkv, Kn, (K_b, K_h, K_n) = _cache(K, "K")
    if Hq % Hkv:
        raise ValueError(f"Hq={Hq} must be a multiple of Hkv={Hkv}")
    if slopes is not None:
        _need(slopes, "slopes", torch.float32, 1)
        _extent(slopes, "slopes", (Hq,))
    N, pages, page, st = _paged_or_not(K, B, Hkv, Kb, Kn, N, block_table, weights=weights)
    if window or sinks:
        window, sinks = _window(window, sinks)
    _indices(pos, "pos", (B,))
    if count is not None:
        _indices(count, "count", (B,))
    l_b, l_h = _float_rows(lse, "lse", B, Hq, T, False, False)
    w_b, w_h = _float_rows(weights, "weights", B, Hkv, N, True, True)
    _on_gpu(q, K, lse, weights, pos, count, block_table, slopes)
    dev = q.get_device()
    if stream is not None or dev != _current_device():
        with _place(q, stream):
            return key_weights(q, K, lse, weights, pos, sm_scale, N, count=count, block_table=block_table, softcap=softcap,
                               slopes=slopes, window=window, sinks=sinks, decay=decay)
    status = _lib.bpc_key_weights(
        q.data_ptr(), q_b, q_h, q_t, K.data_ptr(), K_b, K_h, K_n, lse.data_ptr(), l_b, l_h, weights.data_ptr(), w_b, w_h,
        _ptr(block_table), st, pages, page, pos.data_ptr(), _ptr(count), B, Hq, Hkv, T, N, 128,
        _SM_SCALE if sm_scale is None else sm_scale, softcap, _ptr(slopes), window, sinks, decay, _current_stream(dev))
    if status:
        _check(status, "bpc_key_weights")
    return weights


@functools.lru_cache(maxsize=4096)
def evict_workspace_bytes(B: int, Hkv: int, N: int, keep: int) -> int:
    return int(_lib.bpc_evict_workspace_bytes(B, Hkv, N, keep))


def evict_kv(K: torch.Tensor, V: torch.Tensor, weights: torch.Tensor, lens: torch.Tensor, keep: int, K_out: torch.Tensor,
             V_out: torch.Tensor, *, sinks: int = 0, recent: int = 0, N: Optional[int] = None,
             block_table: Optional[torch.Tensor] = None, table_out: Optional[torch.Tensor] = None,
             codes: Optional[torch.Tensor] = None, codes_out: Optional[torch.Tensor] = None,
             weights_out: Optional[torch.Tensor] = None, kept_out: Optional[torch.Tensor] = None,
             workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Cuts a cache to `keep` slots of each KV head: the first `sinks`, the last
    `recent`, and of the others those of the largest weights [B, Hkv, >=N] fp32, the
    lower slot first among equals (all lens[b] of them where these are not more;
    lens int32 [B]).  Their rows of K and V go, in order, to the first slots of
    K_out and V_out, those of codes to codes_out, their weights to weights_out
    (zeros behind); returns their old slots [B, Hkv, keep] int32, -1 behind.

    K, V are the contiguous cache [B, Hkv, >=N, 128], or with block_table pools of
    pages; K_out, V_out [B, Hkv, >=keep, 128], or with table_out (int32 [B, pages of
    a sequence]) pools of pages, which may be K and V themselves as long as no page
    that is written is read or written twice.  codes as build_hash gives them.  N:
    slots that any sequence may use (default: what the cache or the table, and the
    weights, hold); one whose lens[b] is not in [0, N] is skipped (its slots in the
    result are undefined where that is allocated here).  The sequences' new lengths
    are lens.clamp(max=keep); windows and slopes of chunk_attention and key_weights
    count the slots that are left from then on."""
    Kb, Hkv, Kn, (K_b, K_h, K_n) = _cache(K, "K")
    Vb, Vh, Vn, (V_b, V_h, V_n) = _cache(V, "V")
    if type(lens) is not torch.Tensor or lens.dtype is not torch.int32 or lens.dim() != 1 or not lens.is_contiguous():
        _need(lens, "lens", torch.int32, 1)
    B = lens.shape[0]
    if Vh != Hkv:
        _extent(V, "V", (Vb, Hkv, Vn, 128))
    N, pages, page, st = _paged_or_not(K, B, Hkv, Kb, Kn, N, block_table, V, (Vb, Vh, Vn), weights)
    if not 1 <= keep <= N:
        raise ValueError(f"keep={keep} must be in [1, N={N}]")
    if sinks < 0 or recent < 0 or sinks + recent > keep:
        raise ValueError(f"sinks={sinks} and recent={recent} must be >= 0, together at most keep={keep}")
    Ob, Oh, On, (Ko_b, Ko_h, Ko_n) = _written(K_out, "K_out")
    Pb, Ph, Pn, (Vo_b, Vo_h, Vo_n) = _written(V_out, "V_out")
    out_pages = out_page = sto = 0
    if table_out is None:
        if Ob != B or Oh != Hkv or On < keep:
            _extent(K_out, "K_out", (B, Hkv, ("ge", keep), 128))
        if Pb != B or Ph != Hkv or Pn < keep:
            _extent(V_out, "V_out", (B, Hkv, ("ge", keep), 128))
    else:
        if Oh != Hkv:
            _extent(K_out, "K_out", (Ob, Hkv, On, 128))
        if Pb != Ob or Ph != Hkv or Pn != On:
            _extent(V_out, "V_out", (Ob, Hkv, On, 128))
        out_pages, out_page = Ob, On
        _page_rows(out_page)
        sto, most = _block_table(table_out, B)
        if most * out_page < keep:
            raise ValueError(f"table_out holds {most * out_page} slots per sequence, keep={keep}")
    w_b, w_h = _float_rows(weights, "weights", B, Hkv, N, True, False)
    wo_b = wo_h = cap = 0
    if weights_out is not None:
        wo_b, wo_h = _float_rows(weights_out, "weights_out", B, Hkv, keep, True, True)
        cap = weights_out.shape[2]
    if (codes is None) != (codes_out is None):
        raise ValueError("codes and codes_out are given together or not at all")
    W, sC, sCo = 0, (0, 0), (0, 0)
    if codes is not None:
        _u32_codes(codes)
        _u32_codes(codes_out, "codes_out")
        W = codes.shape[3]
        if W not in (1, 2, 4):
            raise ValueError(f"codes of {W} words: the code length must be 32, 64 or 128")
        _extent(codes, "codes", (B, Hkv, ("ge", N), W))
        _extent(codes_out, "codes_out", (B, Hkv, ("ge", keep), W))
        sC, sCo = (codes.stride(0), codes.stride(1)), (codes_out.stride(0), codes_out.stride(1))
    if kept_out is not None:
        _exact_out(kept_out, "kept_out", torch.int32, (B, Hkv, keep))
    if workspace is not None and (workspace.dtype != torch.uint8 or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 tensor")
    _on_gpu(K, V, weights, lens, K_out, V_out, block_table, table_out, codes, codes_out, weights_out, kept_out, workspace)
    dev = K.get_device()
    if stream is not None or dev != _current_device():
        with _place(K, stream):
            return evict_kv(K, V, weights, lens, keep, K_out, V_out, sinks=sinks, recent=recent, N=N, block_table=block_table,
                            table_out=table_out, codes=codes, codes_out=codes_out, weights_out=weights_out,
                            kept_out=kept_out, workspace=workspace)
    if kept_out is None:
        kept_out = lens.new_empty((B, Hkv, keep))
    if workspace is None:
        need = evict_workspace_bytes(B, Hkv, N, keep)
        if need:
            workspace = lens.new_empty(need, dtype=torch.uint8)
    status = _lib.bpc_evict_kv(
        K.data_ptr(), K_b, K_h, K_n, V.data_ptr(), V_b, V_h, V_n, _ptr(block_table), st, pages, page, weights.data_ptr(), w_b, w_h,
        lens.data_ptr(), B, Hkv, N, 128, keep, sinks, recent, K_out.data_ptr(), Ko_b, Ko_h, Ko_n, V_out.data_ptr(), Vo_b, Vo_h, Vo_n,
        _ptr(table_out), sto, out_pages, out_page, _ptr(codes), *sC, _ptr(codes_out), *sCo, W, _ptr(weights_out), wo_b, wo_h, cap,
        kept_out.data_ptr(), _ptr(workspace), 0 if workspace is None else workspace.numel(), _current_stream(dev))
    if status:
        _check(status, "bpc_evict_kv")
    return kept_out
