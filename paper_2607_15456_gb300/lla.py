"""Thin Python binding of liblla (include/lla.h): argument marshalling only.

Every function here has the name of the C entry point it calls and does nothing but turn
torch tensors into device pointers, fill the ABI structs and raise ``LLAError`` on a non-zero
status.  The calls of a decode step and of a prompt are marshalled by ``_lla_native``
(csrc/lla_binding.cpp) when their arguments are the ordinary ones, contiguous CUDA tensors and ints;
it answers None to anything else, which the Python marshalling below takes or refuses, as it does
every call where that module is missing.  All computation happens in the CUDA kernels of liblla.so;
there is no fallback: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import importlib
import math
import os
import warnings
from dataclasses import dataclass
from typing import Optional

import torch

from .build import LIB, NATIVE, binding_abi

LLA_BLOCK_TOKENS = 64
LLA_MAX_BATCH = 1024
LLA_BF16, LLA_F32 = 0, 1
LLA_ROPE_HALF, LLA_ROPE_ADJACENT = 0, 1
LLA_DEVERR_BLOCK_ID = 0x1
LLA_DEVERR_CONTEXT = 0x2
LLA_DEVERR_EMPTY_PASS2 = 0x4
LLA_DEVERR_TIMEOUT = 0x8
LLA_DEVERR_SLOT = 0x10
LLA_DEVERR_SEQUENCE = 0x20
LLA_DEVERR_PAGES = 0x40
LLA_MAX_BEAMS = 32

_STATUS = {0: "LLA_OK", 1: "LLA_ERR_INVALID_ARG", 2: "LLA_ERR_UNSUPPORTED", 3: "LLA_ERR_CUDA",
           4: "LLA_ERR_TIMEOUT", 5: "LLA_ERR_DEVICE_CHECK", 6: "LLA_ERR_WORKSPACE"}


class LLAError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} returned {_STATUS.get(status, status)}")


class lla_geometry(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("r_k", ctypes.c_int32), ("r_v", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("storage", ctypes.c_int32), ("scale", ctypes.c_float)]


class lla_codec(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("w_down_k", "w_down_v", "w_up_k", "w_up_v", "mu_k", "mu_v")]


class lla_rope(ctypes.Structure):
    _fields_ = [("base", ctypes.c_double), ("pairing", ctypes.c_int32)]


class lla_cache(ctypes.Structure):
    _fields_ = [("pool", ctypes.c_void_p), ("num_blocks", ctypes.c_int64),
                ("block_table", ctypes.c_void_p), ("max_blocks_per_seq", ctypes.c_int32)]


class lla_pages(ctypes.Structure):
    _fields_ = [("ref_count", ctypes.c_void_p), ("num_blocks", ctypes.c_int64),
                ("block_table", ctypes.c_void_p), ("max_blocks_per_seq", ctypes.c_int32),
                ("context_lens", ctypes.c_void_p), ("S", ctypes.c_int32)]


class lla_pool(ctypes.Structure):
    _fields_ = [("base", ctypes.c_void_p), ("pages", ctypes.c_int32),
                ("k_row_bytes", ctypes.c_int32), ("v_row_bytes", ctypes.c_int32)]


# lla_capture_fn, lla_query_fn and lla_step_fn of include/lla.h
CAPTURE_FN = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p),
                              ctypes.POINTER(ctypes.c_void_p), ctypes.c_void_p, ctypes.c_void_p)
QUERY_FN = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                            ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p),
                            ctypes.c_void_p, ctypes.c_void_p)

STEP_FN = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(lla_pages), ctypes.c_void_p,
                           ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p),
                           ctypes.POINTER(ctypes.c_int64), ctypes.c_void_p, ctypes.c_void_p)

_lib = None
_native_module = None


class _Absent:
    """In the place of _lla_native where it cannot be loaded: leaves every call to Python."""

    def __getattr__(self, name):
        return lambda *args: None


def _native():
    """The native marshalling module, loaded with the library it calls."""
    global _native_module
    if _native_module is None:
        library()
        try:
            with open(NATIVE + ".abi") as f:
                abi = f.read()
            if abi != binding_abi():  # its tensors would be misread
                raise ImportError(f"built for {abi}, not for {binding_abi()}")
            module = importlib.import_module("._lla_native", __package__)
        except (ImportError, OSError) as e:
            warnings.warn(f"calls are marshalled in Python (several us each): _lla_native.so is not loaded: {e}")
            module = _Absent()
        _native_module = module
    return _native_module


def library() -> ctypes.CDLL:
    """Loads liblla.so from the package directory (built by ``__graft_entry__.build()``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB):
            raise RuntimeError(f"liblla.so not found at {LIB}: build it first "
                               "(python -c 'import __graft_entry__ as g; g.build()')")
        lib = ctypes.CDLL(LIB)
        P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        sig = {
            "lla_status_string": (ctypes.c_char_p, [I32]),
            "lla_version": (I32, []),
            "lla_cache_block_bytes": (I32, [P, P]),
            "lla_encode": (I32, [P, P, P, P, P, I32, P, I32, P]),
            "lla_encode_layers": (I32, [P, I32, P, P, P, P, I32, P, I32, P]),
            "lla_decode_workspace_size": (I32, [P, I32, P]),
            "lla_decode_workspace_init": (I32, [P, SZ, P]),
            "lla_decode_attn": (I32, [P, P, P, P, I32, I32, I32, P, P, P, I32, P, P, SZ, P]),
            "lla_decode_attn_noalloc": (I32, [P, P, P, P, I32, I32, I32, P, P, P, I32, P, P]),
            "lla_decode_attn_rope": (I32, [P, P, P, P, P, I32, I32, I32, P, P, P, I32, P, P, SZ,
                                           P]),
            "lla_decode_loops_workspace_size": (I32, [P, I32, P]),
            "lla_decode_attn_loops": (I32, [P, P, P, P, I32, I32, P, P, P, I32, P, P, SZ, P]),
            "lla_prefill_attn": (I32, [P, P, P, P, I32, I32, I32, P, I32, P, P]),
            "lla_prefill_rope_workspace_size": (I32, [P, I32, I32, P]),
            "lla_prefill_attn_rope": (I32, [P, P, P, P, P, I32, I32, I32, P, I32, P, P, SZ, P]),
            "lla_dense_store": (I32, [P, P, P, P, I32, P, I32, P]),
            "lla_dense_decode_attn": (I32, [P, P, P, I32, I32, P, P, P, I32, P, P, SZ, P]),
            "lla_cache_2d_block_bytes": (I32, [P, P]),
            "lla_encode_2d": (I32, [P, P, P, P, P, I32, P, I32, P]),
            "lla_decode_2d_workspace_size": (I32, [P, I32, P]),
            "lla_decode_attn_2d": (I32, [P, P, P, P, I32, I32, I32, P, P, P, I32, P, P, SZ, P]),
            "lla_rope_plane_bytes": (I32, [I32, P]),
            "lla_encode_rope_keys": (I32, [I32, P, P, I64, P, I32, P, P, I32, P]),
            "lla_decode_decoupled_workspace_size": (I32, [P, I32, I32, P]),
            "lla_decode_attn_decoupled": (I32, [P, P, P, P, I32, P, P, I32, I32, I32, P, P, P, P, P, I32,
                                                P, P, SZ, P]),
            "lla_get_device_error": (I32, [P, P]),
            "lla_clear_device_error": (I32, [P]),
            "lla_prefill_two_pass": (I32, [P, I32, P, P, I32, P, I32, P, I32, I32, I32, P, CAPTURE_FN,
                                           QUERY_FN, P, P, SZ, P]),
            "lla_cache_pool": (I32, [P, P, P]),
            "lla_cache_2d_pool": (I32, [P, P, P]),
            "lla_rope_pool": (I32, [I32, P, P]),
            "lla_pages_fork": (I32, [P, P, P, P]),
            "lla_pages_extend_workspace_size": (I32, [I32, P]),
            "lla_pages_extend": (I32, [P, P, I32, P, I32, P, P, P, P, P, SZ, P]),
            "lla_pages_free": (I32, [P, P, I32, P]),
            "lla_pages_compact_workspace_size": (I32, [I64, P]),
            "lla_pages_compact": (I32, [P, P, I32, P, P, P, SZ, P]),
            "lla_beam_select_workspace_size": (I32, [I32, I32, I32, I32, I32, P]),
            "lla_beam_select": (I32, [I32, I32, I32, I32, P, I64, I32, P, P, P, I32, ctypes.c_float, P, P, P,
                                      P, P, P, SZ, P]),
            "lla_beam_search_workspace_size": (I32, [I32, I32, I32, I32, P]),
            "lla_beam_search": (I32, [P, P, P, I32, I32, I32, I32, I32, I32, I32, ctypes.c_float, P, P, P, P,
                                      P, STEP_FN, P, P, SZ, P]),
            "lla_set_wait_limit_ns": (I32, [ctypes.c_uint64]),
            "lla_get_wait_limit_ns": (ctypes.c_uint64, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _check(fn: str, status: int):
    if status != 0:
        raise LLAError(fn, status)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensors passed to liblla must be contiguous")
    if not t.is_cuda:
        # every buffer of the ABI is a device buffer: a host address would fault the kernel
        raise ValueError("tensors passed to liblla must be CUDA tensors")
    return t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return LLA_BF16
    if t.dtype == torch.float32:
        return LLA_F32
    raise ValueError(f"unsupported dtype {t.dtype}")


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _handle(stream):
    """A stream for _lla_native: None (the current stream, looked up there) or its handle."""
    return None if stream is None else _stream(stream)


def _done(fn: str, status) -> bool:
    """Whether _lla_native took the call (a status; non-zero raises) or left it (None)."""
    if status is None:
        return False
    if status != 0:
        raise LLAError(fn, status)
    return True


@dataclass
class Geometry:
    T: int
    H: int
    d: int
    r_k: int
    r_v: int
    storage: str = "bf16"
    scale: Optional[float] = None

    def c(self) -> lla_geometry:
        scale = self.scale if self.scale is not None else 1.0 / math.sqrt(self.d)
        return lla_geometry(self.T, self.H, self.d, self.r_k, self.r_v, LLA_BLOCK_TOKENS,
                            LLA_BF16 if self.storage == "bf16" else LLA_F32, scale)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.storage == "bf16" else torch.float32


@dataclass
class Codec:
    """Codec of one layer: w_down_* [H][T*d][r], w_up_* [H][T][d][r], mu_* [H][T*d] fp32."""
    w_down_k: torch.Tensor
    w_down_v: torch.Tensor
    w_up_k: torch.Tensor
    w_up_v: torch.Tensor
    mu_k: Optional[torch.Tensor] = None
    mu_v: Optional[torch.Tensor] = None

    def c(self) -> lla_codec:
        return lla_codec(*(_ptr(t) for t in (self.w_down_k, self.w_down_v, self.w_up_k,
                                             self.w_up_v, self.mu_k, self.mu_v)))


@dataclass
class Cache:
    """Paged cache of one layer: pool (uint8 or any dtype, 16-byte aligned), block table
    [B][max_blocks_per_seq] int32."""
    pool: torch.Tensor
    num_blocks: int
    block_table: Optional[torch.Tensor]
    max_blocks_per_seq: int

    def c(self) -> lla_cache:
        return lla_cache(_ptr(self.pool), self.num_blocks, _ptr(self.block_table),
                         self.max_blocks_per_seq)


def lla_status_string(status: int) -> str:
    return library().lla_status_string(status).decode()


def lla_version() -> int:
    return library().lla_version()


def lla_cache_block_bytes(geom: Geometry) -> int:
    out = ctypes.c_size_t(0)
    g = geom.c()
    _check("lla_cache_block_bytes",
           library().lla_cache_block_bytes(ctypes.byref(g), ctypes.byref(out)))
    return out.value


def lla_encode(geom: Geometry, codec: Codec, cache: Cache, x_k: torch.Tensor, x_v: torch.Tensor,
               slot_mapping: torch.Tensor, stream=None) -> None:
    """x_k, x_v [T][N][H][d] (bf16 or fp32); slot_mapping [N] int64."""
    if _done("lla_encode", _native().encode(
            geom, codec, cache, x_k, x_v, slot_mapping, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    N = x_k.shape[1] if x_k.dim() == 4 else 0
    _check("lla_encode", library().lla_encode(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(x_k), _ptr(x_v),
        _dtype_code(x_k), _ptr(slot_mapping), N, _stream(stream)))


def lla_encode_layers(geom: Geometry, codecs, caches, x_k, x_v, slot_mapping: torch.Tensor,
                      stream=None) -> None:
    """The same encode in several layers at once: codecs, caches, x_k, x_v are per-layer lists
    (x_k[l], x_v[l] [T][N][H][d]); slot_mapping [N] int64 is shared."""
    if _done("lla_encode_layers", _native().encode_layers(
            geom, codecs, caches, x_k, x_v, slot_mapping, _handle(stream))):
        return
    L = len(codecs)
    if not (len(caches) == len(x_k) == len(x_v) == L):
        raise ValueError("one codec, cache and input pair per layer")
    g = geom.c()
    cds = (lla_codec * max(L, 1))(*[c.c() for c in codecs])
    chs = (lla_cache * max(L, 1))(*[c.c() for c in caches])
    xk = (ctypes.c_void_p * max(L, 1))(*[_ptr(t) for t in x_k])
    xv = (ctypes.c_void_p * max(L, 1))(*[_ptr(t) for t in x_v])
    N = x_k[0].shape[1] if L and x_k[0].dim() == 4 else 0
    _check("lla_encode_layers", library().lla_encode_layers(
        ctypes.byref(g), L, cds, chs, xk, xv, _dtype_code(x_k[0]) if L else 0, _ptr(slot_mapping), N,
        _stream(stream)))


def lla_decode_workspace_size(geom: Geometry, B: int) -> int:
    out = ctypes.c_size_t(0)
    g = geom.c()
    _check("lla_decode_workspace_size",
           library().lla_decode_workspace_size(ctypes.byref(g), B, ctypes.byref(out)))
    return out.value


def lla_decode_workspace_init(workspace: torch.Tensor, stream=None) -> None:
    nbytes = workspace.numel() * workspace.element_size()
    _check("lla_decode_workspace_init",
           library().lla_decode_workspace_init(_ptr(workspace), nbytes, _stream(stream)))


def lla_decode_attn(geom: Geometry, codec: Codec, cache: Cache, context_lens: torch.Tensor,
                    max_ctx: int, loop: int, q: torch.Tensor, cur_k: Optional[torch.Tensor],
                    cur_v: Optional[torch.Tensor], out: torch.Tensor, workspace: torch.Tensor,
                    stream=None) -> None:
    """q, cur_k, cur_v, out [B][H][d]; cur_k = cur_v = None selects pass 2."""
    if _done("lla_decode_attn", _native().decode_attn(
            geom, codec, cache, context_lens, max_ctx, loop, q, cur_k, cur_v, out, workspace, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    B = q.shape[0]
    _check("lla_decode_attn", library().lla_decode_attn(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(context_lens), B, max_ctx,
        loop, _ptr(q), _ptr(cur_k), _ptr(cur_v), _dtype_code(q), _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def lla_decode_attn_rope(geom: Geometry, codec: Codec, cache: Cache, rope_base: float,
                         rope_pairing: int, context_lens: torch.Tensor, max_ctx: int, loop: int,
                         q: torch.Tensor, cur_k: Optional[torch.Tensor],
                         cur_v: Optional[torch.Tensor], out: torch.Tensor,
                         workspace: torch.Tensor, stream=None) -> None:
    """lla_decode_attn with RoPE after reconstruction; q and cur_k pre-RoPE.  rope_pairing:
    LLA_ROPE_HALF (pairs (j, j + d/2)) or LLA_ROPE_ADJACENT (pairs (2j, 2j + 1))."""
    if _done("lla_decode_attn_rope", _native().decode_attn_rope(
            geom, codec, cache, rope_base, rope_pairing, context_lens, max_ctx, loop, q, cur_k, cur_v, out,
            workspace, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    rp = lla_rope(float(rope_base), int(rope_pairing))
    _check("lla_decode_attn_rope", library().lla_decode_attn_rope(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), ctypes.byref(rp),
        _ptr(context_lens), q.shape[0], max_ctx, loop, _ptr(q), _ptr(cur_k), _ptr(cur_v),
        _dtype_code(q), _ptr(out), _ptr(workspace), workspace.numel() * workspace.element_size(),
        _stream(stream)))


def lla_decode_loops_workspace_size(geom: Geometry, B: int) -> int:
    g = geom.c()
    out = ctypes.c_size_t()
    _check("lla_decode_loops_workspace_size",
           library().lla_decode_loops_workspace_size(ctypes.byref(g), B, ctypes.byref(out)))
    return out.value


def lla_decode_attn_loops(geom: Geometry, codec: Codec, cache: Cache, context_lens: torch.Tensor,
                          max_ctx: int, q: torch.Tensor, cur_k: Optional[torch.Tensor],
                          cur_v: Optional[torch.Tensor], out: torch.Tensor,
                          workspace: torch.Tensor, stream=None) -> None:
    """All T loops' decode calls in one pass over the latents: q, cur_k, cur_v, out [T][B][H][d]."""
    if _done("lla_decode_attn_loops", _native().decode_attn_loops(
            geom, codec, cache, context_lens, max_ctx, q, cur_k, cur_v, out, workspace, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    _check("lla_decode_attn_loops", library().lla_decode_attn_loops(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(context_lens), q.shape[1],
        max_ctx, _ptr(q), _ptr(cur_k), _ptr(cur_v), _dtype_code(q), _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def lla_decode_attn_noalloc(geom: Geometry, codec: Codec, cache: Cache,
                            context_lens: torch.Tensor, max_ctx: int, loop: int,
                            q: torch.Tensor, cur_k: Optional[torch.Tensor],
                            cur_v: Optional[torch.Tensor], out: torch.Tensor,
                            stream=None) -> None:
    """lla_decode_attn with the library's own 1 MiB device scratch instead of a caller
    workspace, for callers that cannot allocate device memory (see include/lla.h)."""
    g, cd, ch = geom.c(), codec.c(), cache.c()
    _check("lla_decode_attn_noalloc", library().lla_decode_attn_noalloc(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(context_lens), q.shape[0],
        max_ctx, loop, _ptr(q), _ptr(cur_k), _ptr(cur_v), _dtype_code(q), _ptr(out),
        _stream(stream)))


def lla_prefill_attn(geom: Geometry, codec: Codec, cache: Cache, cu_seqlens: torch.Tensor,
                     max_len: int, loop: int, q: torch.Tensor, out: torch.Tensor,
                     stream=None) -> None:
    """q, out [Ntok][H][d]; cu_seqlens [B+1] int32."""
    if _done("lla_prefill_attn", _native().prefill_attn(
            geom, codec, cache, cu_seqlens, max_len, loop, q, out, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    B = cu_seqlens.shape[0] - 1
    _check("lla_prefill_attn", library().lla_prefill_attn(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(cu_seqlens), B, max_len, loop,
        _ptr(q), _dtype_code(q), _ptr(out), _stream(stream)))


def lla_prefill_rope_workspace_size(geom: Geometry, B: int, max_len: int) -> int:
    g = geom.c()
    out = ctypes.c_size_t()
    _check("lla_prefill_rope_workspace_size",
           library().lla_prefill_rope_workspace_size(ctypes.byref(g), B, max_len, ctypes.byref(out)))
    return out.value


def lla_prefill_attn_rope(geom: Geometry, codec: Codec, cache: Cache, rope_base: float,
                          rope_pairing: int, cu_seqlens: torch.Tensor, max_len: int, loop: int,
                          q: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                          stream=None) -> None:
    """lla_prefill_attn with RoPE after reconstruction; q pre-RoPE [Ntok][H][d]."""
    if _done("lla_prefill_attn_rope", _native().prefill_attn_rope(
            geom, codec, cache, rope_base, rope_pairing, cu_seqlens, max_len, loop, q, out, workspace, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    rp = lla_rope(float(rope_base), int(rope_pairing))
    B = cu_seqlens.shape[0] - 1
    _check("lla_prefill_attn_rope", library().lla_prefill_attn_rope(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), ctypes.byref(rp), _ptr(cu_seqlens), B,
        max_len, loop, _ptr(q), _dtype_code(q), _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def lla_prefill_two_pass(geom: Geometry, codecs, caches, slot_mapping: torch.Tensor,
                         cu_seqlens: torch.Tensor, max_len: int, capture, query,
                         x_dtype=torch.bfloat16, io_dtype=torch.bfloat16, rope_base=None,
                         rope_pairing: int = LLA_ROPE_HALF, workspace: Optional[torch.Tensor] = None,
                         stream=None) -> None:
    """Two-pass prefill of len(cu_seqlens) - 1 prompts through len(codecs) layers, streamed layer
    by layer.  capture(layer) returns layer's pass-1 (x_k, x_v) [T][N][H][d]; query(layer, loop)
    returns (q, out) [N][H][d].  Both are called from inside the C call, in its order; the
    tensors they return are kept alive until it returns (stream order covers the rest).
    rope_base None: positions-free content path; else RoPE after reconstruction (workspace of
    lla_prefill_rope_workspace_size bytes)."""
    D = len(codecs)
    if len(caches) != D:
        raise ValueError("one cache per codec")
    cds = (lla_codec * max(D, 1))(*[c.c() for c in codecs])
    chs = (lla_cache * max(D, 1))(*[c.c() for c in caches])
    g = geom.c()
    keep, errors = [], []

    def _capture(layer, pk, pv, _stream_, _user):
        try:
            xk, xv = capture(layer)
            keep.append((xk, xv))
            pk[0], pv[0] = _ptr(xk), _ptr(xv)
            return 0
        except Exception as e:  # reported after the C call returns
            errors.append(e)
            return 1

    def _query(layer, loop, pq, po, _stream_, _user):
        try:
            q, out = query(layer, loop)
            keep.append((q, out))
            pq[0], po[0] = _ptr(q), _ptr(out)
            return 0
        except Exception as e:
            errors.append(e)
            return 1

    cb_c, cb_q = CAPTURE_FN(_capture), QUERY_FN(_query)
    rp = None if rope_base is None else lla_rope(float(rope_base), int(rope_pairing))
    xd = LLA_BF16 if x_dtype == torch.bfloat16 else LLA_F32
    iod = LLA_BF16 if io_dtype == torch.bfloat16 else LLA_F32
    B = cu_seqlens.shape[0] - 1
    st = library().lla_prefill_two_pass(
        ctypes.byref(g), D, cds, chs, xd, _ptr(slot_mapping), slot_mapping.numel(), _ptr(cu_seqlens),
        B, max_len, iod, None if rp is None else ctypes.byref(rp), cb_c, cb_q, None, _ptr(workspace),
        0 if workspace is None else workspace.numel() * workspace.element_size(), _stream(stream))
    if errors:
        raise errors[0]
    _check("lla_prefill_two_pass", st)


def lla_cache_2d_block_bytes(geom: Geometry) -> int:
    """Bytes of one LLA-2D cache block (one page of 64 tokens for all heads)."""
    out = ctypes.c_size_t(0)
    g = geom.c()
    _check("lla_cache_2d_block_bytes",
           library().lla_cache_2d_block_bytes(ctypes.byref(g), ctypes.byref(out)))
    return out.value


def lla_encode_2d(geom: Geometry, codec: Codec, cache: Cache, x_k: torch.Tensor,
                  x_v: torch.Tensor, slot_mapping: torch.Tensor, stream=None) -> None:
    """LLA-2D encode.  x_k, x_v [T][N][H][d]; codec w_down_* [T*H*d][r], mu_* [T*H*d];
    cache with one page per block."""
    if _done("lla_encode_2d", _native().encode_2d(
            geom, codec, cache, x_k, x_v, slot_mapping, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    N = x_k.shape[1] if x_k.dim() == 4 else 0
    _check("lla_encode_2d", library().lla_encode_2d(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(x_k), _ptr(x_v),
        _dtype_code(x_k), _ptr(slot_mapping), N, _stream(stream)))


def lla_decode_2d_workspace_size(geom: Geometry, B: int) -> int:
    out = ctypes.c_size_t(0)
    g = geom.c()
    _check("lla_decode_2d_workspace_size",
           library().lla_decode_2d_workspace_size(ctypes.byref(g), B, ctypes.byref(out)))
    return out.value


def lla_decode_attn_2d(geom: Geometry, codec: Codec, cache: Cache, context_lens: torch.Tensor,
                       max_ctx: int, loop: int, q: torch.Tensor, cur_k: Optional[torch.Tensor],
                       cur_v: Optional[torch.Tensor], out: torch.Tensor, workspace: torch.Tensor,
                       stream=None) -> None:
    """LLA-2D decode call; codec w_up_* [T][H][d][r]; q, cur_k, cur_v, out [B][H][d]."""
    if _done("lla_decode_attn_2d", _native().decode_attn_2d(
            geom, codec, cache, context_lens, max_ctx, loop, q, cur_k, cur_v, out, workspace, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    _check("lla_decode_attn_2d", library().lla_decode_attn_2d(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(context_lens), q.shape[0],
        max_ctx, loop, _ptr(q), _ptr(cur_k), _ptr(cur_v), _dtype_code(q), _ptr(out),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def lla_rope_plane_bytes(d_rope: int) -> int:
    out = ctypes.c_size_t(0)
    _check("lla_rope_plane_bytes", library().lla_rope_plane_bytes(d_rope, ctypes.byref(out)))
    return out.value


def lla_encode_rope_keys(d_rope: int, rope_base: float, rope_pairing: int, rope_pool: torch.Tensor,
                         num_blocks: int, k_rope: torch.Tensor, positions: torch.Tensor,
                         slot_mapping: torch.Tensor, stream=None) -> None:
    """Rotary keys k_rope [N][d_rope], turned at positions [N] int32, into the rotary planes."""
    rp = lla_rope(float(rope_base), int(rope_pairing))
    N = k_rope.shape[0] if k_rope.dim() == 2 else 0
    _check("lla_encode_rope_keys", library().lla_encode_rope_keys(
        d_rope, ctypes.byref(rp), _ptr(rope_pool), num_blocks, _ptr(k_rope), _dtype_code(k_rope),
        _ptr(positions), _ptr(slot_mapping), N, _stream(stream)))


def lla_decode_decoupled_workspace_size(geom: Geometry, d_rope: int, B: int) -> int:
    out = ctypes.c_size_t(0)
    g = geom.c()
    _check("lla_decode_decoupled_workspace_size", library().lla_decode_decoupled_workspace_size(
        ctypes.byref(g), d_rope, B, ctypes.byref(out)))
    return out.value


def lla_decode_attn_decoupled(geom: Geometry, codec: Codec, cache: Cache, rope_pool: torch.Tensor,
                              d_rope: int, rope_base: float, rope_pairing: int,
                              context_lens: torch.Tensor, max_ctx: int, loop: int, q: torch.Tensor,
                              q_rope: torch.Tensor, cur_k: Optional[torch.Tensor],
                              cur_v: Optional[torch.Tensor], cur_k_rope: Optional[torch.Tensor],
                              out: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """Per-head LLA decode with the decoupled rotary branch; q, cur_k, cur_v, out [B][H][d],
    q_rope [B][H][d_rope], cur_k_rope [B][d_rope] (pass 1) or None."""
    if _done("lla_decode_attn_decoupled", _native().decode_attn_decoupled(
            geom, codec, cache, rope_pool, d_rope, rope_base, rope_pairing, context_lens, max_ctx, loop, q, q_rope,
            cur_k, cur_v, cur_k_rope, out, workspace, _handle(stream))):
        return
    g, cd, ch = geom.c(), codec.c(), cache.c()
    rp = lla_rope(float(rope_base), int(rope_pairing))
    _check("lla_decode_attn_decoupled", library().lla_decode_attn_decoupled(
        ctypes.byref(g), ctypes.byref(cd), ctypes.byref(ch), _ptr(rope_pool), d_rope, ctypes.byref(rp),
        _ptr(context_lens), q.shape[0], max_ctx, loop, _ptr(q), _ptr(q_rope), _ptr(cur_k), _ptr(cur_v),
        _ptr(cur_k_rope), _dtype_code(q), _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def lla_dense_store(geom: Geometry, cache: Cache, k: torch.Tensor, v: torch.Tensor,
                    slot_mapping: torch.Tensor, stream=None) -> None:
    """k, v [N][H][d]: plain loop-t keys and values for the uncompressed comparator."""
    g, ch = geom.c(), cache.c()
    _check("lla_dense_store", library().lla_dense_store(
        ctypes.byref(g), ctypes.byref(ch), _ptr(k), _ptr(v), _dtype_code(k), _ptr(slot_mapping),
        k.shape[0], _stream(stream)))


def lla_dense_decode_attn(geom: Geometry, cache: Cache, context_lens: torch.Tensor, max_ctx: int,
                          q: torch.Tensor, cur_k: Optional[torch.Tensor],
                          cur_v: Optional[torch.Tensor], out: torch.Tensor,
                          workspace: torch.Tensor, stream=None) -> None:
    g, ch = geom.c(), cache.c()
    _check("lla_dense_decode_attn", library().lla_dense_decode_attn(
        ctypes.byref(g), ctypes.byref(ch), _ptr(context_lens), q.shape[0], max_ctx, _ptr(q),
        _ptr(cur_k), _ptr(cur_v), _dtype_code(q), _ptr(out), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream(stream)))


def _typed(t: Optional[torch.Tensor], dtype, name: str, shape=None):
    """The address of a contiguous tensor of `dtype` (and `shape`) on the current device, or None."""
    if t is None:
        return None
    p = _ptr(t)
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, which is not the current device")
    return p


def _scratch(t: torch.Tensor):
    """Address and bytes of a workspace on the current device."""
    p = _ptr(t)
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"the workspace is on {t.device}, which is not the current device")
    return p, t.numel() * t.element_size()


@dataclass
class Pages:
    """Sequences that share the blocks of a pool: ref_count [num_blocks] int32 (sequences that hold
    each block; 0: free), block_table [S][max_blocks] int32, context_lens [S] int32.  All zero: every block is
    free, every sequence empty.  Page sets over one pool share the ref_count tensor."""
    ref_count: torch.Tensor
    block_table: torch.Tensor
    context_lens: torch.Tensor

    def c(self) -> lla_pages:
        if self.ref_count.dim() != 1 or self.block_table.dim() != 2:
            raise ValueError("ref_count is [num_blocks], block_table [S][max_blocks]")
        S, mb = self.block_table.shape
        return lla_pages(_typed(self.ref_count, torch.int32, "ref_count"), self.ref_count.shape[0],
                         _typed(self.block_table, torch.int32, "block_table"), mb,
                         _typed(self.context_lens, torch.int32, "context_lens", (S,)), S)


@dataclass
class Pool:
    """One pool that page calls copy in, as lla_cache_pool, lla_cache_2d_pool or lla_rope_pool describe it."""
    base: torch.Tensor
    pages: int
    k_row_bytes: int
    v_row_bytes: int

    def c(self) -> lla_pool:
        return lla_pool(_ptr(self.base), self.pages, self.k_row_bytes, self.v_row_bytes)


class Pools:
    """The pools that a page call copies in (every layer's, and its rotary planes), marshalled once for all calls that
    take it (a list of Pool is marshalled at each)."""

    def __init__(self, pools=()):
        self.pools = tuple(pools)
        self.count = len(self.pools)
        self.array = (lla_pool * max(1, self.count))(*[p.c() for p in self.pools])
        self.address = ctypes.addressof(self.array)
        # blocks that every one of them has room for
        self.blocks = min((p.base.numel() * p.base.element_size() //
                           (LLA_BLOCK_TOKENS * p.pages * (p.k_row_bytes + p.v_row_bytes)) for p in self.pools),
                          default=1 << 62)
        self.device = self.pools[0].base.device.index if self.pools else -1
        if any(p.base.device.index != self.device for p in self.pools):
            raise ValueError("pools of one call must be on one device")

    def check(self, pages: Pages) -> None:
        if self.blocks < pages.ref_count.shape[0]:
            raise ValueError(f"a pool has {self.blocks} blocks, ref_count {pages.ref_count.shape[0]}")
        if self.count and self.device != torch.cuda.current_device():
            raise ValueError("the pools are not on the current device")


def _pool(fn: str, first, pool: torch.Tensor) -> Pool:
    out = lla_pool()
    _check(fn, getattr(library(), fn)(first, _ptr(pool), ctypes.byref(out)))
    return Pool(pool, out.pages, out.k_row_bytes, out.v_row_bytes)


def lla_cache_pool(geom: Geometry, pool: torch.Tensor) -> Pool:
    return _pool("lla_cache_pool", ctypes.byref(geom.c()), pool)


def lla_cache_2d_pool(geom: Geometry, pool: torch.Tensor) -> Pool:
    return _pool("lla_cache_2d_pool", ctypes.byref(geom.c()), pool)


def lla_rope_pool(d_rope: int, rope_pool: torch.Tensor) -> Pool:
    return _pool("lla_rope_pool", d_rope, rope_pool)


def lla_pages_fork(src: Pages, dst: Pages, parents: torch.Tensor, stream=None) -> None:
    """dst's sequence s becomes a copy of src's sequence parents[s] ([S] int32; -1: empty) on the same pages;
    src holds nothing afterwards."""
    if _done("lla_pages_fork", _native().pages_fork(src, dst, parents, _handle(stream))):
        return
    a, b = src.c(), dst.c()
    _check("lla_pages_fork", library().lla_pages_fork(
        ctypes.byref(a), ctypes.byref(b), _typed(parents, torch.int32, "parents", (b.S,)), _stream(stream)))


def lla_pages_extend_workspace_size(S: int) -> int:
    out = ctypes.c_size_t(0)
    _check("lla_pages_extend_workspace_size",
           library().lla_pages_extend_workspace_size(S, ctypes.byref(out)))
    return out.value


def lla_pages_extend(pages: Pages, pools: Pools, slot_mapping: torch.Tensor, workspace: torch.Tensor,
                     cu_new: Optional[torch.Tensor] = None, skip: Optional[torch.Tensor] = None,
                     lens_before: Optional[torch.Tensor] = None, free_blocks: Optional[torch.Tensor] = None,
                     stream=None) -> None:
    """Sequence s grows by cu_new[s + 1] - cu_new[s] tokens (cu_new [S + 1] int32), or each by
    slot_mapping.numel() / S; slot_mapping [N] int64 is written.  skip [S] uint8 (or bool): sequences that do not
    grow.  lens_before [S] int32, free_blocks [1] int32: written where given."""
    if _done("lla_pages_extend", _native().pages_extend(
            pages, pools, slot_mapping, workspace, cu_new, skip, lens_before, free_blocks, _handle(stream))):
        return
    p = pages.c()
    pools = pools if isinstance(pools, Pools) else Pools(pools)
    pools.check(pages)
    if skip is not None and skip.dtype == torch.bool:
        skip = skip.view(torch.uint8)
    _check("lla_pages_extend", library().lla_pages_extend(
        ctypes.byref(p), pools.address, pools.count, _typed(slot_mapping, torch.int64, "slot_mapping"),
        slot_mapping.numel(), _typed(cu_new, torch.int32, "cu_new", (p.S + 1,)),
        _typed(skip, torch.uint8, "skip", (p.S,)), _typed(lens_before, torch.int32, "lens_before", (p.S,)),
        _typed(free_blocks, torch.int32, "free_blocks", (1,)), *_scratch(workspace), _stream(stream)))


def lla_pages_free(pages: Pages, seqs: torch.Tensor, stream=None) -> None:
    """Frees the pages of the sequences seqs [n] int32 (negative: skipped)."""
    if _done("lla_pages_free", _native().pages_free(pages, seqs, _handle(stream))):
        return
    p = pages.c()
    _check("lla_pages_free", library().lla_pages_free(
        ctypes.byref(p), _typed(seqs, torch.int32, "seqs"), seqs.numel(), _stream(stream)))


def lla_pages_compact_workspace_size(num_blocks: int) -> int:
    out = ctypes.c_size_t(0)
    _check("lla_pages_compact_workspace_size",
           library().lla_pages_compact_workspace_size(num_blocks, ctypes.byref(out)))
    return out.value


def lla_pages_compact(pages: Pages, pools: Pools, remap: torch.Tensor, live: torch.Tensor,
                      workspace: torch.Tensor, stream=None) -> None:
    """Moves the blocks in use to the front of every pool.  remap [num_blocks] int32 (new number of each block, -1
    where free) and live [1] int32 (blocks in use) are written."""
    if _done("lla_pages_compact", _native().pages_compact(pages, pools, remap, live, workspace, _handle(stream))):
        return
    p = pages.c()
    pools = pools if isinstance(pools, Pools) else Pools(pools)
    pools.check(pages)
    _check("lla_pages_compact", library().lla_pages_compact(
        ctypes.byref(p), pools.address, pools.count, _typed(remap, torch.int32, "remap", (p.num_blocks,)),
        _typed(live, torch.int32, "live", (1,)), *_scratch(workspace), _stream(stream)))


def lla_beam_select_workspace_size(B: int, W: int, V: int, K: int, dtype=torch.bfloat16) -> int:
    out = ctypes.c_size_t(0)
    _check("lla_beam_select_workspace_size", library().lla_beam_select_workspace_size(
        B, W, V, K, LLA_BF16 if dtype == torch.bfloat16 else LLA_F32, ctypes.byref(out)))
    return out.value


def _logit_rows(logits: torch.Tensor) -> int:
    """The distance of the rows of logits [B][W][V], whose last dimension is dense (rows may be padded)."""
    if logits.dim() != 3 or logits.stride(2) != 1 and logits.shape[2] > 1:
        raise ValueError("logits are [B][W][V] with a dense last dimension")
    B, W, V = logits.shape
    rows = logits.stride(1) if W > 1 else logits.stride(0) if B > 1 else V
    if B > 1 and W > 1 and logits.stride(0) != W * rows:
        raise ValueError("the rows of logits must lie at one distance")
    if not logits.is_cuda:
        raise ValueError("tensors passed to liblla must be CUDA tensors")
    if logits.device.index != torch.cuda.current_device():
        raise ValueError(f"logits are on {logits.device}, which is not the current device")
    return rows


def lla_beam_select(logits: torch.Tensor, scores: torch.Tensor, parents: torch.Tensor, tokens: torch.Tensor,
                    out_scores: torch.Tensor, workspace: torch.Tensor, finished: Optional[torch.Tensor] = None,
                    lengths: Optional[torch.Tensor] = None, out_finished: Optional[torch.Tensor] = None,
                    out_lengths: Optional[torch.Tensor] = None, eos: int = -1, length_penalty: float = 0.0,
                    stream=None) -> None:
    """The best K = parents.shape[1] continuations of the beams: logits [B][W][V] (bf16 or fp32; rows may be
    padded), scores [B][W] fp32, finished [B][W] uint8, lengths [B][W] int32; parents, tokens [B][K] int32,
    out_scores [B][K] fp32, out_finished [B][K] uint8 and out_lengths [B][K] int32 are written."""
    if _done("lla_beam_select", _native().beam_select(
            logits, scores, parents, tokens, out_scores, workspace, finished, lengths, out_finished, out_lengths, eos,
            length_penalty, _handle(stream))):
        return
    rows = _logit_rows(logits)
    B, W, V = logits.shape
    if parents.dim() != 2:
        raise ValueError("parents are [B][K]")
    K = parents.shape[1]
    _check("lla_beam_select", library().lla_beam_select(
        B, W, V, K, logits.data_ptr(), rows, _dtype_code(logits), _typed(scores, torch.float32, "scores", (B, W)),
        _typed(finished, torch.uint8, "finished", (B, W)), _typed(lengths, torch.int32, "lengths", (B, W)), eos,
        length_penalty, _typed(parents, torch.int32, "parents", (B, K)), _typed(tokens, torch.int32, "tokens", (B, K)),
        _typed(out_scores, torch.float32, "out_scores", (B, K)),
        _typed(out_finished, torch.uint8, "out_finished", (B, K)),
        _typed(out_lengths, torch.int32, "out_lengths", (B, K)), *_scratch(workspace), _stream(stream)))


def lla_beam_search_workspace_size(B: int, W: int, V: int, dtype=torch.bfloat16) -> int:
    out = ctypes.c_size_t(0)
    _check("lla_beam_search_workspace_size", library().lla_beam_search_workspace_size(
        B, W, V, LLA_BF16 if dtype == torch.bfloat16 else LLA_F32, ctypes.byref(out)))
    return out.value


def lla_beam_search(pages_a: Pages, pages_b: Pages, pools: Pools, V: int, step, tokens: torch.Tensor,
                    scores: torch.Tensor, finished: torch.Tensor, lengths: torch.Tensor, parents: torch.Tensor,
                    workspace: torch.Tensor, dtype=torch.bfloat16, eos: int = -1, length_penalty: float = 0.0,
                    stream=None) -> None:
    """Beam search over parents.shape[0] steps: tokens, scores, finished, lengths [steps + 1][B][W] (slab 0 filled
    by the caller), parents [steps][B][W].  step(i, pages, lens_before, tokens, slots) runs the model for step i
    and returns its logits [B][W][V] of `dtype` (kept alive until the next step): pages is pages_a or pages_b,
    lens_before [B W] int32, tokens [B][W] int32 (slab 0, then the selected ones with 0 for the -1 of dead beams), slots
    [B W] int64 (-1: the beam does not grow).  It runs with `stream` as the current one."""
    if parents.dim() != 3:
        raise ValueError("parents are [steps][B][W]")
    steps, B, W = parents.shape
    slabs = (steps + 1, B, W)
    a, b = pages_a.c(), pages_b.c()
    pools = pools if isinstance(pools, Pools) else Pools(pools)
    pools.check(pages_a)
    pools.check(pages_b)
    base, nbytes = _scratch(workspace)
    flat = workspace.view(-1).view(torch.uint8)
    held, errors = [], []

    def _view(address, dtype_, size):
        return flat[address - base:address - base + size].view(dtype_)

    def _step(i, _pages, before, model_tokens, slots, logits, row_stride, _stream_, _user):
        try:
            n = B * W
            held.clear()  # the selection that reads the last step's logits is on the stream
            z = step(i, pages_b if i % 2 else pages_a, _view(before, torch.int32, 4 * n),
                     _view(model_tokens, torch.int32, 4 * n).view(B, W) if i else tokens[0], _view(slots, torch.int64, 8 * n))
            if z.dtype != dtype or tuple(z.shape) != (B, W, V):
                raise ValueError(f"step must return {dtype} logits of shape {(B, W, V)}, not {z.dtype} {tuple(z.shape)}")
            row_stride[0] = _logit_rows(z)
            logits[0] = z.data_ptr()
            held.append(z)
            z.record_stream(torch.cuda.current_stream())  # (of another stream's allocations the memory waits for this one)
            return 0
        except Exception as e:  # reported after the C call returns
            errors.append(e)
            return 1

    if dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"unsupported dtype {dtype}")
    cb = STEP_FN(_step)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream)
    with torch.cuda.stream(stream):  # None: the current one
        st = library().lla_beam_search(
            ctypes.byref(a), ctypes.byref(b), pools.address, pools.count, B, W, V,
            LLA_BF16 if dtype == torch.bfloat16 else LLA_F32, steps, eos, length_penalty,
            _typed(tokens, torch.int32, "tokens", slabs), _typed(scores, torch.float32, "scores", slabs),
            _typed(finished, torch.uint8, "finished", slabs), _typed(lengths, torch.int32, "lengths", slabs),
            _typed(parents, torch.int32, "parents"), cb, None, base, nbytes, _stream(None))
    if errors:
        raise errors[0]
    _check("lla_beam_search", st)


def lla_get_device_error(stream=None) -> int:
    """Returns the device error word (0 = no error) without raising."""
    word = ctypes.c_uint32(0)
    st = library().lla_get_device_error(_stream(stream), ctypes.byref(word))
    if st not in (0, 4, 5):
        raise LLAError("lla_get_device_error", st)
    return word.value


def lla_clear_device_error(stream=None) -> None:
    _check("lla_clear_device_error", library().lla_clear_device_error(_stream(stream)))


def lla_set_wait_limit_ns(nanoseconds: int) -> None:
    _check("lla_set_wait_limit_ns", library().lla_set_wait_limit_ns(int(nanoseconds)))


def lla_get_wait_limit_ns() -> int:
    return int(library().lla_get_wait_limit_ns())
