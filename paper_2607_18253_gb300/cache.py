"""Thin Python binding of the paged KV cache and its attention (lr_cache_* in include/latency_router.h).

Argument marshalling only, as in ``router``: every step runs in the CUDA library, PyTorch
supplies device memory and the current stream, and without the library construction raises.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from .router import LR_OK, LRError, _CacheBatch, _CacheConfig, _P, _dev, _stream, load_library

LR_BF16, LR_FP16, LR_FP32 = 0, 1, 2
LR_CACHE_16BIT, LR_CACHE_E4M3, LR_CACHE_INT8 = 0, 1, 2

_DTYPES = {torch.bfloat16: LR_BF16, torch.float16: LR_FP16, torch.float32: LR_FP32}


def _i32(x) -> int:
    """x, or the nearest 32-bit number, which the library refuses: ctypes alone takes it modulo 2^32."""
    return x if -0x80000000 <= x <= 0x7FFFFFFF else -0x80000000 if x < 0 else 0x7FFFFFFF


class CacheBatch:
    """One token batch (lr_cache_batch): sequence s brings its last q_start[s+1] - q_start[s] of kv_len[s] tokens.

    q_start [n + 1], kv_len [n], block_table [n, >= 1]: int32 device tensors, kept and read by every call
    that takes the batch; max_q: no sequence brings more tokens than this."""

    def __init__(self, q_start: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, max_q: int):
        n = int(kv_len.numel())
        if block_table.dim() != 2 or block_table.shape[0] != n or (n > 0 and block_table.stride(1) != 1 and block_table.shape[1] > 1):
            raise ValueError("block_table must be [num_seqs, blocks] with unit stride along a row")
        if not block_table.is_cuda or block_table.dtype != torch.int32:
            raise TypeError("block_table must be an int32 CUDA tensor")
        self._keep = (q_start, kv_len, block_table)
        self._c = _CacheBatch(n, _i32(int(max_q)), _dev(q_start, torch.int32, "q_start", n + 1),
                              _dev(kv_len, torch.int32, "kv_len", n), block_table.data_ptr(),
                              max(int(block_table.stride(0)), int(block_table.shape[1])) if n <= 1 else int(block_table.stride(0)),
                              int(block_table.shape[1]))
        self._ref = ctypes.byref(self._c)


def _strides(t: torch.Tensor, name: str, heads: int, dim: int, dtype: torch.dtype) -> Tuple[int, int, int]:
    """(T, token stride, head stride) of a [T, heads, dim] CUDA tensor whose last dimension is dense."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{name} must be [T, {heads}, {dim}], got {tuple(shape)}")
    st, sh, sd = t.stride()
    if sd != 1:
        raise ValueError(f"{name} must be dense along its last dimension")
    # (a dimension of one element is never stepped along: its stride says nothing)
    T = shape[0]
    return T, (st if T > 1 else heads * dim), (sh if heads > 1 else dim)


class PagedCache:
    """A paged KV cache over caller-owned tensors, and the calls on it.

    k, v: [num_blocks, block_size, num_kv_heads, head_dim], of any equal strides that keep every vector dense and
    16-byte aligned (e.g. a transposed [num_blocks, num_kv_heads, block_size, head_dim]); their
    type is the format: `dtype` itself, torch.float8_e4m3fn or torch.int8.  The 8-bit formats take
    k_scale, v_scale: [num_blocks, block_size, num_kv_heads] float32 of equal strides.  The tensors are kept."""

    def __init__(self, *, k: torch.Tensor, v: torch.Tensor, num_q_heads: int, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16, max_seqs: int = 256):
        self._h = None
        self._lib = load_library()
        if dtype not in (torch.bfloat16, torch.float16):
            raise TypeError(f"dtype must be bfloat16 or float16, got {dtype}")
        fmt = {dtype: LR_CACHE_16BIT, torch.float8_e4m3fn: LR_CACHE_E4M3, torch.int8: LR_CACHE_INT8}.get(k.dtype)
        if fmt is None:
            raise TypeError(f"k must be {dtype}, float8_e4m3fn or int8, got {k.dtype}")
        for t, u, what in ((k, v, "k and v"),) + (((k_scale, v_scale, "k_scale and v_scale"),) if fmt else ()):
            if not isinstance(t, torch.Tensor) or not isinstance(u, torch.Tensor) or not t.is_cuda or not u.is_cuda:
                raise TypeError(f"{what} must be CUDA tensors")
            if t.dtype != u.dtype or t.shape != u.shape or t.stride() != u.stride():
                raise ValueError(f"{what} must have one type, shape and strides")
        if k.dim() != 4 or (k.shape[3] > 1 and k.stride(3) != 1):
            raise ValueError("k and v must be [num_blocks, block_size, num_kv_heads, head_dim], dense along the last dimension")
        nb, bs, H, D = k.shape
        if fmt and (k_scale.dtype != torch.float32 or tuple(k_scale.shape) != (nb, bs, H)):
            raise ValueError(f"k_scale and v_scale must be float32 [{nb}, {bs}, {H}]")
        # (the stride of a dimension of one element says nothing: zero is aligned)
        st = [0 if n == 1 else s for n, s in zip((nb, bs, H), k.stride())]
        ss = list(k_scale.stride()) if fmt else [0, 0, 0]
        self.num_q_heads, self.num_kv_heads, self.head_dim, self.dtype = int(num_q_heads), int(H), int(D), dtype
        cfg = _CacheConfig(_i32(int(num_q_heads)), H, D, _DTYPES[dtype], fmt, bs, nb, _i32(int(max_seqs)), k.data_ptr(), v.data_ptr(),
                           k_scale.data_ptr() if fmt else None, v_scale.data_ptr() if fmt else None, *st, *ss)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self._scale = 1.0 / math.sqrt(self.head_dim)
        torch.cuda.init()
        h = _P()
        rc = self._lib.lr_cache_create(ctypes.byref(cfg), ctypes.byref(h))
        if rc != LR_OK:
            raise LRError(rc, "lr_cache_create")
        self._h = h

    def close(self):
        if getattr(self, "_h", None):
            self._lib.lr_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int, what: str):
        if rc != LR_OK:
            raise LRError(rc, f"{what}: {self._lib.lr_cache_last_error(self._h).decode()}")

    def write(self, k: torch.Tensor, v: torch.Tensor, batch: CacheBatch, stream=None):
        """Store the batch's K and V, [T, num_kv_heads, head_dim] of equal strides (slices of a fused projection too)."""
        s = _strides(k, "k", self.num_kv_heads, self.head_dim, self.dtype)
        if _strides(v, "v", self.num_kv_heads, self.head_dim, self.dtype) != s:
            raise ValueError("k and v must have one shape and strides")
        rc = self._lib.lr_cache_write(self._h, batch._ref, s[0], k.data_ptr(), v.data_ptr(), s[1], s[2], _stream(stream))
        if rc:
            self._check(rc, "lr_cache_write")

    def read(self, batch: CacheBatch, tokens: int, dtype: Optional[torch.dtype] = None,
             out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """The batch's `tokens` tokens as values, (k, v) [tokens, num_kv_heads, head_dim] of the cache's dtype or float32."""
        dt = self.dtype if dtype is None else dtype
        T, H, D = int(tokens), self.num_kv_heads, self.head_dim
        if out is None:
            k = torch.empty((T, H, D), dtype=dt, device=self.k.device)
            v = torch.empty_like(k)
            kp, vp = k.data_ptr(), v.data_ptr()
        else:
            k, v = out
            kp, vp = _dev(k, dt, "k_out", T * H * D), _dev(v, dt, "v_out", T * H * D)
        rc = self._lib.lr_cache_read(self._h, batch._ref, T, _DTYPES.get(dt, -1), kp, vp, _stream(stream))
        if rc:
            self._check(rc, "lr_cache_read")
        return k, v

    def attend(self, q: torch.Tensor, batch: CacheBatch, scale: Optional[float] = None, window: int = 0, sinks: int = 0,
               out: Optional[torch.Tensor] = None, lse=False, stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """(out, lse) of the batch's queries [T, num_q_heads, head_dim]: out like q, lse [T, num_q_heads] float32 or None.

        scale: head_dim ** -0.5 if not given.  window, sinks: see lr_cache_attend.  lse: True, or the tensor to write."""
        Hq, D = self.num_q_heads, self.head_dim
        T, qt, qh = _strides(q, "q", Hq, D, self.dtype)
        if out is None:
            out = torch.empty((T, Hq, D), dtype=self.dtype, device=q.device)
            ot, oh = Hq * D, D
        else:
            To, ot, oh = _strides(out, "out", Hq, D, self.dtype)
            if To != T:
                raise ValueError("out must have q's shape")
        if lse is True:
            lse = torch.empty((T, Hq), dtype=torch.float32, device=q.device)
            lp = lse.data_ptr()
        else:
            lse = None if lse is False else lse
            lp = _dev(lse, torch.float32, "lse_out", T * Hq)
        rc = self._lib.lr_cache_attend(self._h, batch._ref, T, q.data_ptr(), qt, qh, self._scale if scale is None else scale,
                                       _i32(window), _i32(sinks), out.data_ptr(), ot, oh, lp, _stream(stream))
        if rc:
            self._check(rc, "lr_cache_attend")
        return out, lse

    def status(self, stream=None) -> int:
        """Synchronize the stream; return and clear the device status word."""
        return int(self._lib.lr_cache_status(self._h, _stream(stream)))
