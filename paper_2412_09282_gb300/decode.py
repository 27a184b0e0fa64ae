"""Binding of the decode-step calls: the paged 8-bit key/value cache, attention over it and products
with 4-bit weights (argument marshalling only; semantics in include/crvq.h).

KVCache and Q4Matrix are handles that a program makes once around its tensors: they check types and
layouts and hold the C structure, so that a call marshals only what is new to it.
"""
from __future__ import annotations

import ctypes as C
import math

import torch

from . import _lib
from .api import _check, _L

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_FORMATS = {torch.int8: 0, torch.float8_e4m3fn: 1}
_addressof, _empty = C.addressof, torch.empty
# (a step's calls are short: the stream's handle without the Stream object around it, 2 us less)
_raw_stream = torch._C._cuda_getCurrentRawStream


def _foreign(stream, *tensors):
    """The handle of a stream given by the caller, on which the call's tensors are then in use: memory that a tensor gives
    up meanwhile waits for it. (The caller's to order: that stream after the work that makes the inputs.)"""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
    return stream.cuda_stream


def _device(t, dtype, name):
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _type(t, name):
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    return code


def _heads(t, name, head_dim):
    """crvq_heads of a tokens x heads x head_dim view with unit stride in the last dimension."""
    code = _TYPES.get(t.dtype)
    if code is None or not t.is_cuda:
        _type(t, name)                                           # (raises)
    shape, stride = t.shape, t.stride()
    if len(stride) != 3 or stride[2] != 1 or shape[2] != head_dim:
        raise ValueError(f"{name} must be tokens x heads x {head_dim} with unit stride in the last dimension")
    return _lib.crvq_heads(t.data_ptr(), stride[0], stride[1], shape[1], code)


def _offsets(off, n_seq, name):
    if off is None:
        return None
    _device(off, torch.int32, name)
    if off.shape != (n_seq + 1,) or not off.is_contiguous():
        raise ValueError(f"{name} must be contiguous with n_seq + 1 = {n_seq + 1} entries")
    return off.data_ptr()


class KVCache:
    """A paged cache in 8 bits (crvq_kv_cache): K, V [n_pages x n_kv x page x head_dim] int8 or
    float8_e4m3fn (the first dimension may have any stride that is a multiple of 16), k_scale, v_scale
    [n_pages x n_kv x page / 16] float32, pages [n_seq x max_pages] int32, lens [n_seq] int32 (tokens of
    every sequence, those of the present step included). The tensors are the caller's, and what they hold may
    change from call to call; for other tensors make another handle."""

    __slots__ = ("K", "V", "k_scale", "v_scale", "pages", "lens", "_c", "_addr", "n_seq", "n_kv", "head_dim",
                 "page", "device", "index")

    def __init__(self, K, V, k_scale, v_scale, pages, lens):
        if K.dtype not in _FORMATS:
            raise TypeError(f"K must be int8 or float8_e4m3fn, got {K.dtype}")
        _device(K, None, "K")
        _device(V, K.dtype, "V")
        _device(k_scale, torch.float32, "k_scale")
        _device(v_scale, torch.float32, "v_scale")
        _device(pages, torch.int32, "pages")
        _device(lens, torch.int32, "lens")
        if K.dim() != 4 or V.shape != K.shape or V.stride() != K.stride():
            raise ValueError("K and V must be n_pages x n_kv x page x head_dim, alike in shape and strides")
        n_pages, n_kv, page, d = K.shape
        if K.stride()[1:] != (page * d, d, 1):
            raise ValueError("K and V must be contiguous within a page")
        if page % 16:
            raise ValueError("page must be a multiple of 16 tokens")
        for name, s in (("k_scale", k_scale), ("v_scale", v_scale)):
            if s.shape != (n_pages, n_kv, page // 16) or not s.is_contiguous():
                raise ValueError(f"{name} must be n_pages x n_kv x page / 16, contiguous")
        if pages.dim() != 2 or pages.stride(1) != 1:
            raise ValueError("pages must be n_seq x max_pages with unit column stride")
        if lens.shape != (pages.shape[0],) or not lens.is_contiguous():
            raise ValueError("lens must be contiguous with one entry per sequence")
        stride = K.stride(0) if n_pages > 1 else n_kv * page * d
        ld = pages.stride(0) if pages.shape[0] > 1 else pages.shape[1]
        self.K, self.V, self.k_scale, self.v_scale, self.pages, self.lens = K, V, k_scale, v_scale, pages, lens
        self.n_seq, self.n_kv, self.page, self.head_dim = pages.shape[0], n_kv, page, d
        self.device, self.index = K.device, K.get_device()
        self._c = _lib.crvq_kv_cache(K.data_ptr(), V.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                     pages.data_ptr(), lens.data_ptr(), n_pages, stride, ld, pages.shape[0],
                                     pages.shape[1], page, n_kv, d, _FORMATS[K.dtype])
        self._addr = _addressof(self._c)

    def tensors(self):
        return self.K, self.V, self.k_scale, self.v_scale, self.pages, self.lens

    @staticmethod
    def empty(n_pages, n_kv, page, head_dim, pages, lens, dtype=torch.int8):
        """A cache over a new pool of pages (its codes are whatever the memory holds)."""
        dev = pages.device
        K = _empty((n_pages, n_kv, page, head_dim), device=dev, dtype=dtype)
        s = _empty((n_pages, n_kv, page // 16), device=dev, dtype=torch.float32)
        return KVCache(K, torch.empty_like(K), s, torch.empty_like(s), pages, lens)


def crvq_cache_append(cache, k, v, new_off=None, cos=None, sin=None, positions=None, interleaved=False,
                      q=None, q_out=None, stream=None):
    """Append new tokens' keys (rotated by the rows of cos / sin, [n_pos x half], at each token's place or
    `positions`) and values (tokens x n_kv x head_dim views) to the cache, whose lens count them already.
    With q (tokens x heads x head_dim), returns its rotated values (q_out, or a new tensor)."""
    d = cache.head_dim
    n_tok = k.shape[0]
    kc, vc = _heads(k, "k", d), _heads(v, "v", d)
    if v.shape[0] != n_tok:
        raise ValueError("k and v differ in tokens")
    rot = None
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin: give both or neither")
    if positions is not None and cos is None:
        raise ValueError("positions are rows of cos and sin, which are missing")
    if cos is not None:
        _device(cos, torch.float32, "cos")
        _device(sin, torch.float32, "sin")
        if cos.dim() != 2 or cos.stride(1) != 1 or sin.shape != cos.shape or sin.stride() != cos.stride():
            raise ValueError("cos and sin must be n_pos x half with unit column stride, alike")
        if positions is not None:
            _device(positions, torch.int32, "positions")
            if positions.shape != (n_tok,) or not positions.is_contiguous():
                raise ValueError("positions must be contiguous with one entry per token")
        n_pos, half = cos.shape
        rot = _lib.crvq_rotary(cos.data_ptr(), sin.data_ptr(), None if positions is None else positions.data_ptr(),
                               n_pos, cos.stride(0) if n_pos > 1 else half, half, 1 if interleaved else 0)
    qc = oc = None
    if q is not None:
        if q.shape[0] != n_tok:
            raise ValueError("q and k differ in tokens")
        if q_out is None:
            q_out = _empty(q.shape, device=q.device, dtype=q.dtype)
        elif q_out.shape != q.shape:
            raise ValueError("q_out must have the shape of q")
        qc, oc = _heads(q, "q", d), _heads(q_out, "q_out", d)
    st = _L().crvq_cache_append(cache._addr, _addressof(kc), _addressof(vc), n_tok,
                                _offsets(new_off, cache.n_seq, "new_off"),
                                None if rot is None else _addressof(rot), None if qc is None else _addressof(qc),
                                None if oc is None else _addressof(oc),
                                _raw_stream(cache.index) if stream is None else
                                _foreign(stream, k, v, q, q_out, new_off, cos, sin, positions, *cache.tensors()))
    if st:
        _check(st)
    return q_out


def crvq_cache_read(cache, start, off, n_tok, dtype=torch.float32, K_out=None, V_out=None, stream=None):
    """(K, V) values, [n_tok x n_kv x head_dim], of the tokens start[b] .. of every sequence b, whose rows
    are off[b] .. off[b + 1)."""
    shape = (n_tok, cache.n_kv, cache.head_dim)
    _device(start, torch.int32, "start")
    if start.shape != (cache.n_seq,) or not start.is_contiguous():
        raise ValueError("start must be contiguous with one entry per sequence")
    if K_out is None:
        K_out = _empty(shape, device=cache.device, dtype=dtype)
    elif K_out.shape != shape or not K_out.is_contiguous() or K_out.dtype != dtype:
        raise ValueError(f"K_out must be contiguous n_tok x n_kv x head_dim of {dtype}")
    if V_out is None:
        V_out = _empty(shape, device=cache.device, dtype=dtype)
    elif V_out.shape != shape or not V_out.is_contiguous() or V_out.dtype != dtype:
        raise ValueError(f"V_out must be contiguous n_tok x n_kv x head_dim of {dtype}")
    st = _L().crvq_cache_read(cache._addr, start.data_ptr(), _offsets(off, cache.n_seq, "off"), n_tok,
                              _type(K_out, "K_out"), K_out.data_ptr(), V_out.data_ptr(),
                              _raw_stream(cache.index) if stream is None else
                              _foreign(stream, K_out, V_out, start, off, *cache.tensors()))
    if st:
        _check(st)
    return K_out, V_out


def crvq_cache_attention(cache, q, q_off=None, scale=None, causal=True, window=0, out=None, want_lse=False,
                         stream=None):
    """Attention of the newest tokens' queries (tokens x heads x head_dim; scale 1 / sqrt(head_dim) unless
    given) over the cache; returns out, or (out, lse) with want_lse."""
    d = cache.head_dim
    qc = _heads(q, "q", d)
    if out is None:
        out = _empty(q.shape, device=q.device, dtype=q.dtype)
    elif out.shape != q.shape:
        raise ValueError("out must have the shape of q")
    oc = _heads(out, "out", d)
    lse = _empty(q.shape[:2], device=q.device, dtype=torch.float32) if want_lse else None
    st = _L().crvq_cache_attention(cache._addr, _addressof(qc), q.shape[0], _offsets(q_off, cache.n_seq, "q_off"),
                                   1.0 / math.sqrt(d) if scale is None else scale, causal, window,
                                   _addressof(oc), None if lse is None else lse.data_ptr(),
                                   _raw_stream(cache.index) if stream is None else
                                   _foreign(stream, q, out, lse, q_off, *cache.tensors()))
    if st:
        _check(st)
    return (out, lse) if want_lse else out


class Q4Matrix:
    """A matrix with 4-bit weights (crvq_q4_matrix): codes [M x ceil(N / 2)] uint8 (two per byte, the even
    column in the low bits), scales [M x ceil(N / group)] bfloat16, zeros of that shape, uint8, or None (8).
    Rows that begin on 16-byte boundaries are read fastest."""

    __slots__ = ("codes", "scales", "zeros", "M", "N", "group", "_c", "_addr", "device", "index")

    def __init__(self, codes, scales, zeros, N, group):
        _device(codes, torch.uint8, "codes")
        _device(scales, torch.bfloat16, "scales")
        M, half, G = codes.shape[0], (N + 1) // 2, -(-N // group)
        if codes.dim() != 2 or codes.shape[1] != half or codes.stride(1) != 1:
            raise ValueError("codes must be M x ceil(N / 2) with unit column stride")
        if scales.shape != (M, G) or (G > 1 and scales.stride(1) != 1):
            raise ValueError("scales must be M x ceil(N / group) with unit column stride")
        if zeros is not None:
            _device(zeros, torch.uint8, "zeros")
            if zeros.shape != scales.shape or zeros.stride() != scales.stride():
                raise ValueError("zeros must have the shape and strides of scales")
        self._set(codes, scales, zeros, M, N, group, codes.stride(0) if M > 1 else max(half, codes.stride(0)),
                  scales.stride(0) if M > 1 else G)

    def _set(self, codes, scales, zeros, M, N, group, ld_codes, ld_scales):
        self.codes, self.scales, self.zeros = codes, scales, zeros
        self.M, self.N, self.group, self.device, self.index = M, N, group, codes.device, codes.get_device()
        self._c = _lib.crvq_q4_matrix(codes.data_ptr(), scales.data_ptr(),
                                      None if zeros is None else zeros.data_ptr(), M, N, ld_codes, ld_scales,
                                      group, 0)
        self._addr = _addressof(self._c)

    @staticmethod
    def empty(M, N, group, zeros=False, device="cuda"):
        """Memory for an M x N matrix, rows on 16-byte boundaries."""
        half, G = (N + 1) // 2, -(-N // group)
        row = (half + 15) // 16 * 16
        codes = torch.empty_strided((M, half), (row, 1), device=device, dtype=torch.uint8)
        scales = _empty((M, G), device=device, dtype=torch.bfloat16)
        m = Q4Matrix.__new__(Q4Matrix)
        m._set(codes, scales, _empty((M, G), device=device, dtype=torch.uint8) if zeros else None, M, N, group, row, G)
        return m


def crvq_q4_quantize(W, group=128, symmetric=True, want_W_hat=False, out=None, stream=None):
    """W (M x N, unit column stride) in 4 bits by rounding, with a zero point per group unless symmetric:
    returns (Q4Matrix, W_hat fp32 or None)."""
    t = _type(W, "W")
    shape, stride = W.shape, W.stride()
    if len(shape) != 2 or stride[1] != 1:
        raise ValueError("W must be a 2-D tensor with unit column stride")
    M, N = shape
    if out is None:
        out = Q4Matrix.empty(M, N, group, zeros=not symmetric, device=W.device)
    elif (out.M, out.N, out.group, out.zeros is None) != (M, N, group, bool(symmetric)):
        raise ValueError("out is for another matrix")
    W_hat = _empty((M, N), device=W.device, dtype=torch.float32) if want_W_hat else None
    st = _L().crvq_q4_quantize(W.data_ptr(), stride[0] if M > 1 else N, t, out._addr,
                               None if W_hat is None else W_hat.data_ptr(),
                               _raw_stream(out.index) if stream is None else
                               _foreign(stream, W, W_hat, out.codes, out.scales, out.zeros))
    if st:
        _check(st)
    return out, W_hat


def crvq_q4_matvec(X, matrix, Y=None, stream=None):
    """Y = X W^T (b x M, of X's type) for 1 to 32 inputs X (b x N; a 1-D input is one row)."""
    t = _type(X, "X")
    if X.dim() == 1:
        X = X.unsqueeze(0)
    shape, stride, M = X.shape, X.stride(), matrix.M
    if len(shape) != 2 or stride[1] != 1 or shape[1] != matrix.N:
        raise ValueError(f"X must be b x {matrix.N} with unit column stride")
    b = shape[0]
    if Y is None:
        Y, ldy = _empty((b, M), device=matrix.device, dtype=X.dtype), M
    else:
        if Y.shape != (b, M) or Y.dtype != X.dtype or Y.stride(1) != 1:
            raise ValueError("Y must be b x M of X's type with unit column stride")
        ldy = Y.stride(0) if b > 1 else M
    st = _L().crvq_q4_matvec(matrix._addr, X.data_ptr(), stride[0] if b > 1 else shape[1], b, t, Y.data_ptr(), ldy,
                             _raw_stream(matrix.index) if stream is None else
                             _foreign(stream, X, Y, matrix.codes, matrix.scales, matrix.zeros))
    if st:
        _check(st)
    return Y
