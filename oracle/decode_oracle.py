"""CPU oracle of the decode-step calls: the 8-bit cache, attention over it and 4-bit products, plain and
slow, in numpy.

The cache is four arrays: codes K, V [n_pages, n_kv, page, d] as float values of the codes, scales
[n_pages, n_kv, page / 16]. What rounds to codes is restated in fp32, operation by operation (append,
q4_quantize: codes then compare as equal); sums are in fp64 (attention, q4_matvec).
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 16
F = np.float32


def e4m3(x):
    """Nearest e4m3 value (ties to even, saturating at 448), of fp32 or fp64 values."""
    x = np.asarray(x)
    a = np.minimum(np.abs(x.astype(np.float64)), 448.0)
    _, e = np.frexp(a)                               # a = m 2^e, m in [1/2, 1)
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    return np.copysign(np.rint(a / step) * step, x).astype(np.float32)


def to_codes(x, fmt):
    return np.clip(np.rint(x), -127, 127).astype(np.float32) if fmt == "int8" else e4m3(x)


def rotate(x, cos, sin, interleaved):
    """x [tokens, heads, d] fp32; cos, sin [tokens, half] fp32: every product and sum rounded to fp32."""
    y = x.astype(F).copy()
    h = cos.shape[1]
    c, s = cos[:, None, :].astype(F), sin[:, None, :].astype(F)
    ia, ib = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    a, b = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def place(pages, page, b, p):
    return int(pages[b][p // page]), p % page


def append(cache, x, counts, fmt):
    """Writes the new tokens x {"K", "V"} [tokens, n_kv, d] (keys already rotated) into the cache dict
    (K, V, k_scale, v_scale, pages, lens) in place; lens count them already."""
    page = cache["K"].shape[2]
    inv = F(1.0 / (127.0 if fmt == "int8" else 448.0))
    first = 0
    for b, n in enumerate(counts):
        length = int(cache["lens"][b])
        held = length - n
        if n == 0:
            continue
        for p0 in range(held // BLOCK * BLOCK, length, BLOCK):
            pg, at = place(cache["pages"], page, b, p0)
            end = min(p0 + BLOCK, length)
            for name, scales in (("K", "k_scale"), ("V", "v_scale")):
                lo = max(p0, held)
                new = x[name][first + lo - held:first + end - held].astype(F)      # tokens x heads x d
                new = np.where(np.isfinite(new), new, F(0))
                s = np.abs(new).max((0, 2)) * inv
                old = cache[name][pg, :, at:at + max(0, held - p0)]
                s0 = cache[scales][pg, :, at // BLOCK].copy()
                if held > p0:
                    s = np.maximum(s, s0)
                safe = np.where(s > 0, s, F(1))
                if held > p0:
                    old[...] = to_codes(old * (s0 / safe).astype(F)[:, None, None], fmt)
                cache[name][pg, :, at + lo - p0:at + end - p0] = \
                    to_codes(new / safe[:, None], fmt).transpose(1, 0, 2) if n else 0
                cache[scales][pg, :, at // BLOCK] = s
        first += n


def values(cache, name, b, first, last):
    """[last - first, n_kv, d] fp64."""
    page = cache["K"].shape[2]
    s = cache["k_scale" if name == "K" else "v_scale"]
    out = np.empty((last - first,) + (cache["K"].shape[1], cache["K"].shape[3]))
    for i, p in enumerate(range(first, last)):
        pg, at = place(cache["pages"], page, b, p)
        out[i] = cache[name][pg, :, at].astype(np.float64) * s[pg, :, at // BLOCK].astype(np.float64)[:, None]
    return out


def attention(cache, q, counts, scale, causal=True, window=0):
    """(out, lse, bound pieces): out [tokens, heads, d] fp64; mass = sum_j p_j |V_j| and shake = the largest
    error of a score per unit roundoff, (d + 16) scale sum |q||k|, for tolerances."""
    n_kv = cache["K"].shape[1]
    out = np.zeros(q.shape)
    mass, shake = np.zeros(q.shape), np.zeros(q.shape[:2])
    lse = np.full(q.shape[:2], -np.inf)
    g = q.shape[1] // n_kv
    d = q.shape[2]
    first = 0
    for b, n in enumerate(counts):
        length = int(cache["lens"][b])
        K, V = values(cache, "K", b, 0, length), values(cache, "V", b, 0, length)
        for j in range(n):
            pos = length - n + j
            lo = max(0, pos - window + 1) if window else 0
            hi = min(length, pos + 1) if causal else length
            if hi <= lo:
                continue
            for h in range(q.shape[1]):
                x = q[first + j, h].astype(np.float64)
                z = scale * (K[lo:hi, h // g] @ x)
                top = z.max()
                p = np.exp(z - top)
                L = p.sum()
                out[first + j, h] = p @ V[lo:hi, h // g] / L
                mass[first + j, h] = p @ np.abs(V[lo:hi, h // g]) / L
                lse[first + j, h] = top + math.log(L)
                shake[first + j, h] = (d + 16) * abs(scale) * (np.abs(K[lo:hi, h // g]) @ np.abs(x)).max()
        first += n
    return out, lse, mass, shake


def bf16(x):
    """fp32 values rounded to bf16 (ties to even)."""
    u = np.asarray(x, F).view(np.uint32)
    r = (u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)
    return r.view(F)


def q4_quantize(W, group, symmetric):
    """(codes [M, N] ints, scales [M, G] fp32 values of bf16, zeros [M, G]) as the call rounds them."""
    W = np.where(np.isfinite(W), W, 0).astype(F)
    M, N = W.shape
    G = -(-N // group)
    codes, scales, zeros = np.zeros((M, N), np.int64), np.zeros((M, G), F), np.full((M, G), 8.0, F)
    for g in range(G):
        w = W[:, g * group:(g + 1) * group]
        lo, hi = np.minimum(w.min(1), F(0)), np.maximum(w.max(1), F(0))
        if symmetric:
            s = np.maximum(hi, -lo) * F(1.0 / 7.0)
        else:
            with np.errstate(over="ignore"):
                s = (hi - lo) * F(1.0 / 15.0)
            s = np.where(np.isinf(s), hi * F(1.0 / 15.0) - lo * F(1.0 / 15.0), s)
        s = bf16(s)
        safe = np.where(s > 0, s, F(1))
        if not symmetric:
            zeros[:, g] = np.where(s > 0, np.clip(np.rint(-lo / safe), 0, 15), 0)
        q = np.clip(np.where(s[:, None] > 0, np.rint(w / safe[:, None]), 0) + zeros[:, g:g + 1], 0, 15)
        level = q - zeros[:, g:g + 1]
        above = np.abs(level.astype(np.float64) * s[:, None]) >= 2.0 ** 128 - 2.0 ** 103   # (rounds to infinity)
        codes[:, g * group:(g + 1) * group] = (q - np.where(above, np.sign(level), 0)).astype(np.int64)
        scales[:, g] = s
    return codes, scales, zeros


def q4_values(codes, scales, zeros, group):
    at = np.arange(codes.shape[1]) // group
    return (codes - zeros[:, at].astype(np.float64)) * scales[:, at].astype(np.float64)


def pack(codes):
    """Two codes per byte, the even column in the low bits."""
    M, N = codes.shape
    c = np.zeros((M, N + N % 2), np.uint8)
    c[:, :N] = codes
    return (c[:, 0::2] | c[:, 1::2] << 4).astype(np.uint8)


def unpack(packed, N):
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[0], -1)[:, :N].astype(np.int64)
