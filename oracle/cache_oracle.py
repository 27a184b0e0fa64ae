"""CPU oracle of what is done around the 8-bit cache beside appending, reading and attending in order: trees of
drafted tokens, how much attention cached tokens get, which of them stay, and moving those together. Plain and slow,
in numpy, over the cache dicts of decode_oracle; sums in fp64, what rounds to codes in fp32, operation by operation.
"""
from __future__ import annotations

import math

import numpy as np

from oracle.decode_oracle import BLOCK, place, to_codes, values

F = np.float32


def ancestors(parents):
    """One tree: for every token the list of itself and its ancestors, itself first."""
    out = []
    for i, p in enumerate(parents):
        out.append([i] + (out[p] if 0 <= p < i else []))
    return out


def tree_mask(parents, counts, words, window=0, lens=None):
    """(mask [tokens, words] uint32, positions [tokens])."""
    mask = np.zeros((len(parents), words), np.uint32)
    positions = np.zeros(len(parents), np.int32)
    first = 0
    for b, n in enumerate(counts):
        for i, path in enumerate(ancestors(parents[first:first + n])):
            for j in path[:window] if window else path:
                if j < 32 * words:
                    mask[first + i, j // 32] |= np.uint32(1) << np.uint32(j % 32)
            positions[first + i] = (0 if lens is None else int(lens[b]) - n) + len(path) - 1
        first += n
    return mask, positions


def _attend(cache, q, counts, seen, scale):
    """decode_oracle.attention with seen(b, row, j, n, length) -> truth values of the sequence's tokens."""
    n_kv = cache["K"].shape[1]
    g, d = q.shape[1] // n_kv, q.shape[2]
    out, mass = np.zeros(q.shape), np.zeros(q.shape)
    shake, lse = np.zeros(q.shape[:2]), np.full(q.shape[:2], -np.inf)
    first = 0
    for b, n in enumerate(counts):
        length = int(cache["lens"][b])
        K, V = values(cache, "K", b, 0, length), values(cache, "V", b, 0, length)
        for j in range(n):
            see = seen(b, first + j, j, n, length)
            if not see.any():
                continue
            for h in range(q.shape[1]):
                x = q[first + j, h].astype(np.float64)
                k, v = K[see, h // g], V[see, h // g]
                z = scale * (k @ x)
                p = np.exp(z - z.max())
                out[first + j, h] = p @ v / p.sum()
                mass[first + j, h] = p @ np.abs(v) / p.sum()
                lse[first + j, h] = z.max() + math.log(p.sum())
                shake[first + j, h] = (d + 16) * abs(scale) * (np.abs(k) @ np.abs(x)).max()
        first += n
    return out, lse, mass, shake


def tree_attention(cache, q, counts, mask, scale, window=0, positions=None):
    """(out, lse, mass, shake) as decode_oracle.attention returns them."""
    words = mask.shape[1]

    def seen(b, row, j, n, length):
        t, held = np.arange(length), length - n
        lo = 0
        if window:
            lo = max(0, min(max(int(positions[row]), held), length - 1) - window + 1)
        i = t - held
        bits = np.zeros(length, bool)
        ok = (i >= 0) & (i < 32 * words)
        bits[ok] = mask[row, i[ok] // 32] >> (i[ok] % 32).astype(np.uint32) & 1
        return np.where(i < 0, t >= lo, bits)

    return _attend(cache, q, counts, seen, scale)


def token_weights(cache, q, lse, counts, scale, causal, window, before, decay, width):
    """(weights [n_seq, n_kv, width], slack of the same shape: the sum of every term times its score's error per unit
    roundoff)."""
    n_seq, n_kv = len(counts), cache["K"].shape[1]
    g, d = q.shape[1] // n_kv, q.shape[2]
    out, slack = np.zeros((n_seq, n_kv, width)), np.zeros((n_seq, n_kv, width))
    first = 0
    for b, n in enumerate(counts):
        length = int(cache["lens"][b])
        K = values(cache, "K", b, 0, length)
        t = np.arange(length)
        for j in range(n):
            pos = length - n + j
            see = (t <= pos) if causal else t >= 0
            if window:
                see = see & (t > pos - window)
            for h in range(q.shape[1]):
                if not math.isfinite(lse[first + j, h]):
                    continue
                x = q[first + j, h].astype(np.float64)
                p = np.where(see, np.exp(scale * (K[:, h // g] @ x) - lse[first + j, h]), 0.0)
                out[b, h // g, :length] += p
                slack[b, h // g, :length] += p * ((d + 16) * abs(scale) * (np.abs(K[:, h // g]) @ np.abs(x))
                                                  + abs(lse[first + j, h]) + 2)
        if before is not None:
            out[b, :, :length] += decay * before[b, :, :length].astype(np.float64)
        first += n
    return out, slack


def select(w, lens, keep, first, recent):
    """(idx [n_seq, n_kv, keep] with -1 behind the last, count [n_seq], weights [like w] of those that stay, in order)."""
    n_seq, n_kv, _ = w.shape
    idx = np.full((n_seq, n_kv, keep), -1, np.int32)
    out = np.zeros_like(w)
    count = np.minimum(np.asarray(lens, np.int32), keep).astype(np.int32)
    for b, length in enumerate(lens):
        for h in range(n_kv):
            t = np.arange(length)
            if length > keep:
                lo, hi = first, length - recent
                x = w[b, h, lo:hi].astype(np.float64)
                nan = np.isnan(x)                              # (above infinity)
                best = lo + np.lexsort((-np.where(nan, 0.0, x), ~nan))[:keep - first - recent]
                t = np.concatenate([t[:lo], np.sort(best), t[hi:]])
            idx[b, h, :len(t)] = t
            out[b, h, :len(t)] = w[b, h, t]
    return idx, count, out


def keep(cache, idx, count, start, out, fmt):
    """Moves tokens idx[b, h, r] of cache to places start[b] + r of out, r < count[b], in place (out may be cache)."""
    page, to_page, n_kv = cache["K"].shape[2], out["K"].shape[2], cache["K"].shape[1]
    old = {k: v.copy() for k, v in cache.items()}
    before = {k: v.copy() for k, v in out.items()}
    for b, n in enumerate(count):
        a = int(start[b])
        for p0 in range(a // BLOCK * BLOCK, a + n if n else 0, BLOCK):
            pg, at = place(out["pages"], to_page, b, p0)
            for h in range(n_kv):
                r = idx[b] if idx.ndim == 2 else idx[b, h]
                for name, scales in (("K", "k_scale"), ("V", "v_scale")):
                    codes, had = [], []
                    for p in range(p0, min(p0 + BLOCK, a + n)):
                        src, sp, s_at = before, pg, at + p - p0
                        if p >= a:
                            src = old
                            sp, s_at = place(old["pages"], page, b, int(r[p - a]))
                        codes.append(src[name][sp, h, s_at].astype(F))
                        had.append(src[scales][sp, h, s_at // BLOCK])
                    s = max(had)
                    for i, (c, f) in enumerate(zip(codes, had)):
                        out[name][pg, h, at + i] = to_codes(c * (f / s).astype(F), fmt) if s > 0 else 0
                    out[scales][pg, h, at // BLOCK] = s
