"""How much attention cached tokens get, by the columns (query, head) that a sequence has and the size of its queries, against
the fp64 oracle. The bar is that of test_gpu_cache_weights.py."""
import math

import numpy as np
import pytest
import torch

import decode_util as U
from oracle import cache_oracle as C
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu


def _queries(seed, n, heads, d, dtype, size=1.0):
    """Normal numbers times size (a number, or one per token and head), as the type holds them."""
    x = np.random.default_rng(seed).standard_normal((n, heads, d)) * np.asarray(size, np.float64).reshape(
        np.shape(size) + (1,) * (3 - np.ndim(size)))
    return torch.from_numpy(x).to(U.TORCH[dtype]).float().numpy()


def _check(host, gpu, q, counts, dtype, width, scale=None, ragged=True, causal=True, window=0, gap=0, seed=None, decay=0.75):
    """crvq_cache_weights with the softmax's exact sums, against the oracle; returns the weights."""
    import paper_2412_09282_gb300 as P
    d, n_kv = q.shape[2], host["K"].shape[1]
    scale = float(np.float32(1.0 / math.sqrt(d) if scale is None else scale))
    lse = D.attention(host, q, counts, scale, causal, window)[1].astype(np.float32)
    before = None
    if seed is not None:
        before = np.random.default_rng(seed).exponential(1.0, (len(counts), n_kv, width)).astype(np.float32)
    ref, slack = C.token_weights(host, q, lse, counts, scale, causal, window, before, float(np.float32(decay)), width)
    out = P.crvq_cache_weights(gpu, U.heads(q, dtype, gap), torch.from_numpy(lse).cuda(), scale=scale,
                               q_off=U.offsets(counts) if ragged else None, causal=causal, window=window,
                               weights=None if before is None else torch.from_numpy(before).cuda(), decay=decay,
                               out=torch.full((len(counts), n_kv, width), np.nan, device="cuda"))
    P.crvq_sync()
    per = 2.0 ** -23 + (2.0 ** -21 / (d + 16) if dtype == "f32" else 0.0)
    n = max(counts) * (q.shape[1] // n_kv)
    bound = per * slack * 1.01 + (2.0 ** -24 * n + 2.0 ** -23) * np.abs(ref) + n * 2.0 ** -125
    err = np.abs(U.exactly(out).astype(np.float64) - ref)
    assert np.all(err <= bound), float(np.nanmax(err / bound))   # (NaN is not)
    return out


@pytest.mark.parametrize("d,dtype,fmt", [(256, "f32", "int8"), (256, "f32", "e4m3"), (256, "bf16", "int8"), (128, "f32", "e4m3"),
                                         (64, "f32", "int8")])
@pytest.mark.parametrize("ragged,counts", [(False, [38, 38]), (False, [40, 40]), (False, [64, 64]), (False, [75, 75]),
                                           (True, [20, 18]), (True, [21, 20]), (True, [75, 1]), (True, [3, 150])])
def test_more_columns_than_shared_memory_holds(d, dtype, fmt, ragged, counts):
    """4 heads on one: 152, 160, 256 and 300 columns a sequence; by offsets, twice the average at a time."""
    host, gpu = U.make(80, [200, 161], 16, 1, d, fmt)
    q = _queries(81, sum(counts), 4, d, dtype)
    _check(host, gpu, q, counts, dtype, 208, ragged=ragged, seed=82)
