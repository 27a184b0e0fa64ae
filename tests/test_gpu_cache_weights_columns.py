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


def _sizes(kind, n, heads):
    """Powers of two that the queries are multiplied by: all alike, or others from query to query and head to head."""
    if not isinstance(kind, list):
        return 2.0 ** kind
    return 2.0 ** np.array([[kind[(3 * i + j) % len(kind)] for j in range(heads)] for i in range(n)], np.float64)


# scores near 1: queries of about 2^a, a scale of 2^-a / sqrt d (keys' scales 2^b, the scale 2^-a-b)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,log_scale,key_log", [
    (113, -113, 0), (116, -116, 0), (120, -120, 0), (125, -125, 0),      # 1e34 to 4e37
    (-60, 60, 0), (-66, 66, 0), (-100, 100, 0), (-120, 120, 0),
    (120, -95, -25), (60, -90, 30), (-40, 66, -26),                      # scale * (key's scale) beyond the normal numbers, or the scale alone
    ([100, 97, 30, -20, 94], -100, 0),                                   # some queries far, others not, and of all sizes
    ([120, 118, 60, 119], -120, 0),
    ([3, -80, 1, -90], 0, 0),                                            # scores of next to nothing
])
@pytest.mark.parametrize("d,n_kv,group,counts,gap", [
    (128, 2, 8, [3, 4], 0),                                              # fewer than 64 columns a sequence on average, and more
    (128, 2, 8, [9, 8], 0), (128, 1, 8, [70, 20], 5), (64, 2, 8, [20, 7], 0)])
def test_queries_of_any_size(dtype, size, log_scale, key_log, d, n_kv, group, counts, gap):
    host, _ = U.make(83, [300, 141], 16, n_kv, d, "int8" if d == 128 else "e4m3")
    host["k_scale"] *= np.float32(2.0 ** key_log)
    gpu = U.on_gpu(host, "int8" if d == 128 else "e4m3")
    q = _queries(84, sum(counts), n_kv * group, d, dtype, _sizes(size, sum(counts), n_kv * group))
    q[0, 1] = 0                                                          # (a query of zeros)
    assert np.isfinite(q).all() and (q != 0).any()
    for window in (0, 50):
        _check(host, gpu, q, counts, dtype, 310, scale=2.0 ** log_scale / math.sqrt(d), gap=gap, window=window, seed=85)


@pytest.mark.parametrize("d", [64, 128])
def test_far_and_ordinary_queries_by_turns(d):
    """Queries a sequence's several fillings of shared memory hold: far ones in some, none in others, and call after call."""
    host, gpu = U.make(86, [700], 32, 2, d, "int8")
    for kinds in ([0], [118], [0, 118]):
        size = np.ones((330, 8))
        for i, k in enumerate(kinds):
            size[128 * (2 * i):128 * (2 * i + 1)] = 2.0 ** k            # (4 heads on one: 512 columns, 128 queries a filling)
        q = _queries(87, 330, 8, d, "bf16", size)
        _check(host, gpu, q, [330], "bf16", 704, scale=2.0 ** -max(kinds) / math.sqrt(d), ragged=False, seed=88)


def test_not_finite_queries_beside_far_ones():
    """NaN and infinity stay in the kv head of their query, whatever its neighbours' sizes are."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(89, [200], 16, 2, 128, "int8")
    q = _queries(90, 20, 8, 128, "bf16", 2.0 ** 118)
    scale = 2.0 ** -118 / math.sqrt(128)
    lse = D.attention(host, q, [20], scale)[1].astype(np.float32)
    ref, _ = C.token_weights(host, q, lse, [20], scale, True, 0, None, 1.0, 200)
    for bad in (np.nan, np.inf):
        x = q.copy()
        x[19, 6, 3] = bad
        w = P.crvq_cache_weights(gpu, U.heads(x, "bf16"), torch.from_numpy(lse).cuda(), scale=scale,
                                 out=torch.empty((1, 2, 200), device="cuda"))
        P.crvq_sync()
        w = U.exactly(w)
        assert np.allclose(w[0, 0], ref[0, 0], rtol=1e-4, atol=1e-30) and not np.isfinite(w[0, 1]).all()
