"""How exact cache attention is: root mean squares over all outputs, against the fp64 oracle, where the bars of single outputs are too
wide to show a lost low piece of a query or of a weight.

fp32 queries: two fp16 pieces hold an element to 2^-22 and a score's additions may truncate by 2^-23 of sum |q| |k| scale each:
about 2 sqrt(2 d / 16) of them that do not conspire, for a sum of about 0.64 sqrt(d) times the sizes of q and K (here 2 and 1),
so at most 5e-6 of a weight for d <= 256; weights hold 22 bits, and a sum of p V as many as its terms do. 5e-6 of the outputs' root mean
square, then; without q's low pieces it would be 3e-4, without the weights' 1e-4.
fp16 queries are exact operands and weights hold 22 bits: the outputs' rounding is all that shows (1.05 times it).
"""
import math

import numpy as np
import pytest
import torch

import decode_util as U
import test_gpu_attention as T
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("wide", [None, 1200])                       # clusters of CTAs, shares of a line
@pytest.mark.parametrize("d,n_kv,group,counts", [
    (64, 2, 8, [1, 1, 1]), (128, 2, 8, [1, 1, 1]), (256, 2, 4, [1, 1, 1]),     # units of 8 columns
    (64, 2, 4, [5, 3, 4]), (128, 2, 4, [5, 3, 4]), (256, 1, 4, [5, 3, 4]),     # of 16 (of 256 channels: 8)
])
def test_few_queries_are_as_exact_as_their_pieces(fmt, dtype, wide, d, n_kv, group, counts):
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(94, [300, 900, 77], 16, n_kv, d, fmt, wide=wide)
    q = T._queries(95, sum(counts), n_kv * group, d, dtype, 2.0)
    ref, lse_ref, _, _ = D.attention(host, q, counts, float(np.float32(1.0 / math.sqrt(d))), True, 0)
    out, lse = P.crvq_cache_attention(gpu, U.heads(q, dtype), q_off=U.offsets(counts), want_lse=True)
    P.crvq_sync()
    rms = lambda x: float(np.sqrt(np.mean(np.square(x))))
    err = rms(U.exactly(out).astype(np.float64) - ref)
    if dtype == "f32":
        assert err <= 5e-6 * rms(ref), err / rms(ref)
        assert np.abs(U.exactly(lse) - lse_ref).max() <= 5e-6 * max(1.0, np.abs(lse_ref).max())
    else:
        assert err <= 1.05 * rms(ref.astype(np.float16).astype(np.float64) - ref)


@pytest.mark.parametrize("d,counts,group", [(64, [70, 100], 2), (128, [40, 90], 2), (256, [20, 33], 3)])
def test_chunks_of_fp32_queries(d, counts, group):
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(96, [300, 500], 64, 1, d, "int8")
    q = T._queries(97, sum(counts), group, d, "f32", 2.0)
    ref, _, _, _ = D.attention(host, q, counts, float(np.float32(1.0 / math.sqrt(d))), True, 0)
    out = P.crvq_cache_attention(gpu, U.heads(q, "f32"), q_off=U.offsets(counts))
    P.crvq_sync()
    err = U.exactly(out).astype(np.float64) - ref
    assert np.sqrt(np.mean(err ** 2)) <= 5e-6 * np.sqrt(np.mean(ref ** 2))
