"""Attention over the paged 8-bit cache, against the fp64 oracle.

Bar. With r the unit roundoff of the output's type, u that of a weight (2^-11; 2^-21 from fp32, where q
and the weights are two fp16 pieces), and shake = (d + 16) scale sum |q||k| (the largest over the keys):
  |out - ref| <= r |ref| + (2 u + 2^-21 n / 16 + 4 (2^-23 + (2^-21 from fp32) / (d + 16)) shake + 2^-19) sum_j p_j |V_j|,
a score being off by at most 2^-23 per term of its sum (a tensor core's additions may truncate) and by q's
rounding, a weight by e^x of that (twice it, both in the sum and in the product), by its rounding, by exp2f's and
by the joins; the sums of n / 16 blocks' products add up in fp32. lse is off by the score's error, 2^-20 and
a unit of its own.
"""
import math

import numpy as np
import pytest
import torch

import decode_util as U
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu


def _queries(seed, n, heads, d, dtype, size=1.0):
    x = np.random.default_rng(seed).standard_normal((n, heads, d)).astype(np.float32) * np.float32(size)
    return torch.from_numpy(x).to(U.TORCH[dtype]).float().numpy()


def _check(host, gpu, q, counts, dtype, ragged=True, scale=None, causal=True, window=0, gap=0):
    import paper_2412_09282_gb300 as P
    d = q.shape[2]
    sc = 1.0 / math.sqrt(d) if scale is None else scale
    ref, lse_ref, mass, shake = D.attention(host, q, counts, float(np.float32(sc)), causal, window)
    out, lse = P.crvq_cache_attention(gpu, U.heads(q, dtype, gap), q_off=U.offsets(counts) if ragged else None,
                                      scale=sc, causal=causal, window=window, want_lse=True)
    P.crvq_sync()
    n = int(max(host["lens"]))
    per = 2.0 ** -23 + (2.0 ** -21 / (d + 16) if dtype == "f32" else 0.0)
    rel = 2 * U.WEIGHT_ROUND[dtype] + 2.0 ** -21 * n / 16 + 4 * per * shake[..., None] + 2.0 ** -19
    bound = U.OUT_ROUND[dtype] * np.abs(ref) + rel * mass + (2.0 ** -25 if dtype == "f16" else 1e-30)  # (fp16's subnormals)
    got = U.exactly(out).astype(np.float64)
    empty = ~np.isfinite(lse_ref)
    assert np.all(np.abs(got - ref) <= bound), float((np.abs(got - ref) / bound).max())
    assert np.all(got[empty] == 0)
    gl = U.exactly(lse).astype(np.float64)
    assert np.array_equal(np.isneginf(gl), empty)
    tol = 2 * per * shake + 2.0 ** -20 + 2.0 ** -20 * n / 16 + 2.0 ** -22 * np.abs(np.where(empty, 0, lse_ref))
    assert np.all(np.abs(gl[~empty] - lse_ref[~empty]) <= tol[~empty])
    return out


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,page,n_kv,group", [(128, 64, 2, 8), (64, 16, 3, 1), (256, 48, 1, 4), (128, 16, 1, 12)])
def test_single_tokens_of_ragged_lengths(fmt, dtype, d, page, n_kv, group):
    """Lengths around block, tile and page ends; an empty sequence."""
    lens = [1, 0, 15, 16, 17, 63, 64, 65, 129, 300]
    host, gpu = U.make(20, lens, page, n_kv, d, fmt, page_gap=1)
    q = _queries(21, len(lens), n_kv * group, d, dtype, 2.0)
    _check(host, gpu, q, [1] * len(lens), dtype, ragged=False, gap=5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 20), (True, 1), (False, 0), (False, 33)])
@pytest.mark.parametrize("d,group,counts", [
    (128, 4, [3, 1, 0, 9, 5]),            # a few drafted tokens, one sequence without a query
    (64, 1, [20, 2, 1, 40, 6]),           # more columns than a group of 16; more queries than keys (40 of 7)
    (128, 8, [17, 70, 4, 5, 100]),
])
def test_several_queries_masks_and_rows_without_keys(dtype, causal, window, d, group, counts):
    lens = [40, 70, 33, 7, 150]
    host, gpu = U.make(22, lens, 32, 2, d, "int8")
    q = _queries(23, sum(counts), 2 * group, d, dtype)
    _check(host, gpu, q, counts, dtype, causal=causal, window=window)


def test_long_sequences_split_over_many_blocks_and_joined():
    """One long sequence beside short ones: shares begin and end inside units."""
    import paper_2412_09282_gb300 as P
    lens = [9000, 3, 700, 0, 2049]
    host, gpu = U.make(24, lens, 128, 1, 64, "int8")
    q = _queries(25, 5, 2, 64, "f32")
    a = _check(host, gpu, q, [1] * 5, "f32", ragged=False)
    b = P.crvq_cache_attention(gpu, U.heads(q, "f32"))
    P.crvq_sync()
    assert torch.equal(a, b)                                   # no order that depends on timing


def test_scales_far_apart_and_peaked_scores():
    """Value scales from 1e-30 to 1e30 within one sequence, one dominating key, large and tiny queries."""
    host, _ = U.make(26, [200, 200, 200], 16, 1, 64, "e4m3")
    rng = np.random.default_rng(27)
    host["v_scale"] *= np.exp(rng.uniform(-69, 69, host["v_scale"].shape)).astype(np.float32)
    gpu = U.on_gpu(host, "e4m3")
    for dtype, size in (("f32", 1.0), ("bf16", 30.0), ("f32", 1e-6), ("bf16", 1e-30)):
        q = _queries(28, 3, 4, 64, dtype, size)
        _check(host, gpu, q, [1, 1, 1], dtype, ragged=False)
    q = _queries(29, 3, 4, 64, "f32", 1e5)
    _check(host, gpu, q, [1, 1, 1], "f32", ragged=False, scale=1e-5 / 8)


def test_not_finite_queries_stay_in_their_rows():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(30, [100], 16, 1, 64, "int8")
    q = _queries(31, 1, 6, 64, "bf16")
    ref = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "bf16")))
    q[0, 2, 7], q[0, 4, 1] = np.nan, np.inf
    out = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "bf16")))
    P.crvq_sync()
    ok = [0, 1, 3, 5]
    assert np.array_equal(out[0, ok], ref[0, ok]) and np.isnan(out[0, 2]).all() and np.isnan(out[0, 4]).all()


def test_bad_pages_lengths_and_offsets_are_reported():
    import paper_2412_09282_gb300 as P
    q = _queries(32, 2, 2, 64, "f32")
    for change in (lambda h: h["pages"].__setitem__((0, 1), 77), lambda h: h["lens"].__setitem__(0, 1000),
                   lambda h: h["lens"].__setitem__(0, -3)):
        host, _ = U.make(33, [40, 20], 16, 2, 64, "int8")
        change(host)
        gpu = U.on_gpu(host, "int8")
        out = P.crvq_cache_attention(gpu, U.heads(q, "f32"))
        with pytest.raises(P.CrvqError) as e:
            P.crvq_sync()
        assert e.value.status == -7
        one = dict(host, pages=host["pages"][1:], lens=host["lens"][1:])
        ref = D.attention(one, q[1:], [1], 1 / 8)[0]
        assert np.abs(U.exactly(out)[1] - ref[0]).max() < 1e-4
        assert np.isfinite(U.exactly(out)).all()
    host, gpu = U.make(33, [40, 20], 16, 2, 64, "int8")
    P.crvq_cache_attention(gpu, U.heads(q, "f32"), q_off=torch.tensor([0, 3, 2], dtype=torch.int32, device="cuda"))
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -7
    P.crvq_sync()


def test_refusals():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(34, [40, 20], 16, 2, 64, "int8")
    q = torch.ones((2, 4, 64), device="cuda")
    for bad in (dict(scale=float("nan")), dict(scale=float("inf")), dict(window=-1), dict(out=q.bfloat16())):
        with pytest.raises(P.CrvqError) as e:
            P.crvq_cache_attention(gpu, q, **bad)
        assert e.value.status == -1
    with pytest.raises(P.CrvqError):
        P.crvq_cache_attention(gpu, torch.ones((2, 3, 64), device="cuda"))   # no multiple of n_kv
    with pytest.raises(P.CrvqError):
        P.crvq_cache_attention(gpu, torch.ones((3, 4, 64), device="cuda"))   # 3 rows for 2 sequences
    with pytest.raises(TypeError):
        P.crvq_cache_attention(gpu, q.double())
    with pytest.raises(ValueError):
        P.crvq_cache_attention(gpu, torch.ones((2, 4, 128), device="cuda"))
    assert P.crvq_cache_attention(gpu, q[:0], q_off=torch.zeros(3, dtype=torch.int32, device="cuda")).shape[0] == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 70), (False, 0)])
@pytest.mark.parametrize("d,page,n_kv,group,lens,counts", [
    (128, 64, 2, 2, [300, 129], [150, 129]),        # two groups of rows, whole prompts, ends inside tiles
    (64, 16, 1, 8, [40, 700, 5, 0], [40, 33, 9, 2]),  # a short unit, more queries than keys, an empty sequence
    (128, 48, 1, 1, [1000], [700]),                 # three units of one sequence
])
def test_chunks_of_prompts(fmt, dtype, causal, window, d, page, n_kv, group, lens, counts):
    host, gpu = U.make(40, lens, page, n_kv, d, fmt, page_gap=1)
    q = _queries(41, sum(counts), n_kv * group, d, dtype, 1.5)
    _check(host, gpu, q, counts, dtype, causal=causal, window=window, gap=8 if group == 2 else 3)


def test_chunks_with_growing_maxima_and_scales_and_not_finite_queries():
    """Keys and value scales that grow along the sequence (outputs are rescaled many times), and rows with
    NaN and infinities beside finite ones."""
    import paper_2412_09282_gb300 as P
    host, _ = U.make(42, [900], 16, 1, 128, "int8")
    order = host["pages"][0, :57]
    ramp = np.exp(np.linspace(-2.0, 1.5, 57)).astype(np.float32)
    host["k_scale"][order, 0, 0] *= ramp
    host["v_scale"][order, 0, 0] *= np.exp(np.linspace(-8, 8, 57)).astype(np.float32)
    host["v_scale"][order[20], 0, 0] = 0.0
    gpu = U.on_gpu(host, "int8")
    q = _queries(43, 130, 2, 128, "f16", 1.0)
    _check(host, gpu, q, [130], "f16")
    ref = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "f16")))
    q[7, 1, 3], q[100, 0, 5] = np.nan, np.inf
    out = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "f16")))
    again = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "f16")))
    P.crvq_sync()
    same = np.ones((130, 2), bool)
    same[7, 1] = same[100, 0] = False
    assert np.array_equal(out[same], ref[same]) and np.isnan(out[~same]).all()
    assert np.array_equal(out, again, equal_nan=True)


def test_chunks_report_bad_pages_and_skip_them():
    import paper_2412_09282_gb300 as P
    host, _ = U.make(44, [400], 64, 1, 64, "int8")
    host["pages"][0, 2] = 1000
    gpu = U.on_gpu(host, "int8")
    q = _queries(45, 200, 1, 64, "bf16")
    out = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "bf16")))
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -7
    assert np.isfinite(out).all()
    # what is skipped counts as not cached: the same softmax without the tokens 128 .. 191
    K, V = (np.delete(np.concatenate([D.values(host, n, 0, 0, 128), np.zeros((64, 1, 64)), D.values(host, n, 0, 192, 400)]),
                      slice(128, 192), 0) for n in ("K", "V"))
    t = np.delete(np.arange(400), slice(128, 192))
    for j in (0, 57, 199):
        z = (K[:, 0] @ q[j, 0].astype(np.float64)) / 8
        z[t > 200 + j] = -np.inf
        w = np.exp(z - z.max())
        ref = (w / w.sum()) @ V[:, 0]
        assert np.abs(out[j, 0] - ref).max() <= 2.0 ** -7 * np.abs(V).max()


@pytest.mark.parametrize("d,counts", [(128, [40, 100]), (64, [64, 128])])
def test_fp16_chunks_are_as_exact_as_their_rounding(d, counts):
    """fp16 queries are exact operands, weights hold 22 bits: the outputs' rounding is all of the error that shows.
    Root mean squares over all outputs; 1.05 leaves room for the weights' 2^-21 and the sums' 2^-20."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(44, [300, 900], 64, 2, d, "int8")
    q = _queries(45, sum(counts), 16, d, "f16", 2.5)
    ref, _, _, _ = D.attention(host, q, counts, float(np.float32(1.0 / math.sqrt(d))), True, 0)
    out = P.crvq_cache_attention(gpu, U.heads(q, "f16"), q_off=U.offsets(counts))
    P.crvq_sync()
    err = U.exactly(out).astype(np.float64) - ref
    rounding = ref.astype(np.float16).astype(np.float64) - ref
    assert np.sqrt(np.mean(err ** 2)) <= 1.05 * np.sqrt(np.mean(rounding ** 2))


@pytest.mark.parametrize("n_seq,n_kv,group,most", [
    (40, 1, 3, 2),       # clusters of CTAs
    (300, 2, 4, 2),      # shares of a line
    (40, 1, 2, 70),      # tiles of 128 rows
])
def test_many_sequences(n_seq, n_kv, group, most):
    """More sequences than a warp's lanes, of which some are empty or ask nothing."""
    rng = np.random.default_rng(46)
    lens = rng.integers(0, 90, n_seq).tolist()
    counts = [int(rng.integers(min(n, most) // 2, min(n, most) + 1)) if i % 5 else 0 for i, n in enumerate(lens)]
    if most > 2:
        lens, counts = [n + 70 for n in lens], [most if i % 5 else 0 for i in range(n_seq)]
    host, gpu = U.make(47, lens, 16, n_kv, 64, "e4m3")
    q = _queries(48, sum(counts), n_kv * group, 64, "bf16")
    _check(host, gpu, q, counts, "bf16")
