"""Value scales far apart: a row's output depends on the tokens that it sees, by their weights, and not on how
large a scale is of tokens that it does not see or that weigh nothing.

Bar: that of test_gpu_attention, relative to the row's own sum of p |V| channel by channel, and a term for weights that are
small beside the row's largest: a weight is an fp16 number (or two), off by 2^-25 where it is subnormal, and the largest is
2^5 at least for tiles of 128 rows and 2^13 for few queries, so n of them are off by n 2^-30 (n 2^-38) of the largest, which is
at most its token's share of the largest channel's sum p |V| by twice (a token's largest code is not below half of its
block's). This term shows only in channels where the large values are 0. fp16 outputs hold 2^-24 to 2^16, so the
scales of their cases are 2^24 apart, the others' 2^60 (and 2^30); above 65504 they are infinite.
"""
import math

import numpy as np
import pytest
import torch

import decode_util as U
import test_gpu_attention as T
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu

APART = [("f32", 30), ("f32", 60), ("bf16", 30), ("bf16", 60), ("f16", 24)]


def _check(host, gpu, q, counts, dtype, ragged=True, causal=True, window=0, least=2.0 ** -37):
    import paper_2412_09282_gb300 as P
    d, n = q.shape[2], int(max(host["lens"]))
    sc = 1.0 / math.sqrt(d)
    ref, lse_ref, mass, shake = D.attention(host, q, counts, float(np.float32(sc)), causal, window)
    out = P.crvq_cache_attention(gpu, U.heads(q, dtype), q_off=U.offsets(counts) if ragged else None, causal=causal,
                                 window=window)
    P.crvq_sync()
    per = 2.0 ** -23 + (2.0 ** -21 / (d + 16) if dtype == "f32" else 0.0)
    rel = 2 * U.WEIGHT_ROUND[dtype] + 2.0 ** -21 * n / 16 + 4 * per * shake[..., None] + 2.0 ** -19
    bound = U.OUT_ROUND[dtype] * np.abs(ref) + rel * mass + n * least * mass.max(-1, keepdims=True) + \
        (2.0 ** -25 if dtype == "f16" else 1e-30)
    got = U.exactly(out).astype(np.float64)
    fits = np.abs(ref) + bound <= 65504 if dtype == "f16" else np.ones(ref.shape, bool)
    assert np.all((np.abs(got - ref) <= bound)[fits]), float((np.abs(got - ref) / bound)[fits].max())
    assert np.all((got * np.sign(ref))[~fits] >= 65504 * (1 - 2.0 ** -8))
    assert np.all(got[~np.isfinite(lse_ref)] == 0)
    return out


def _apart(host, page, fmt, blocks, by, b=0):
    """The value scales of the given blocks of sequence b 2^by times the others', for every head."""
    top = 40.0 if fmt == "int8" else 120.0
    small = 2.0 ** -16 if by == 24 else 1.0 / top             # (fp16 outputs: see above)
    live = np.isfinite(host["v_scale"])
    host["v_scale"][live] *= np.float32(top * small)
    for i in blocks:
        host["v_scale"][host["pages"][b][16 * i // page], :, i % (page // 16)] *= np.float32(2.0 ** by)


def _away(host, page, blocks, b=0):
    """Keys of the given blocks that queries of positive entries score far below all others (e^-48 and less)."""
    for i in blocks:
        host["K"][host["pages"][b][16 * i // page], :, 16 * i % page:16 * i % page + 16] = -120.0
        host["k_scale"][host["pages"][b][16 * i // page], :, i % (page // 16)] = 1.0 / 16.0


def _ask(seed, n, heads, d, dtype):
    return np.abs(T._queries(seed, n, heads, d, dtype))


CHUNKS = [c for c in APART if c[0] != "f32"]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,by", CHUNKS)
@pytest.mark.parametrize("d,group", [(128, 2), (64, 3)])
def test_chunks_large_scales_that_other_queries_see(fmt, dtype, by, d, group):
    """A block that only later queries of its tile see; a block that only earlier queries' windows hold."""
    host, _ = U.make(70, [300], 16, 1, d, fmt)
    _apart(host, 16, fmt, [7, 17], by)
    gpu = U.on_gpu(host, fmt)
    q = T._queries(71, 300, group, d, dtype)
    _check(host, gpu, q, [300], dtype, least=2.0 ** -29)
    _check(host, gpu, q, [300], dtype, window=40, least=2.0 ** -29)
    _check(host, gpu, q[:90], [90], dtype, causal=False, window=150, least=2.0 ** -29)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,by", CHUNKS)
@pytest.mark.parametrize("at", [0, 3, 9, 18])
def test_chunks_large_scales_that_weigh_nothing(fmt, dtype, by, at):
    """A block that every query sees (if it is not the last) and that none gives weight."""
    host, _ = U.make(72, [300], 16, 1, 128, fmt)
    _apart(host, 16, fmt, [at], by)
    _away(host, 16, [at])
    gpu = U.on_gpu(host, fmt)
    _check(host, gpu, _ask(73, 100, 2, 128, dtype), [100], dtype, least=2.0 ** -29)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_chunks_of_values_with_scale_zero(dtype):
    """Whole tiles, and blocks beside others, whose value scale is zero: their tokens count in the sum alone."""
    host, _ = U.make(74, [300], 16, 1, 64, "int8")
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 11):
        host["v_scale"][host["pages"][0][i]] = 0.0
    gpu = U.on_gpu(host, "int8")
    q = T._queries(75, 300, 2, 64, dtype)
    out = _check(host, gpu, q, [300], dtype, least=2.0 ** -29)
    assert bool((out[:128] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_chunks_with_a_scale_that_is_not_a_number(dtype):
    """Rows that see the block are not numbers, the others are as without it."""
    import paper_2412_09282_gb300 as P
    host, _ = U.make(76, [200], 16, 1, 64, "int8")
    gpu = U.on_gpu(host, "int8")
    q = T._queries(77, 200, 1, 64, dtype)
    ref = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, dtype)))
    gpu.v_scale[int(host["pages"][0][5])] = float("nan")             # tokens 80 .. 95
    out = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, dtype)))
    P.crvq_sync()
    assert np.array_equal(out[:80], ref[:80]) and not np.isfinite(out[80:]).any()


@pytest.mark.parametrize("wide", [None, 800])                        # clusters of CTAs, shares of a line
@pytest.mark.parametrize("dtype,by", APART)
@pytest.mark.parametrize("d,group,count", [(128, 2, 20), (64, 1, 30), (64, 1, 5), (128, 8, 1), (256, 1, 6), (256, 3, 20)])
def test_few_queries_large_scales_that_other_queries_see(dtype, by, d, group, count, wide):
    """Blocks that only some of a unit's queries see, by causality and by the window."""
    for fmt, length in (("int8", 60), ("e4m3", 52)):
        host, _ = U.make(78, [length], 16, 1, d, fmt, wide=wide)
        _apart(host, 16, fmt, [0, 3], by)
        gpu = U.on_gpu(host, fmt)
        q = T._queries(79, count, group, d, dtype)
        _check(host, gpu, q, [count], dtype)
        _check(host, gpu, q, [count], dtype, window=34)


@pytest.mark.parametrize("wide", [None, 800])
@pytest.mark.parametrize("dtype,by", APART)
@pytest.mark.parametrize("d,group", [(128, 8), (64, 1), (256, 4)])
def test_few_queries_large_scales_that_weigh_nothing(dtype, by, d, group, wide):
    """A block that every query sees and that none gives weight: first, between others, last."""
    for fmt in ("int8", "e4m3"):
        for at in (0, 1, 6, 20, 31):
            host, _ = U.make(80, [500], 16, 1, d, fmt, wide=wide)
            _apart(host, 16, fmt, [at], by)
            _away(host, 16, [at])
            _check(host, U.on_gpu(host, fmt), _ask(81, 1, group, d, dtype), [1], dtype, ragged=False)


@pytest.mark.parametrize("wide", [None, 800])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_queries_and_values_with_scale_zero(dtype, wide):
    """Blocks whose value scale is zero, alone and beside others: their tokens count in the sum alone."""
    for lens, zero in (([300], (0, 1, 2, 11)), ([40], (0, 1, 2))):
        host, _ = U.make(82, lens, 16, 1, 64, "int8", wide=wide)
        for i in zero:
            host["v_scale"][host["pages"][0][i]] = 0.0
        gpu = U.on_gpu(host, "int8")
        _check(host, gpu, T._queries(83, 1, 4, 64, dtype), [1], dtype)


@pytest.mark.parametrize("wide", [None, 800])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_few_queries_and_the_smallest_and_largest_scales(d, wide):
    """Scales from fp32's smallest normal number to near its largest, in sequences of their own and within one."""
    for exps in ([-126] * 8, [118] * 8, [-126, 118, -60, 0, 60, -126, 100, -100]):
        host, _ = U.make(84, [128], 16, 1, d, "int8", wide=wide)
        for i, e in enumerate(exps):
            host["v_scale"][host["pages"][0][i]] = np.ldexp(np.float32(1), e)
        _check(host, U.on_gpu(host, "int8"), T._queries(85, 1, 3, d, "f32"), [1], "f32")


@pytest.mark.parametrize("wide", [None, 800])
def test_few_queries_with_a_scale_that_is_not_a_number(wide):
    """Rows that see the block are not finite, the others are as without it."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(86, [60], 16, 1, 64, "int8", wide=wide)
    q = T._queries(87, 30, 1, 64, "f32")
    ref = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "f32")))
    gpu.v_scale[int(host["pages"][0][3])] = float("nan")             # tokens 48 .. 59
    out = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "f32")))
    P.crvq_sync()
    assert np.array_equal(out[:18], ref[:18]) and not np.isfinite(out[18:]).any()


@pytest.mark.parametrize("count", [1, 40])                           # few queries, tiles of 128 rows
def test_scores_of_the_largest_scale(count):
    """Queries of zeros score 0 at any scale that is taken; a scale whose product with log2(e) is not finite is refused."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(88, [60], 16, 1, 64, "int8")
    q = torch.zeros((count, 2, 64), device="cuda", dtype=torch.bfloat16)
    ref = P.crvq_cache_attention(gpu, q, scale=1.0)
    assert torch.equal(P.crvq_cache_attention(gpu, q, scale=2.0 ** 127), ref) and bool(ref.isfinite().all())
    for scale in (3e38, -3e38):
        with pytest.raises(P.CrvqError) as e:
            P.crvq_cache_attention(gpu, q, scale=scale)
        assert e.value.status == -1
