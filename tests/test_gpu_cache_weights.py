"""How much attention cached tokens get, against the fp64 oracle.

Bar. A weight is e^(score - lse), both in fp32: the score is off by at most 2^-23 per term of its sum ((d + 16) scale sum |q||k|
of them; from fp32 queries 2^-21 / (d + 16) more of each, the second fp16 piece's rounding), lse's product with log2 e by
2^-23 |lse|, 2^x by 2^-22; a sum of n of them, in fp32, by 2^-24 n more, and the last sum by a rounding of each of its two
parts. What fp32 cannot hold (weights below 2^-126) counts as 0.
"""
import math

import numpy as np
import pytest
import torch

import decode_util as U
from oracle import cache_oracle as C
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def _queries(seed, n, heads, d, dtype, size=1.0):
    x = np.random.default_rng(seed).standard_normal((n, heads, d)).astype(np.float32) * np.float32(size)
    return torch.from_numpy(x).to(U.TORCH[dtype]).float().numpy()


def _before(seed, host, n_kv, width):
    w = np.random.default_rng(seed).exponential(1.0, (len(host["lens"]), n_kv, width)).astype(np.float32)
    return w                                                     # (places behind a sequence's tokens hold anything)


def _check(host, gpu, q, counts, dtype, width, ragged=True, causal=True, window=0, gap=0, decay=0.75, seed=None, lse=None,
           in_place=False):
    import paper_2412_09282_gb300 as P
    d, n_kv = q.shape[2], host["K"].shape[1]
    scale = 1.0 / math.sqrt(d)
    if lse is None:
        lse = D.attention(host, q, counts, float(np.float32(scale)), causal, window)[1].astype(np.float32)
    before = None if seed is None else _before(seed, host, n_kv, width)
    ref, slack = C.token_weights(host, q, lse, counts, float(np.float32(scale)), causal, window, before,
                                 float(np.float32(decay)), width)
    w = None if before is None else torch.from_numpy(before).cuda()
    out = P.crvq_cache_weights(gpu, U.heads(q, dtype, gap), torch.from_numpy(lse).cuda(),
                               q_off=U.offsets(counts) if ragged else None, causal=causal, window=window, weights=w,
                               decay=decay, out=w if in_place else
                               torch.full((len(counts), n_kv, width), np.nan, device="cuda"))
    P.crvq_sync()
    per = 2.0 ** -23 + (2.0 ** -21 / (d + 16) if dtype == "f32" else 0.0)
    n = max(counts) * (q.shape[1] // n_kv)
    bound = per * slack * 1.01 + (2.0 ** -24 * n + 2.0 ** -23) * np.abs(ref) + n * 2.0 ** -125
    got = U.exactly(out).astype(np.float64)
    assert np.all(np.abs(got - ref) <= bound), float((np.abs(got - ref) / bound).max())
    return out


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,page,n_kv,group", [(128, 64, 2, 8), (64, 16, 3, 1), (256, 48, 1, 4), (128, 16, 1, 12)])
def test_single_tokens_of_ragged_lengths(fmt, dtype, d, page, n_kv, group):
    lens = [1, 0, 15, 16, 17, 63, 64, 65, 129, 300]
    host, gpu = U.make(50, lens, page, n_kv, d, fmt, page_gap=1)
    q = _queries(51, len(lens), n_kv * group, d, dtype, 2.0)
    _check(host, gpu, q, [1] * len(lens), dtype, 320, ragged=False, gap=5, seed=52)
    _check(host, gpu, q, [1] * len(lens), dtype, 300, ragged=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 20), (True, 1), (False, 0), (False, 33)])
@pytest.mark.parametrize("d,group,counts", [
    (128, 4, [3, 1, 0, 9, 5]),            # one sequence without a query: what its tokens had, decayed
    (64, 1, [20, 2, 1, 40, 6]),           # more queries than keys (40 of 7)
    (128, 8, [17, 70, 4, 5, 100]),        # more columns than are taken at a time
    (64, 8, [40, 70, 33, 7, 64]),
])
def test_several_queries_and_masks(dtype, causal, window, d, group, counts):
    lens = [40, 70, 33, 7, 150]
    host, gpu = U.make(53, lens, 32, 2, d, "int8")
    q = _queries(54, sum(counts), 2 * group, d, dtype)
    _check(host, gpu, q, counts, dtype, 160, causal=causal, window=window, seed=55)
    _check(host, gpu, q, counts, dtype, 150, causal=causal, window=window, seed=56, decay=0.0, in_place=True)


@pytest.mark.parametrize("dtype,group,counts", [("f32", 1, [1, 1, 1]), ("bf16", 8, [20, 9, 1]), ("f16", 1, [3, 130, 2])])
def test_long_sequences_beside_short_ones_and_repeats(dtype, group, counts):
    host, gpu = U.make(57, [9000, 131, 2049], 128, 1, 64, "int8")
    q = _queries(58, sum(counts), group, 64, dtype)
    a = _check(host, gpu, q, counts, dtype, 9003, seed=59)
    b = _check(host, gpu, q, counts, dtype, 9003, seed=59)
    assert torch.equal(a, b)


def test_sums_are_the_softmaxs():
    """With the lse of attention itself every query gives its heads' weights, 1 each: a kv head's sum is the queries times
    the group."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(60, [500, 40], 16, 2, 128, "e4m3")
    q = U.heads(_queries(61, 20, 6, 128, "bf16"), "bf16")
    off = U.offsets([12, 8])
    _, lse = P.crvq_cache_attention(gpu, q, q_off=off, want_lse=True, window=30)
    w = P.crvq_cache_weights(gpu, q, lse, q_off=off, window=30)
    P.crvq_sync()
    # a score's two roundings (2^-23 of its 144 |q||k| / sqrt d, at most 2^-23 * 144 * 8 * |q| ~ 2^-13) and the sums'
    assert np.allclose(w.double().sum(2).cpu().numpy(), [[36, 36], [24, 24]], rtol=2.0 ** -11)


def test_queries_without_a_softmax_and_not_finite_ones():
    """Infinite lse adds nothing; NaN stays in the kv head of its query."""
    host, gpu = U.make(62, [100, 30], 16, 2, 64, "int8")
    q = _queries(63, 6, 4, 64, "f32")
    lse = D.attention(host, q, [4, 2], 0.125)[1].astype(np.float32)
    lse[1, 2], lse[3, 0], lse[5] = -np.inf, np.inf, -np.inf
    q[1, 2, 5] = np.nan                                         # (such a query's elements are not looked at)
    import paper_2412_09282_gb300 as P
    clean = q.copy()
    clean[1, 2, 5] = 0
    ref, _ = C.token_weights(host, clean, lse, [4, 2], 0.125, True, 0, None, 1.0, 100)
    got = P.crvq_cache_weights(gpu, U.heads(q, "f32"), torch.from_numpy(lse).cuda(), q_off=U.offsets([4, 2]),
                               out=torch.empty((2, 2, 100), device="cuda"))
    P.crvq_sync()
    assert np.allclose(U.exactly(got), ref, rtol=1e-4, atol=1e-30)
    q[0, 3, 1] = np.nan
    got = U.exactly(P.crvq_cache_weights(gpu, U.heads(q, "f32"), torch.from_numpy(lse).cuda(), q_off=U.offsets([4, 2]),
                                         out=torch.empty((2, 2, 100), device="cuda")))
    P.crvq_sync()
    assert np.isnan(got[0, 1, :97]).all() and np.allclose(got[0, 0], ref[0, 0], rtol=1e-4, atol=1e-30)
    assert np.allclose(got[1], ref[1], rtol=1e-4, atol=1e-30)


def test_views_of_sums():
    """Rows of a larger buffer, heads outside sequences, other strides before and after; what lies between stays."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(65, [50, 33, 7], 16, 2, 64, "int8")
    q = _queries(66, 3, 2, 64, "f32")
    lse = D.attention(host, q, [1, 1, 1], 0.125)[1].astype(np.float32)
    b = torch.rand((2, 3, 70), device="cuda")
    buf = torch.full((3, 2, 90), 5.0, device="cuda")
    before, out = b.transpose(0, 1)[:, :, :61], buf[:, :, 7:68]
    P.crvq_cache_weights(gpu, U.heads(q, "f32"), torch.from_numpy(lse).cuda(), weights=before, decay=0.5, out=out)
    P.crvq_sync()
    ref, _ = C.token_weights(host, q, lse, [1, 1, 1], 0.125, True, 0, before.cpu().numpy(), 0.5, 61)
    assert np.allclose(U.exactly(out), ref, rtol=1e-4, atol=1e-30)
    assert (buf[:, :, :7] == 5).all() and (buf[:, :, 68:] == 5).all()


def test_too_narrow_rows_bad_pages_and_lengths_are_reported():
    import paper_2412_09282_gb300 as P
    q = _queries(67, 2, 2, 64, "f32")
    lse = torch.zeros((2, 2), device="cuda")
    host, gpu = U.make(68, [60, 20], 16, 2, 64, "int8")
    buf = torch.full((2, 2, 48), 5.0, device="cuda")
    P.crvq_cache_weights(gpu, U.heads(q, "f32"), lse, out=buf[:, :, :40])
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -7
    assert (buf[:, :, 40:] == 5).all() and (buf[0, :, :40] != 5).all() and (buf[1, :, 20:40] == 0).all()
    for change in (lambda h: h["pages"].__setitem__((0, 1), 77), lambda h: h["lens"].__setitem__(0, 1000),
                   lambda h: h["lens"].__setitem__(0, -3)):
        host, _ = U.make(68, [60, 20], 16, 2, 64, "int8")
        change(host)
        gpu = U.on_gpu(host, "int8")
        w = P.crvq_cache_weights(gpu, U.heads(q, "f32"), lse)
        with pytest.raises(P.CrvqError) as e:
            P.crvq_sync()
        assert e.value.status == -7
        assert torch.isfinite(w).all() and (w[1, :, :20] > 0).all()
    P.crvq_sync()


def test_refusals():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(69, [40, 20], 16, 2, 64, "int8")
    q, lse, w = torch.ones((2, 4, 64), device="cuda"), torch.zeros((2, 4), device="cuda"), torch.zeros((2, 2, 48), device="cuda")
    for bad in (dict(scale=float("nan")), dict(window=-1), dict(decay=float("inf")), dict(decay=float("nan")),
                dict(weights=w[:, :, :40], out=w), dict(weights=w.as_strided((2, 2, 48), (48, 48, 1))),
                dict(out=w.as_strided((2, 2, 48), (48, 24, 1))), dict(weights=w, out=w.as_strided((2, 2, 48), (48, 96, 1)))):
        with pytest.raises(P.CrvqError) as e:
            P.crvq_cache_weights(gpu, q, lse, **bad)
        assert e.value.status == -1
    for bad in (dict(weights=w.double()), dict(out=w[:1]), dict(out=w[0]), dict(out=w.transpose(1, 2)), dict(weights=w.cpu())):
        with pytest.raises((TypeError, ValueError)):
            P.crvq_cache_weights(gpu, q, lse, **bad)
    for bad in (lse[:1], lse.double(), lse.t()):
        with pytest.raises((TypeError, ValueError)):
            P.crvq_cache_weights(gpu, q, bad)
    # no query at all: what was there, decayed
    w.fill_(2.0)
    out = P.crvq_cache_weights(gpu, q[:0], lse[:0], q_off=U.offsets([0, 0]), weights=w, decay=0.25)
    P.crvq_sync()
    assert (out[0, :, :40] == 0.5).all() and (out[0, :, 40:] == 0).all() and (out[1, :, :20] == 0.5).all() and (out[1, :, 20:] == 0).all()


def test_a_captured_step_replays_with_new_inputs():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(70, [90, 200], 16, 2, 64, "int8")
    q, w = torch.zeros((2, 8, 64), device="cuda", dtype=torch.bfloat16), torch.zeros((2, 2, 208), device="cuda")

    def step(w):
        out, lse = P.crvq_cache_attention(gpu, q, want_lse=True)
        return P.crvq_cache_weights(gpu, q, lse, weights=w, decay=0.9, out=w)

    step(w)
    torch.cuda.synchronize()
    w.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(w)
    eager = torch.zeros_like(w)
    for seed, lens in ((71, [90, 200]), (72, [7, 131])):
        q.copy_(torch.from_numpy(_queries(seed, 2, 8, 64, "bf16")))
        gpu.lens.copy_(_ints(lens))
        g.replay()
        step(eager)
        P.crvq_sync()
        assert torch.equal(w, eager) and (w != 0).any()
