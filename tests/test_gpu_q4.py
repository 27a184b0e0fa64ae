"""4-bit weights with group scales: quantizing (equal to the oracle's codes, scales and values) and the
product, against fp64.

Bar of the product: codes, zero points and inputs are exact operands (fp32 inputs in three pieces), so
with S = sum over the inputs of |scale (code - zero) x|
  |y - ref| <= r |ref| + (136 + N / 64 + 24) 2^-23 S,
r the output's unit roundoff: up to 128 additions of a group (3 pieces: the same terms, thrice smaller
ones), N / 64 groups and warps in order at most; a tensor core's additions may truncate.
"""
import numpy as np
import pytest
import torch

import decode_util as U
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu


def _matrix(seed, M, N, group, zeros, pad=True):
    import paper_2412_09282_gb300 as P
    rng = np.random.default_rng(seed)
    G = -(-N // group)
    codes = rng.integers(0, 16, (M, N))
    scales = D.bf16(np.exp(rng.standard_normal((M, G))).astype(np.float32) * np.float32(0.01))
    z = rng.integers(0, 16, (M, G)).astype(np.float32) if zeros else np.full((M, G), 8.0, np.float32)
    packed = D.pack(codes)
    if N % 2:
        packed[:, -1] |= 0xF0                                  # past the row's end: ignored
    half = packed.shape[1]
    row = -(-half // 16) * 16 if pad else half
    buf = torch.full((M, row), 0xFF, dtype=torch.uint8)
    buf[:, :half] = torch.from_numpy(packed)
    m = P.Q4Matrix(buf.cuda()[:, :half], torch.from_numpy(scales).to(torch.bfloat16).cuda(),
                   torch.from_numpy(z).to(torch.uint8).cuda() if zeros else None, N, group)
    return m, D.q4_values(codes, scales, z, group)


def _check(m, W, X, dtype, gap=0):
    import paper_2412_09282_gb300 as P
    b, N = X.shape
    x = torch.from_numpy(X).to(U.TORCH[dtype])
    X = x.float().numpy().astype(np.float64)
    buf = torch.zeros((b, N + gap), dtype=x.dtype, device="cuda")
    buf[:, :N] = x.cuda()
    Y = P.crvq_q4_matvec(buf[:, :N], m)
    P.crvq_sync()
    ref, S = X @ W.T, np.abs(X) @ np.abs(W).T
    err = np.abs(U.exactly(Y).astype(np.float64) - ref)
    bound = U.OUT_ROUND[dtype] * np.abs(ref) + (160 + N / 64) * 2.0 ** -23 * S + 1e-30
    assert np.all(err <= bound), float((err / bound).max())
    return Y


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("b,M,N,zeros,pad", [
    (1, 1, 1, True, True), (1, 16, 128, False, True), (3, 37, 200, True, False), (8, 130, 1000, False, True),
    (9, 65, 1111, True, True), (16, 64, 2048, False, True), (17, 33, 640, True, False), (32, 100, 1536, True, True),
])
def test_matvec(dtype, group, b, M, N, zeros, pad):
    m, W = _matrix(40, M, N, group, zeros, pad)
    X = np.random.default_rng(41).standard_normal((b, N)).astype(np.float32)
    _check(m, W, X, dtype, gap=3 if b == 3 else 0)


def test_matvec_of_the_layer_shapes_and_repeatable():
    import paper_2412_09282_gb300 as P
    m, W = _matrix(42, 4096, 1032, 128, True)
    X = np.random.default_rng(43).standard_normal((5, 1032)).astype(np.float32)
    a = _check(m, W, X, "f32")
    assert torch.equal(a, P.crvq_q4_matvec(torch.from_numpy(X).cuda(), m))
    y = P.crvq_q4_matvec(torch.from_numpy(X[2]).cuda(), m)     # a 1-D input is one row
    assert y.shape == (1, 4096)


def test_matvec_wide_ranges_and_not_finite_inputs():
    import paper_2412_09282_gb300 as P
    m, W = _matrix(44, 48, 512, 64, True)
    X = np.random.default_rng(45).standard_normal((4, 512)).astype(np.float32)
    X *= np.exp2(np.random.default_rng(46).integers(-60, 60, X.shape)).astype(np.float32)
    _check(m, W, X, "f32")
    X = np.random.default_rng(45).standard_normal((4, 512)).astype(np.float32)
    ref = P.crvq_q4_matvec(torch.from_numpy(X).cuda(), m)
    X[1, 3], X[2, 200] = np.nan, np.inf
    Y = P.crvq_q4_matvec(torch.from_numpy(X).cuda(), m)
    P.crvq_sync()
    assert torch.equal(Y[0], ref[0]) and torch.equal(Y[3], ref[3])
    assert bool(Y[1].isnan().all()) and not bool(Y[2].isfinite().any())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("symmetric", [True, False])
@pytest.mark.parametrize("M,N,group", [(1, 1, 32), (5, 32, 32), (7, 75, 32), (33, 200, 64), (64, 512, 128), (9, 1001, 128)])
def test_quantize(dtype, symmetric, M, N, group):
    import paper_2412_09282_gb300 as P
    rng = np.random.default_rng(47)
    W = rng.standard_normal((M, N)).astype(np.float32) * 0.02
    W[0, :min(N, 40)] = 0
    W[M // 2] = np.abs(W[M // 2])
    w = torch.from_numpy(W).to(U.TORCH[dtype])
    codes, scales, zeros = D.q4_quantize(w.float().numpy(), group, symmetric)
    buf = torch.zeros((M, N + 3), dtype=w.dtype, device="cuda")
    buf[:, :N] = w.cuda()
    for src in (w.cuda(), buf[:, :N]):
        m, W_hat = P.crvq_q4_quantize(src, group, symmetric, want_W_hat=True)
        P.crvq_sync()
        assert np.array_equal(D.unpack(m.codes.cpu().numpy(), N), codes)
        assert np.array_equal(U.exactly(m.scales), scales)
        if not symmetric:
            assert np.array_equal(m.zeros.cpu().numpy(), zeros.astype(np.uint8))
        assert np.array_equal(U.exactly(W_hat), D.q4_values(codes, scales, zeros, group).astype(np.float32))
    Y = P.crvq_q4_matvec(torch.eye(N, device="cuda")[:min(N, 8)], m)
    assert torch.equal(Y, W_hat[:, :min(N, 8)].t())


def test_quantize_reports_what_is_not_finite_and_refusals():
    import paper_2412_09282_gb300 as P
    W = torch.randn(4, 64, device="cuda")
    ref, _ = P.crvq_q4_quantize(W, 32)
    W[2, 5] = float("inf")
    m, W_hat = P.crvq_q4_quantize(W, 32, want_W_hat=True)
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -6
    assert float(W_hat[2, 5]) == 0 and torch.equal(m.codes[:2], ref.codes[:2])
    P.crvq_sync()
    X = torch.ones((33, 64), device="cuda")
    with pytest.raises(P.CrvqError) as e:
        P.crvq_q4_matvec(X, m)
    assert e.value.status == -2
    with pytest.raises(ValueError):
        P.crvq_q4_matvec(torch.ones((2, 63), device="cuda"), m)
    with pytest.raises(TypeError):
        P.crvq_q4_matvec(torch.ones((2, 64), device="cuda", dtype=torch.float64), m)
    with pytest.raises(P.CrvqError) as e:
        P.crvq_q4_quantize(W, 96)
    assert e.value.status == -2


@pytest.mark.parametrize("symmetric", [True, False])
def test_quantize_wide_ranges_and_ties(symmetric):
    """Rows from subnormal to 2^120 (quotients by corrected products and by division), and weights halfway between
    two levels: codes, scales and values equal to the oracle's."""
    import paper_2412_09282_gb300 as P
    rng = np.random.default_rng(48)
    exps = np.array([-147, -140, -128, -120, -100, -82, -81, -80, -79, -78, -77, -76, -60, -3, 0, 5, 60, 76, 77, 78, 79, 80,
                     81, 82, 83, 84, 100, 120])
    W = np.ldexp(rng.standard_normal((len(exps), 128)), exps[:, None]).astype(np.float32)
    ties = np.tile((np.arange(128) % 15 - 7.5).astype(np.float32), (2, 1))    # scale 7.5 / 7 or 1, both rounded to bf16
    ties[1] = np.clip(ties[1], -7, 7)
    ties[1, 0] = 7                                                            # scale 1: halves are ties
    W = np.concatenate([W, ties])
    codes, scales, zeros = D.q4_quantize(W, 64, symmetric)
    m, W_hat = P.crvq_q4_quantize(torch.from_numpy(W).cuda(), 64, symmetric, want_W_hat=True)
    P.crvq_sync()
    assert np.array_equal(U.exactly(m.scales), scales)
    assert np.array_equal(D.unpack(m.codes.cpu().numpy(), 128), codes)
    assert np.array_equal(U.exactly(W_hat), D.q4_values(codes, scales, zeros, 64).astype(np.float32))
