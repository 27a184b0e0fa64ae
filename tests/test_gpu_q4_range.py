"""Quantizing weights up to fp32's largest number, with ranges above it: codes, scales and values equal to the oracle's,
finite, and as near as the levels allow."""
import numpy as np
import pytest
import torch

import decode_util as U
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu

TOP = float(np.finfo(np.float32).max)


def _weights(dtype):
    rng = np.random.default_rng(91)
    W = np.clip(rng.standard_normal((40, 128)) * 1.5e38, -TOP, TOP)
    W[0] = np.linspace(-TOP, TOP, 128)
    W[1, :64], W[1, 64:] = TOP, -TOP
    W[2] = np.where(np.arange(128) % 3 == 0, -TOP, np.linspace(0, TOP, 128))
    W[3] = np.linspace(-0.51 * TOP, 0.51 * TOP, 128)             # (hi - lo a little above)
    W[4] = np.linspace(-0.49 * TOP, 0.49 * TOP, 128)             # (and below)
    W[5] = TOP
    W[6] = -TOP
    W[7:23] *= np.linspace(0.5, 1.2, 16)[:, None]
    w = torch.from_numpy(np.clip(W, -TOP, TOP).astype(np.float32)).to(U.TORCH[dtype])
    return torch.where(w.isinf(), w.sign() * torch.finfo(w.dtype).max, w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("symmetric", [True, False])
@pytest.mark.parametrize("group", [32, 128])
def test_ranges_above_the_largest_number(dtype, symmetric, group):
    import paper_2412_09282_gb300 as P
    w = _weights(dtype)
    W = w.float().numpy()
    codes, scales, zeros = D.q4_quantize(W, group, symmetric)
    m, W_hat = P.crvq_q4_quantize(w.cuda(), group, symmetric, want_W_hat=True)
    P.crvq_sync()
    assert np.array_equal(U.exactly(m.scales), scales) and np.isfinite(scales).all()
    assert np.array_equal(D.unpack(m.codes.cpu().numpy(), 128), codes)
    V = D.q4_values(codes, scales, zeros, group)
    assert np.array_equal(U.exactly(W_hat), V.astype(np.float32)) and np.isfinite(U.exactly(W_hat)).all()
    # half a step, what the roundings of the scale and the zero point clip, and one step below the largest number
    s = scales[:, np.arange(128) // group].astype(np.float64)
    assert np.all(np.abs(V - W) <= s * ((0.5 + 8 * 2.0 ** -8 if symmetric else 0.5 + 0.5 + 15 * 2.0 ** -8) + 1.0))
    Y = P.crvq_q4_matvec(torch.eye(128, device="cuda")[:32], m)
    assert torch.equal(Y, W_hat[:, :32].t())
