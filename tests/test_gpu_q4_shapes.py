"""4-bit products of matrices that take the kernel's longer ways: several row tiles per CTA, inputs laid out in several
chunks, clusters, and tiles in several groups; against fp64.

Bars. fp16 inputs are exact operands. bf16 inputs are relative to their group's power of two in one fp16 operand: off by
2^-25 of the group's largest where that is subnormal. fp32 inputs are two such operands: off by 2^-22 of the element besides.
With S = sum |w x| and T the same with every |x| its group's largest,
  |y - ref| <= r |ref| + (2^-22 S + ) 2^-25 T + (additions) 2^-23 S,
r the output's unit roundoff; additions: 128 terms of a group, twice for two pieces, N / group groups, 16 for slices and 24 for
warps in order (a tensor core's may truncate). And in root mean square over the outputs of an input: a group's sum is
16 products of operands in order, each of which may truncate by 2^-23 of what it adds to, so 2^-19 of it, and groups do not
conspire: 2^-18 of the outputs' root mean square and, for 16-bit types, 1.05 times the outputs' own rounding (lost low pieces would be 2^-13).
"""
import pytest
import torch

import decode_util as U

pytestmark = pytest.mark.gpu


def _matrix(M, N, group, zeros):
    import paper_2412_09282_gb300 as P
    g = torch.Generator(device="cuda").manual_seed(92)
    half, G = (N + 1) // 2, -(-N // group)
    row = -(-half // 16) * 16
    codes = torch.randint(0, 256, (M, row), generator=g, device="cuda", dtype=torch.uint8)[:, :half]
    scales = (0.01 * torch.exp(torch.randn((M, G), generator=g, device="cuda"))).to(torch.bfloat16)
    z = torch.randint(0, 16, (M, G), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    return P.Q4Matrix(codes, scales, z, N, group)


def _values(m, r0, r1):
    """Rows r0 .. r1 of the matrix in fp64."""
    c = m.codes[r0:r1]
    q = torch.stack([c & 15, c >> 4], -1).flatten(1)[:, :m.N].double()
    at = torch.arange(m.N, device="cuda") // m.group
    z = 8.0 if m.zeros is None else m.zeros[r0:r1].double()[:, at]
    return (q - z) * m.scales[r0:r1].double()[:, at]


@pytest.mark.parametrize("M,N,group,zeros,b,dtype", [
    (11003, 4096, 128, False, 1, "bf16"),     # several tiles per CTA, a part tile at the end
    (11003, 4096, 64, True, 5, "f32"),
    (11003, 4090, 32, True, 8, "f16"),
    (3000, 11150, 128, False, 32, "f32"),     # several chunks
    (28672, 8192, 64, True, 32, "f32"),       # tiles, chunks and clusters
    (28672, 8192, 128, True, 16, "f16"),
    (512, 28672, 128, False, 2, "bf16"),      # few tiles, many steps
    (238412, 1042, 128, True, 17, "f32"),     # tiles in several groups, several chunks in each
    (238412, 1042, 32, False, 3, "bf16"),
    (60000, 4096, 64, False, 17, "bf16"),     # groups and clusters
    (120000, 4090, 128, True, 8, "f32"),
])
def test_long_ways(M, N, group, zeros, b, dtype):
    import paper_2412_09282_gb300 as P
    m = _matrix(M, N, group, zeros)
    g = torch.Generator(device="cuda").manual_seed(93)
    X = torch.randn((b, N), generator=g, device="cuda").to(U.TORCH[dtype])
    Y = P.crvq_q4_matvec(X, m)
    again = P.crvq_q4_matvec(X, m)
    P.crvq_sync()
    assert torch.equal(Y, again)
    x = X.double()
    G = -(-N // group)
    tops = torch.nn.functional.pad(x.abs(), (0, G * group - N)).view(b, G, group).amax(2)
    tops = tops.repeat_interleave(group, 1)[:, :N]
    adds = (256 if dtype == "f32" else 128) + G + 40
    parts = []
    for r0 in range(0, M, 4096):
        W = _values(m, r0, min(M, r0 + 4096))
        ref, S, T = x @ W.t(), x.abs() @ W.abs().t(), tops @ W.abs().t()
        err = Y[:, r0:r0 + 4096].double() - ref
        bound = U.OUT_ROUND[dtype] * ref.abs() + adds * 2.0 ** -23 * S + 1e-30
        if dtype != "f16":
            bound += 2.0 ** -25 * T
        if dtype == "f32":
            bound += 2.0 ** -22 * S
        assert bool((err.abs() <= bound).all()), (r0, float((err.abs() / bound).max()))
        parts.append(torch.stack([(err ** 2).sum(1), (ref ** 2).sum(1), ((ref.to(Y.dtype).double() - ref) ** 2).sum(1)]))
    err, size, rounding = (v.sqrt() for v in torch.stack(parts).sum(0))
    most = 2.0 ** -18 * size + (1.05 * rounding if dtype != "f32" else 0.0)
    assert bool((err <= most).all()), float((err / most).max())
