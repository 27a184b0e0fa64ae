"""CPU checks of the decode-step calls: the oracle's parts against independent restatements, the C
structures, and refusals before anything reaches a GPU."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

import test_abi_cpu as A
from oracle import decode_oracle as D

STRUCTS = ["crvq_heads", "crvq_kv_cache", "crvq_rotary", "crvq_q4_matrix"]


@pytest.fixture(scope="module")
def lib():
    from paper_2412_09282_gb300 import build
    build.build()
    from paper_2412_09282_gb300 import _lib
    return _lib.load()


def test_e4m3_rounding_equals_torchs_conversion():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * np.exp2(rng.integers(-12, 9, 4000)),
                        np.arange(-480, 480) * 0.5, np.arange(-64, 64) * 2.0 ** -11, [0.0, -0.0, 448.0, 1e30]])
    x = x.astype(np.float32)
    ref = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(D.e4m3(x), ref)


def test_bf16_rounding_equals_torchs_conversion():
    x = np.random.default_rng(1).standard_normal(5000).astype(np.float32)
    assert np.array_equal(D.bf16(x), torch.from_numpy(x).to(torch.bfloat16).float().numpy())


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((3, 2, 64)).astype(np.float32)
    ang = rng.uniform(0, 6, (3, 20))
    y = D.rotate(x, np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32), interleaved)
    if interleaved:
        z = x[..., 0:40:2] + 1j * x[..., 1:40:2]
        w = y[..., 0:40:2] + 1j * y[..., 1:40:2]
    else:
        z, w = x[..., :20] + 1j * x[..., 20:40], y[..., :20] + 1j * y[..., 20:40]
    assert np.allclose(w, z * np.exp(1j * ang)[:, None, :], atol=1e-6)
    assert np.array_equal(y[..., 40:], x[..., 40:])


def test_append_keeps_values_within_half_a_step_of_each_rounding():
    """Tokens appended one by one: a value is rounded once when it comes and once each time its block's
    scale grows, each time by half a step at most."""
    rng = np.random.default_rng(3)
    d, page = 64, 16
    x = rng.standard_normal((16, 1, d)).astype(np.float32) * np.linspace(0.5, 3, 16)[:, None, None].astype(np.float32)
    c = {"K": np.zeros((1, 1, page, d), np.float32), "V": np.zeros((1, 1, page, d), np.float32),
         "k_scale": np.full((1, 1, 1), np.nan, np.float32), "v_scale": np.full((1, 1, 1), np.nan, np.float32),
         "pages": np.zeros((1, 1), np.int32), "lens": np.zeros(1, np.int32)}
    bound = np.zeros(16)
    last = 0.0
    for i in range(16):
        c["lens"][0] = i + 1
        D.append(c, {"K": x[i:i + 1], "V": x[i:i + 1]}, [1], "int8")
        s = float(c["k_scale"][0, 0, 0])
        bound[:i + 1 if s != last else 0] += 0.5 * s
        bound[i] = 0.5 * s
        last = s
        err = np.abs(D.values(c, "K", 0, 0, i + 1)[:, 0] - x[:i + 1, 0]).max(1)
        assert np.all(err <= bound[:i + 1] * (1 + 1e-5))
    assert np.array_equal(c["K"], c["V"])


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 5), (False, 0), (False, 7)])
def test_attention_oracle_against_a_dense_softmax(causal, window):
    rng = np.random.default_rng(4)
    n, m, d = 40, 6, 64
    c = {"K": rng.integers(-127, 128, (3, 2, 16, d)).astype(np.float32),
         "V": rng.integers(-127, 128, (3, 2, 16, d)).astype(np.float32),
         "k_scale": rng.uniform(0.01, 0.02, (3, 2, 1)).astype(np.float32),
         "v_scale": rng.uniform(0.01, 0.02, (3, 2, 1)).astype(np.float32),
         "pages": np.array([[2, 0, 1]], np.int32), "lens": np.array([n], np.int32)}
    q = rng.standard_normal((m, 4, d)).astype(np.float32)
    out, lse, _, _ = D.attention(c, q, [m], 0.125, causal, window)
    K = torch.from_numpy(D.values(c, "K", 0, 0, n)).repeat_interleave(2, 1)
    V = torch.from_numpy(D.values(c, "V", 0, 0, n)).repeat_interleave(2, 1)
    z = torch.einsum("mhd,nhd->hmn", torch.from_numpy(q).double(), K) * 0.125
    t, pos = torch.arange(n), torch.arange(n - m, n)[:, None]
    seen = (t <= pos) if causal else torch.ones(m, n, dtype=torch.bool)
    if window:
        seen = seen & (t > pos - window)
    z = z.masked_fill(~seen, -math.inf)
    ref = torch.einsum("hmn,nhd->mhd", z.softmax(-1), V)
    assert np.allclose(out, ref.numpy(), rtol=1e-12, atol=1e-12)
    assert np.allclose(lse, z.logsumexp(-1).t().numpy(), rtol=1e-12)


def test_attention_oracle_rows_without_keys_are_zero():
    c = {"K": np.zeros((1, 1, 16, 64), np.float32), "V": np.ones((1, 1, 16, 64), np.float32),
         "k_scale": np.ones((1, 1, 1), np.float32), "v_scale": np.ones((1, 1, 1), np.float32),
         "pages": np.zeros((2, 1), np.int32), "lens": np.array([0, 2], np.int32)}
    out, lse, _, _ = D.attention(c, np.ones((5, 1, 64), np.float32), [1, 4], 1.0)
    assert np.array_equal(out[:, 0, 0], [0, 0, 0, 1, 1])
    assert np.array_equal(lse[:3, 0], [-np.inf] * 3)


@pytest.mark.parametrize("symmetric", [True, False])
def test_q4_oracle_rounds_to_the_nearest_level(symmetric):
    rng = np.random.default_rng(5)
    W = rng.standard_normal((7, 75)).astype(np.float32) * 0.02
    W[3, 10:40] = np.abs(W[3, 10:40])
    W[5, :32] = 0
    codes, scales, zeros = D.q4_quantize(W, 32, symmetric)
    V = D.q4_values(codes, scales, zeros, 32)
    s = scales[:, np.arange(75) // 32].astype(np.float64)
    # half a step, and what the scale's rounding to bf16 or the zero point's to a whole step clips
    assert np.all(np.abs(V - W) <= s * (0.5 + 8 * 2.0 ** -8 if symmetric else 0.5 + 0.5 + 15 * 2.0 ** -8))
    assert np.array_equal(D.unpack(D.pack(codes), 75), codes)
    assert np.all(V[5, :32] == 0)


def test_structures_match_the_header_layout(tmp_path):
    import shutil
    import subprocess
    from paper_2412_09282_gb300 import _lib
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "crvq.h"', 'int main(void) {']
    for s in STRUCTS:
        lines.append(f'  printf("{s} size %zu\\n", sizeof({s}));')
        lines += [f'  printf("{s} {f} %zu\\n", offsetof({s}, {f}));' for f in A._header_fields(s)]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(A.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
    got = {tuple(line.split()[:-1]): int(line.split()[-1]) for line in out.splitlines()}
    for s in STRUCTS:
        cls = getattr(_lib, s)
        assert [n for n, _ in cls._fields_] == A._header_fields(s), s
        assert ctypes.sizeof(cls) == got[(s, "size")], s
        for n, _ in cls._fields_:
            assert getattr(cls, n).offset == got[(s, n)], (s, n)


def _structs(**kw):
    from paper_2412_09282_gb300 import _lib
    c = dict(K=16, V=16, k_scale=16, v_scale=16, pages=16, lens=16, n_pages=4, page_stride=2 * 32 * 64,
             ld_pages=2, n_seq=2, max_pages=2, page=32, n_kv=2, head_dim=64, format=0)
    h = dict(data=16, ld_tok=128, ld_head=64, heads=2, type=0)
    q = dict(codes=16, scales=16, zeros=None, M=4, N=64, ld_codes=32, ld_scales=1, group=64, _pad=0)
    for d in (c, h, q):
        d.update({k: v for k, v in kw.items() if k in d})
    return _lib.crvq_kv_cache(**c), _lib.crvq_heads(**h), _lib.crvq_q4_matrix(**q)


def _a(s):
    return None if s is None else ctypes.addressof(s)


INVALID, UNSUPPORTED = -1, -2


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(K=None)), (INVALID, dict(lens=None)), (INVALID, dict(K=24)), (INVALID, dict(n_seq=0)),
    (INVALID, dict(n_pages=0)), (INVALID, dict(page=24)), (INVALID, dict(page=0)), (INVALID, dict(format=2)),
    (INVALID, dict(page_stride=2 * 32 * 64 - 16)), (INVALID, dict(page_stride=2 * 32 * 64 + 8)),
    (INVALID, dict(ld_pages=1)), (INVALID, dict(max_pages=1 << 27, ld_pages=1 << 27)),
    (UNSUPPORTED, dict(head_dim=80)), (UNSUPPORTED, dict(head_dim=0)),
])
def test_cache_refusals(lib, want, change):
    c, h, _ = _structs(**change)
    assert lib.crvq_cache_append(_a(c), _a(h), _a(h), 2, None, None, None, None, None) == want
    assert lib.crvq_cache_read(_a(c), 16, 16, 2, 0, 16, 16, None) == want
    assert lib.crvq_cache_attention(_a(c), _a(h), 2, None, 1.0, 1, 0, _a(h), None, None) == want
    assert lib.crvq_last_error()


def test_host_memory_is_refused(lib):
    c, h, m = _structs()
    assert lib.crvq_cache_append(_a(c), _a(h), _a(h), 2, None, None, None, None, None) == INVALID
    assert b"not device memory" in lib.crvq_last_error()
    assert lib.crvq_cache_attention(_a(c), _a(h), 2, None, 1.0, 1, 0, _a(h), None, None) == INVALID
    assert b"not device memory" in lib.crvq_last_error()
    assert lib.crvq_q4_matvec(_a(m), 16, 64, 1, 0, 16, 4, None) == INVALID
    assert b"not device memory" in lib.crvq_last_error()
    assert lib.crvq_q4_quantize(16, 64, 0, _a(m), None, None) == INVALID
    assert lib.crvq_cache_append(None, _a(h), _a(h), 2, None, None, None, None, None) == INVALID


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(codes=None)), (INVALID, dict(scales=None)), (INVALID, dict(M=0)), (INVALID, dict(N=0)),
    (UNSUPPORTED, dict(group=48)), (INVALID, dict(ld_codes=31)), (INVALID, dict(N=65)), (INVALID, dict(scales=17)),
])
def test_q4_refusals(lib, want, change):
    _, _, m = _structs(**change)
    assert lib.crvq_q4_matvec(_a(m), 16, 128, 1, 0, 16, 16, None) == want
    assert lib.crvq_q4_quantize(16, 128, 0, _a(m), None, None) == want


def test_binding_refuses_host_tensors_and_wrong_layouts():
    import paper_2412_09282_gb300 as P
    K = torch.zeros((2, 2, 16, 64), dtype=torch.int8)
    s = torch.zeros((2, 2, 1))
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        P.KVCache(K, K, s, s, i.view(1, 1), i)
    with pytest.raises(TypeError):
        P.KVCache(K.float(), K.float(), s, s, i.view(1, 1), i)
    with pytest.raises(TypeError):
        P.Q4Matrix(torch.zeros((2, 32), dtype=torch.uint8), torch.zeros((2, 1), dtype=torch.bfloat16), None, 64, 64)
    with pytest.raises(TypeError):
        P.crvq_q4_quantize(torch.zeros((2, 64)))
    with pytest.raises(TypeError):
        P.crvq_q4_quantize(torch.zeros((2, 64), dtype=torch.float64))
