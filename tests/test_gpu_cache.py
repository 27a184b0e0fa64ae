"""The paged 8-bit cache on the GPU: appending and reading, against the oracle.

Codes, scales and rotated queries are compared for equality: both sides round the same fp32 operations in
the same order. What the cache holds beside the appended tokens has to stay as it was.
"""
import numpy as np
import pytest
import torch

import decode_util as U
from oracle import decode_oracle as D

pytestmark = pytest.mark.gpu


def _tables(n_pos, half, seed=9):
    ang = np.random.default_rng(seed).uniform(0, 6.28, (n_pos, half))
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def _rows(rng, n, heads, d, dtype):
    """fp32 host values that `dtype` holds exactly."""
    x = torch.from_numpy((rng.standard_normal((n, heads, d)) * np.exp(rng.standard_normal((n, 1, 1)))).astype(np.float32))
    return x.to(U.TORCH[dtype]).float().numpy()


def _same_cache(gpu, host, lens_before, lens):
    """Every token's code and every held block's scale; nothing else changed."""
    for name, scales in (("K", "k_scale"), ("V", "v_scale")):
        got, ref = U.exactly(getattr(gpu, name)), host[name]
        assert np.array_equal(got, ref, equal_nan=True), name
        gs, rs = U.exactly(getattr(gpu, scales)), host[scales]
        assert np.array_equal(gs, rs, equal_nan=True), scales


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,page,n_kv,held,new", [
    (128, 64, 2, [0, 1, 15, 16, 17, 40], [1, 1, 1, 1, 1, 1]),      # single tokens, every place in a block
    (64, 16, 3, [5, 0, 31, 16], [27, 1, 2, 48]),                   # page ends, whole and part blocks
    (256, 48, 1, [0, 47, 10], [18, 17, 3]),                        # three blocks for 18 tokens from place 15 on
    (128, 32, 2, [15, 14], [18, 18]),
])
def test_append_ragged(fmt, dtype, d, page, n_kv, held, new):
    import paper_2412_09282_gb300 as P
    rng = np.random.default_rng(10)
    lens = [h + c for h, c in zip(held, new)]
    host, _ = U.make(11, held, page, n_kv, d, fmt, wide=-(-max(lens) // page) + 1, spare=len(lens) * 3)
    # room for the new tokens: pages that no sequence has yet
    used = {int(host["pages"][b][i]) for b, h in enumerate(held) for i in range(-(-h // page))}
    free = [p for p in range(host["K"].shape[0]) if p not in used]
    for b, (h, n) in enumerate(zip(held, lens)):
        for i in range(-(-h // page), -(-n // page)):
            host["pages"][b][i] = free.pop()
    host["lens"] = np.asarray(lens, np.int32)
    gpu = U.on_gpu(host, fmt, page_gap=1)
    n_tok, hq, half = sum(new), 2 * n_kv, d // 2
    k, v, q = _rows(rng, n_tok, n_kv, d, dtype), _rows(rng, n_tok, n_kv, d, dtype), _rows(rng, n_tok, hq, d, dtype)
    cos, sin = _tables(max(lens), half)
    pos = np.concatenate([np.arange(h, n) for h, n in zip(held, lens)])
    kr = D.rotate(k, cos[pos], sin[pos], False)
    D.append(host, {"K": kr, "V": v}, new, fmt)
    args = dict(new_off=U.offsets(new), cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda())
    kt, vt, qt = U.heads(k, dtype, 7), U.heads(v, dtype, 8), U.heads(q, dtype)
    out = P.crvq_cache_append(gpu, kt, vt, q=qt, **args)
    P.crvq_sync()
    _same_cache(gpu, host, held, lens)
    ref = torch.from_numpy(D.rotate(q, cos[pos], sin[pos], False)).to(U.TORCH[dtype]).float().numpy()
    assert np.array_equal(U.exactly(out), ref)
    # the same tokens again change nothing; queries in place
    P.crvq_cache_append(gpu, kt, vt, q=qt, q_out=qt, **args)
    P.crvq_sync()
    _same_cache(gpu, host, held, lens)
    assert np.array_equal(U.exactly(qt), ref)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("half", [3, 32, 64])
def test_append_rotation_forms_and_positions(interleaved, half):
    """Partial and whole rotations of both pairings, at given positions, with unaligned tables."""
    import paper_2412_09282_gb300 as P
    rng = np.random.default_rng(12)
    d, n_kv, new = 128, 2, 20
    host, _ = U.make(13, [7, 7], 64, n_kv, d, "int8")
    host["lens"] = np.array([27, 27], np.int32)
    gpu = U.on_gpu(host, "int8")
    k, v, q = (_rows(rng, 2 * new, h, d, "f32") for h in (n_kv, n_kv, 3))
    cos, sin = _tables(50, half)
    pos = rng.integers(0, 50, 2 * new).astype(np.int32)
    D.append(host, {"K": D.rotate(k, cos[pos], sin[pos], interleaved), "V": v}, [new, new], "int8")
    tab = [torch.zeros((50, half + 1), device="cuda")[:, 1:] for _ in range(2)]
    tab[0].copy_(torch.from_numpy(cos))
    tab[1].copy_(torch.from_numpy(sin))
    qt = U.heads(q, "f32")
    P.crvq_cache_append(gpu, U.heads(k, "f32"), U.heads(v, "f32"), cos=tab[0], sin=tab[1],
                        positions=torch.from_numpy(pos).cuda(), interleaved=interleaved, q=qt, q_out=qt)
    P.crvq_sync()
    _same_cache(gpu, host, None, None)
    assert np.array_equal(U.exactly(qt), D.rotate(q, cos[pos], sin[pos], interleaved))


def test_append_without_rotation_zeros_and_tiny_values():
    import paper_2412_09282_gb300 as P
    for fmt in ("int8", "e4m3"):
        host, _ = U.make(14, [0, 3], 16, 1, 64, fmt, spare=4)
        host["pages"][0][0] = [p for p in range(5) if p != host["pages"][1][0]][0]
        host["lens"] = np.array([2, 5], np.int32)
        gpu = U.on_gpu(host, fmt)
        k = np.zeros((4, 1, 64), np.float32)
        v = np.zeros((4, 1, 64), np.float32)
        v[1, 0, 5], v[3, 0, 6] = 1e-44, -3e38
        D.append(host, {"K": k, "V": v}, [2, 2], fmt)
        P.crvq_cache_append(gpu, U.heads(k, "f32"), U.heads(v, "f32"))
        P.crvq_sync()
        _same_cache(gpu, host, None, None)


def test_append_reports_and_skips_what_is_not_finite_or_out_of_range():
    import paper_2412_09282_gb300 as P
    k = np.ones((2, 1, 64), np.float32)

    def case():
        host, _ = U.make(15, [4, 4], 16, 1, 64, "int8")
        host["lens"] = np.array([5, 5], np.int32)
        return host

    host = case()
    gpu = U.on_gpu(host, "int8")
    bad = k.copy()
    bad[0, 0, 3], bad[1, 0, 4] = np.nan, np.inf
    D.append(host, {"K": bad, "V": k}, [1, 1], "int8")
    P.crvq_cache_append(gpu, U.heads(bad, "f32"), U.heads(k, "f32"))
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -6
    _same_cache(gpu, host, None, None)
    for change in (lambda h: h["pages"].__setitem__((0, 0), 99), lambda h: h["pages"].__setitem__((0, 0), -1),
                   lambda h: h["lens"].__setitem__(0, 17), lambda h: h["lens"].__setitem__(0, -1),
                   lambda h: h["lens"].__setitem__(0, 0)):
        host = case()
        change(host)
        gpu = U.on_gpu(host, "int8")
        keep = {n: host[n].copy() for n in ("K", "V", "k_scale", "v_scale")}
        P.crvq_cache_append(gpu, U.heads(k, "f32"), U.heads(k, "f32"))
        with pytest.raises(P.CrvqError) as e:
            P.crvq_sync()
        assert e.value.status == -7
        # the other sequence is appended, nothing else is touched
        one = dict(host, pages=host["pages"][1:], lens=host["lens"][1:])
        D.append(one, {"K": k[1:], "V": k[1:]}, [1], "int8")
        for n in keep:
            assert np.array_equal(U.exactly(getattr(gpu, n)), one[n], equal_nan=True)
    # positions outside the tables, offsets that are not in order
    gpu = U.on_gpu(case(), "int8")
    tab = torch.ones((3, 32), device="cuda")
    P.crvq_cache_append(gpu, U.heads(k, "f32"), U.heads(k, "f32"), cos=tab, sin=tab)
    with pytest.raises(P.CrvqError):
        P.crvq_sync()
    gpu = U.on_gpu(case(), "int8")
    P.crvq_cache_append(gpu, U.heads(k, "f32"), U.heads(k, "f32"),
                        new_off=torch.tensor([0, 5, 2], dtype=torch.int32, device="cuda"))
    with pytest.raises(P.CrvqError):
        P.crvq_sync()
    P.crvq_sync()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_read_ranges(fmt, dtype):
    import paper_2412_09282_gb300 as P
    lens = [33, 1, 0, 100]
    host, gpu = U.make(16, lens, 32, 3, 64, fmt, page_gap=2)
    start, count = [5, 0, 0, 17], [28, 1, 0, 60]
    K, V = P.crvq_cache_read(gpu, torch.tensor(start, dtype=torch.int32).cuda(), U.offsets(count), sum(count),
                             dtype=U.TORCH[dtype])
    P.crvq_sync()
    for got, name in ((K, "K"), (V, "V")):
        ref = np.concatenate([D.values(host, name, b, s, s + c) for b, (s, c) in enumerate(zip(start, count))])
        ref = torch.from_numpy(ref.astype(np.float32)).to(U.TORCH[dtype]).float().numpy()  # one rounding of code x scale
        assert np.array_equal(U.exactly(got), ref)
    # past a sequence's end: zeros and a report
    K, _ = P.crvq_cache_read(gpu, torch.tensor([30, 0, 0, 0], dtype=torch.int32).cuda(), U.offsets([5, 0, 0, 0]), 5)
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -7
    assert bool((K[3:] == 0).all()) and bool((K[:3] != 0).any())


def test_append_refusals_and_streams():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(17, [4, 4], 16, 2, 64, "int8")
    k = torch.ones((2, 2, 64), device="cuda")
    with pytest.raises(P.CrvqError) as e:                      # 3 heads
        P.crvq_cache_append(gpu, torch.ones((2, 3, 64), device="cuda"), k)
    assert e.value.status == -1
    with pytest.raises(P.CrvqError) as e:                      # 3 tokens for 2 sequences
        P.crvq_cache_append(gpu, torch.ones((3, 2, 64), device="cuda"), torch.ones((3, 2, 64), device="cuda"))
    assert e.value.status == -1
    with pytest.raises(ValueError):
        P.crvq_cache_append(gpu, k, torch.ones((4, 2, 64), device="cuda"))
    with pytest.raises(ValueError):
        P.crvq_cache_append(gpu, torch.ones((2, 2, 32), device="cuda"), k)
    with pytest.raises(P.CrvqError):                           # more rotated channels than there are
        P.crvq_cache_append(gpu, k, k, cos=torch.ones((9, 33), device="cuda"), sin=torch.ones((9, 33), device="cuda"))
    P.crvq_cache_append(gpu, k[:0], k[:0], new_off=torch.zeros(3, dtype=torch.int32, device="cuda"))  # nothing to do
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        P.crvq_cache_append(gpu, k, k)
        K, _ = P.crvq_cache_read(gpu, torch.tensor([3, 3], dtype=torch.int32, device="cuda"), U.offsets([1, 1]), 2)
    P.crvq_sync(stream=s)
    assert np.allclose(U.exactly(K), 1.0, atol=float(gpu.k_scale[host["pages"][:, 0]].max()) / 2)


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB: the last pages are appended to and read."""
    import paper_2412_09282_gb300 as P
    n_pages, page, n_kv, d = 5000, 256, 32, 128                # 1 MiB a page
    pages = torch.tensor([[n_pages - 1], [4097]], dtype=torch.int32, device="cuda")
    gpu = P.KVCache.empty(n_pages, n_kv, page, d, pages, torch.tensor([20, 256], dtype=torch.int32, device="cuda"))
    rng = np.random.default_rng(18)
    k, v = (rng.standard_normal((276, n_kv, d)).astype(np.float32) for _ in range(2))
    off = U.offsets([20, 256])
    P.crvq_cache_append(gpu, U.heads(k, "f32"), U.heads(v, "f32"), new_off=off)
    K, V = P.crvq_cache_read(gpu, torch.zeros(2, dtype=torch.int32, device="cuda"), off, 276)
    q = rng.standard_normal((2, n_kv, d)).astype(np.float32)
    out = P.crvq_cache_attention(gpu, U.heads(q, "f32"))
    P.crvq_sync()
    assert np.abs(U.exactly(K) - k).max() <= 0.5 * 6 / 127 and np.abs(U.exactly(V) - v).max() <= 0.5 * 6 / 127
    for b, rows in ((0, slice(0, 20)), (1, slice(20, 276))):
        z = np.einsum("hd,nhd->hn", q[b].astype(np.float64), U.exactly(K)[rows].astype(np.float64)) / np.sqrt(d)
        p = np.exp(z - z.max(1, keepdims=True))
        ref = np.einsum("hn,nhd->hd", p / p.sum(1, keepdims=True), U.exactly(V)[rows].astype(np.float64))
        assert np.abs(U.exactly(out)[b] - ref).max() <= 1e-5


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_wide_ranges(fmt):
    """Blocks whose scales run from subnormal to 2^110 (quotients by corrected products and by division), new and
    joined by larger and smaller values of a later call: equal to the oracle's codes and scales."""
    import paper_2412_09282_gb300 as P
    rng = np.random.default_rng(60)
    exps = [-140, -126, -110, -80, -74, -72, -71, -40, 0, 50, 84, 86, 87, 88, 89, 110]
    host, _ = U.make(61, [0] * 16, 16, 1, 64, fmt, wide=1, spare=16)
    host["pages"] = np.arange(16, dtype=np.int32)[:, None].copy()
    host["lens"] = np.full(16, 9, np.int32)
    gpu = U.on_gpu(host, fmt)
    for step, (n, by) in enumerate(((9, 0), (3, 6), (2, -9))):
        if step:
            host["lens"] = host["lens"] + np.int32(n)
            gpu.lens.add_(n)
        x = {name: np.ldexp(rng.standard_normal((16 * n, 1, 64)), np.repeat(exps, n)[:, None, None] + by).astype(np.float32)
             for name in ("K", "V")}
        D.append(host, x, [n] * 16, fmt)
        P.crvq_cache_append(gpu, U.heads(x["K"], "f32"), U.heads(x["V"], "f32"))
        P.crvq_sync()
        _same_cache(gpu, host, None, None)


@pytest.mark.parametrize("n_seq", [33, 70, 1100])
def test_append_many_sequences(n_seq):
    """More sequences than a warp's lanes, and than offsets fit beside the kernel's data; many without new tokens."""
    rng = np.random.default_rng(62)
    held, new = rng.integers(0, 40, n_seq).tolist(), rng.choice([0, 0, 1, 1, 2, 19], n_seq).tolist()
    test_append_ragged("int8", "bf16", 64, 16, 1, held, new)
