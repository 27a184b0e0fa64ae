"""CPU checks of the calls around the cache (trees of drafted tokens, attention weights, selection, moving kept tokens): the
oracle's parts against independent restatements, the C structure, and refusals before anything reaches a GPU."""
import ctypes
import os

import numpy as np
import pytest
import torch

import test_abi_cpu as A
from oracle import cache_oracle as C
from oracle import decode_oracle as D


@pytest.fixture(scope="module")
def lib():
    from paper_2412_09282_gb300 import build
    build.build()
    from paper_2412_09282_gb300 import _lib
    return _lib.load()


# ---------------------------------------------------------------- oracle
def _parents(rng, n):
    return [int(rng.integers(-1, i)) for i in range(n)]


def test_masks_are_powers_of_the_parent_relation():
    rng = np.random.default_rng(0)
    counts = [1, 7, 0, 40]
    parents = sum((_parents(rng, n) for n in counts), [])
    mask, positions = C.tree_mask(np.asarray(parents), counts, 2, 0, [5, 9, 3, 60])
    at = 0
    for b, n in enumerate(counts):
        step = np.zeros((n, n), int)
        for i in range(n):
            if parents[at + i] >= 0:
                step[i, parents[at + i]] = 1
        reach = sum((np.linalg.matrix_power(step, k) for k in range(n + 1)), np.zeros((n, n), int))
        got = [[mask[at + i, j // 32] >> np.uint32(j % 32) & 1 for j in range(n)] for i in range(n)]
        assert np.array_equal(np.asarray(got).reshape(n, n), reach)
        assert np.array_equal(positions[at:at + n], [5, 9, 3, 60][b] - n + reach.sum(1) - 1)
        at += n
    short, _ = C.tree_mask(np.asarray(parents), counts, 2, 3)
    assert all(bin(int(a)).count("1") + bin(int(b)).count("1") <= 3 for a, b in short)


def _cache(rng, n, d=64, heads=2, page=16, fmt="int8"):
    pages = -(-n // page)
    top = 127 if fmt == "int8" else 448
    c = {k: D.to_codes(rng.uniform(-top, top, (pages, heads, page, d)), fmt) for k in ("K", "V")}
    c.update({k: rng.uniform(0.005, 0.02, (pages, heads, page // 16)).astype(np.float32) for k in ("k_scale", "v_scale")})
    return dict(c, pages=rng.permutation(pages)[None].astype(np.int32), lens=np.array([n], np.int32))


def test_a_chain_attends_as_causal_queries_do():
    rng = np.random.default_rng(1)
    c = _cache(rng, 50)
    q = rng.standard_normal((6, 4, 64)).astype(np.float32)
    for window in (0, 5):
        mask, pos = C.tree_mask(np.arange(-1, 5), [6], 1, window, c["lens"])
        a = C.tree_attention(c, q, [6], mask, 0.125, window, pos)
        b = D.attention(c, q, [6], 0.125, True, window)
        for x, y in zip(a, b):
            assert np.allclose(x, y, rtol=1e-12)


def test_siblings_do_not_see_each_other():
    """A star's tokens attend as single tokens behind the cache each do."""
    rng = np.random.default_rng(2)
    c = _cache(rng, 44)
    q = rng.standard_normal((4, 2, 64)).astype(np.float32)
    mask, _ = C.tree_mask(np.full(4, -1), [4], 1)
    out, lse, _, _ = C.tree_attention(c, q, [4], mask, 0.125)
    K, V = D.values(c, "K", 0, 0, 44), D.values(c, "V", 0, 0, 44)
    for i in range(4):
        t = np.r_[0:40, 40 + i]
        z = np.einsum("hd,thd->ht", q[i].astype(np.float64), K[t]) * 0.125
        p = np.exp(z - z.max(1, keepdims=True))
        assert np.allclose(out[i], np.einsum("ht,thd->hd", p / p.sum(1, keepdims=True), V[t]), rtol=1e-10)


def test_weights_are_the_softmax_summed_over_queries_and_heads():
    rng = np.random.default_rng(3)
    c = _cache(rng, 40)
    q = rng.standard_normal((3, 6, 64)).astype(np.float32)
    lse = D.attention(c, q, [3], 0.125, True, 9)[1]
    w, _ = C.token_weights(c, q, lse, [3], 0.125, True, 9, None, 1.0, 48)
    assert np.allclose(w.sum(2), 9.0) and (w[:, :, 40:] == 0).all() and (w[:, :, :29] == 0).all()
    before = rng.random((1, 2, 48)).astype(np.float32)
    w2, _ = C.token_weights(c, q, lse, [3], 0.125, True, 9, before, 0.5, 48)
    assert np.allclose(w2[:, :, :40], w[:, :, :40] + 0.5 * before[:, :, :40]) and (w2[:, :, 40:] == 0).all()


def test_selection_is_a_stable_sort():
    rng = np.random.default_rng(4)
    w = rng.integers(0, 4, (2, 3, 30)).astype(np.float32)
    idx, count, out = C.select(w, [30, 9], 12, 2, 3)
    assert count.tolist() == [12, 9]
    for h in range(3):
        assert idx[1, h, :9].tolist() == list(range(9)) and (idx[1, h, 9:] == -1).all()
        ranked = sorted(range(2, 27), key=lambda t: (-w[0, h, t], t))[:7]
        assert idx[0, h].tolist() == [0, 1] + sorted(ranked) + [27, 28, 29]
        assert np.array_equal(out[0, h, :12], w[0, h, idx[0, h]]) and (out[0, h, 12:] == 0).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_moved_values_are_within_half_a_step(fmt):
    """A value moved is off by half a step of its new scale at most (int8), half a step of e4m3 there; codes that keep their
    block's scale stay."""
    rng = np.random.default_rng(5)
    c = _cache(rng, 64, fmt=fmt)
    idx = np.sort(rng.permutation(64)[:37])[None].astype(np.int32)
    was = {n: D.values(c, n, 0, 0, 64)[idx[0]] for n in ("K", "V")}
    new = {k: v.copy() for k, v in c.items()}
    C.keep(c, idx, [37], [0], new, fmt)
    new["lens"] = np.array([37], np.int32)
    for n, s in (("K", "k_scale"), ("V", "v_scale")):
        got = D.values(new, n, 0, 0, 37)
        step = np.stack([new[s][new["pages"][0, r // 16], :, 0] for r in range(37)])[:, :, None].astype(np.float64)
        half = 0.5 * step if fmt == "int8" else np.maximum(np.abs(was[n]) * 2.0 ** -4, step * 2.0 ** -10)
        assert np.all(np.abs(got - was[n]) <= half * (1 + 1e-5))
    same = {k: v.copy() for k, v in c.items()}
    C.keep(c, np.arange(64, dtype=np.int32)[None], [64], [0], same, fmt)
    assert all(np.array_equal(same[k], c[k]) for k in c)


# ---------------------------------------------------------------- structure and refusals
def test_the_structure_matches_the_header_layout(tmp_path):
    import shutil
    import subprocess
    from paper_2412_09282_gb300 import _lib
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    fields = A._header_fields("crvq_token_sums")
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "crvq.h"', 'int main(void) {',
             '  printf("%zu\\n", sizeof(crvq_token_sums));']
    lines += [f'  printf("%zu\\n", offsetof(crvq_token_sums, {f}));' for f in fields]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(A.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    cls = _lib.crvq_token_sums
    assert [n for n, _ in cls._fields_] == fields
    assert got == [ctypes.sizeof(cls)] + [getattr(cls, n).offset for n, _ in cls._fields_]


def _a(s):
    return None if s is None else ctypes.addressof(s)


def _cache_struct(**kw):
    from paper_2412_09282_gb300 import _lib
    c = dict(K=16, V=16, k_scale=16, v_scale=16, pages=16, lens=16, n_pages=4, page_stride=2 * 32 * 64, ld_pages=2, n_seq=2,
             max_pages=2, page=32, n_kv=2, head_dim=64, format=0)
    c.update(kw)
    return _lib.crvq_kv_cache(**c)


def _heads_struct(**kw):
    from paper_2412_09282_gb300 import _lib
    return _lib.crvq_heads(**dict(dict(data=16, ld_tok=128, ld_head=64, heads=2, type=0), **kw))


def _sums_struct(**kw):
    from paper_2412_09282_gb300 import _lib
    return _lib.crvq_token_sums(**dict(dict(data=16, ld_seq=128, ld_head=64, width=64), **kw))


INVALID, UNSUPPORTED = -1, -2


def _mask(lib, parents=16, n=4, off=None, n_seq=2, lens=None, window=0, mask=16, words=1, positions=None):
    return lib.crvq_tree_mask(parents, n, off, n_seq, lens, window, mask, words, positions, None)


@pytest.mark.parametrize("change", [dict(parents=None), dict(mask=None), dict(n=-1), dict(n=3), dict(n_seq=0), dict(window=-1),
                                    dict(words=0), dict(words=(1 << 20) + 1), dict(parents=18), dict(positions=17), dict(lens=18),
                                    dict(off=18), {}])
def test_tree_mask_refusals(lib, change):
    assert _mask(lib, **change) == INVALID                       # ({}: host memory)
    assert lib.crvq_last_error()
    assert _mask(lib, n=0) == 0


def _tree(lib, c=None, q=None, n=2, off=None, mask=16, words=1, positions=None, scale=1.0, window=0, out=None, lse=None):
    return lib.crvq_cache_tree_attention(_a(c or _cache_struct()), _a(q or _heads_struct()), n, off, mask, words, positions, scale,
                                         window, _a(out or _heads_struct()), lse, None)


@pytest.mark.parametrize("change", [dict(mask=None), dict(mask=18), dict(words=0), dict(n=66), dict(n=3), dict(window=-1),
                                    dict(window=4), dict(scale=float("inf")), dict(scale=float("nan")), dict(lse=18), {}])
def test_tree_attention_refusals(lib, change):
    assert _tree(lib, **change) == INVALID
    assert _tree(lib, c=_cache_struct(K=24), **change) == INVALID
    assert _tree(lib, c=_cache_struct(head_dim=80), **change) == UNSUPPORTED


def _weights(lib, c=None, n=2, off=None, scale=1.0, window=0, lse=16, before=None, decay=1.0, out=0):
    return lib.crvq_cache_weights(_a(c or _cache_struct()), _a(_heads_struct()), n, off, scale, 1, window, lse, _a(before), decay,
                                  _a(_sums_struct() if out == 0 else out), None)


def test_weights_refusals(lib):
    for change in (dict(out=None), dict(out=_sums_struct(data=None)), dict(out=_sums_struct(data=18)), dict(out=_sums_struct(width=0)),
                   dict(out=_sums_struct(width=1 << 31)), dict(out=_sums_struct(ld_head=63)), dict(out=_sums_struct(ld_seq=127)),
                   dict(lse=None), dict(lse=18), dict(decay=float("nan")), dict(decay=float("inf")), dict(window=-1), dict(n=3), {}):
        assert _weights(lib, **change) == INVALID, change
        assert lib.crvq_last_error()
    assert _weights(lib, c=_cache_struct(head_dim=80)) == UNSUPPORTED


def _select(lib, w=0, lens=16, n_seq=2, n_kv=2, keep=8, first=0, recent=0, idx=16, count=16, out=None):
    return lib.crvq_cache_select(_a(_sums_struct() if w == 0 else w), lens, n_seq, n_kv, keep, first, recent, idx, count, _a(out), None)


def test_select_refusals(lib):
    for change in (dict(w=None), dict(w=_sums_struct(ld_head=8)), dict(lens=None), dict(lens=18), dict(n_seq=0), dict(n_kv=0),
                   dict(keep=0), dict(first=-1), dict(recent=-1), dict(first=5, recent=4), dict(first=1 << 30, recent=1 << 30),
                   dict(idx=None), dict(count=18), {}):
        assert _select(lib, **change) == INVALID, change
        assert lib.crvq_last_error()


def _keep(lib, c=None, idx=16, ld_seq=16, ld_head=8, most=8, count=16, start=None, out=None):
    return lib.crvq_cache_keep(_a(c or _cache_struct()), idx, ld_seq, ld_head, most, count, start, _a(out or _cache_struct()), None)


def test_keep_refusals(lib):
    for change in (dict(idx=18), dict(count=None), dict(count=18), dict(start=18), dict(most=-1), dict(ld_head=7),
                   dict(out=_cache_struct(n_seq=1)), dict(out=_cache_struct(n_kv=1)), dict(out=_cache_struct(format=1)),
                   dict(out=_cache_struct(head_dim=128, page_stride=2 * 32 * 128)), dict(c=_cache_struct(pages=None)), {}):
        assert _keep(lib, **change) == INVALID, change
        assert lib.crvq_last_error()
    assert _keep(lib, c=_cache_struct(head_dim=80)) == UNSUPPORTED


def test_the_binding_refuses_host_tensors():
    import paper_2412_09282_gb300 as P
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        P.crvq_tree_mask(i, 2)
    with pytest.raises(TypeError):
        P.crvq_cache_select(torch.zeros((1, 1, 4)), i[:1], 2)
    with pytest.raises(ValueError):
        P.crvq_cache_select(torch.zeros((1, 4)), i[:1], 2)
