"""Trees of drafted tokens over the paged 8-bit cache, against the fp64 oracle.

Masks and positions are whole numbers: equal. Attention's bar is that of test_gpu_attention.py: the products, weights and
sums are the same, only which keys count differs.
"""
import math

import numpy as np
import pytest
import torch

import decode_util as U
from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def _bits(x):
    return torch.from_numpy(np.ascontiguousarray(x).view(np.int32)).cuda()


def _parents(seed, counts, kind="random"):
    rng = np.random.default_rng(seed)
    out = []
    for n in counts:
        if kind == "chain":
            out += list(range(-1, n - 1))
        elif kind == "star":
            out += [-1] * n
        else:
            out += [int(max(-1, i - 1 - rng.integers(0, 4))) if rng.random() < 0.8 else int(rng.integers(-1, i)) for i in range(n)]
    return np.asarray(out, np.int32)


def _queries(seed, n, heads, d, dtype, size=1.0):
    x = np.random.default_rng(seed).standard_normal((n, heads, d)).astype(np.float32) * np.float32(size)
    return torch.from_numpy(x).to(U.TORCH[dtype]).float().numpy()


def _check(host, gpu, q, counts, mask, dtype, ragged=True, positions=None, window=0, gap=0, least=0.0):
    import paper_2412_09282_gb300 as P
    d = q.shape[2]
    scale = 1.0 / math.sqrt(d)
    ref, lse_ref, mass, shake = C.tree_attention(host, q, counts, mask, float(np.float32(scale)), window, positions)
    out, lse = P.crvq_cache_tree_attention(gpu, U.heads(q, dtype, gap), _bits(mask), window=window, want_lse=True,
                                           q_off=U.offsets(counts) if ragged else None,
                                           positions=None if positions is None else _ints(positions))
    P.crvq_sync()
    n = int(max(host["lens"]))
    per = 2.0 ** -23 + (2.0 ** -21 / (d + 16) if dtype == "f32" else 0.0)
    rel = 2 * U.WEIGHT_ROUND[dtype] + 2.0 ** -21 * n / 16 + 4 * per * shake[..., None] + 2.0 ** -19
    bound = U.OUT_ROUND[dtype] * np.abs(ref) + rel * mass + n * least * mass.max(-1, keepdims=True) + \
        (2.0 ** -25 if dtype == "f16" else 1e-30)
    got = U.exactly(out).astype(np.float64)
    empty = ~np.isfinite(lse_ref)
    assert np.all(np.abs(got - ref) <= bound), float((np.abs(got - ref) / bound).max())
    assert np.all(got[empty] == 0)
    gl = U.exactly(lse).astype(np.float64)
    assert np.array_equal(np.isneginf(gl), empty)
    tol = 2 * per * shake + 2.0 ** -20 + 2.0 ** -20 * n / 16 + 2.0 ** -22 * np.abs(np.where(empty, 0, lse_ref))
    assert np.all(np.abs(gl[~empty] - lse_ref[~empty]) <= tol[~empty])
    return out


@pytest.mark.parametrize("window", [0, 1, 3])
@pytest.mark.parametrize("kind", ["random", "chain", "star"])
@pytest.mark.parametrize("counts", [[1], [5, 0, 33, 64, 1], [200, 7], [31] * 40])
def test_masks_and_positions(counts, kind, window):
    import paper_2412_09282_gb300 as P
    parents = _parents(1, counts, kind)
    lens = np.asarray([n + 3 * b for b, n in enumerate(counts)], np.int32)
    words = -(-max(counts) // 32)
    ref, pos = C.tree_mask(parents, counts, words, window, lens)
    mask, positions = P.crvq_tree_mask(_ints(parents), len(counts), off=U.offsets(counts), lens=_ints(lens),
                                       max_new=max(counts), window=window)
    P.crvq_sync()
    assert np.array_equal(mask.cpu().numpy().view(np.uint32), ref)
    assert np.array_equal(positions.cpu().numpy(), pos)
    if len(set(counts)) == 1:                                  # the same without offsets; positions from 0
        mask, positions = P.crvq_tree_mask(_ints(parents), len(counts), window=window)
        P.crvq_sync()
        assert np.array_equal(mask.cpu().numpy().view(np.uint32), ref)
        assert np.array_equal(positions.cpu().numpy(), pos - np.repeat(lens - counts, counts))


@pytest.mark.parametrize("kind", ["random", "chain"])
def test_a_mask_of_thousands_of_tokens(kind):
    """More parents than lie in shared memory, paths as deep as the tree."""
    import paper_2412_09282_gb300 as P
    n = 4500
    parents = _parents(2, [n], kind)
    ref, pos = C.tree_mask(parents, [n], -(-n // 32))
    mask, positions = P.crvq_tree_mask(_ints(parents), 1)
    P.crvq_sync()
    assert np.array_equal(mask.cpu().numpy().view(np.uint32), ref)
    assert np.array_equal(positions.cpu().numpy(), pos)


def test_bad_parents_are_reported_and_count_as_roots():
    import paper_2412_09282_gb300 as P
    parents = np.asarray([-1, 0, 2, 7, -5, 3, 4], np.int32)     # 2 of itself, 7 behind its child, -5
    mask, _ = P.crvq_tree_mask(_ints(parents), 1)
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -7
    ref, _ = C.tree_mask(parents, [7], 1)
    assert np.array_equal(mask.cpu().numpy().view(np.uint32), ref)
    out = torch.full((3, 1), 99, dtype=torch.int32, device="cuda")
    P.crvq_tree_mask(_ints([-1, 0, 1]), 2, off=torch.tensor([0, 4, 2], dtype=torch.int32, device="cuda"), max_new=3,
                     mask_out=out)                              # offsets that are not in order: nothing is written
    with pytest.raises(P.CrvqError):
        P.crvq_sync()
    assert (out == 99).all()
    # 40 tokens in words for 32: the others' bits are nowhere
    parents = _parents(3, [40], "chain")
    mask, _ = P.crvq_tree_mask(_ints(parents), 1, off=U.offsets([40]), max_new=32)
    with pytest.raises(P.CrvqError):
        P.crvq_sync()
    assert np.array_equal(mask.cpu().numpy().view(np.uint32), C.tree_mask(parents, [40], 1)[0])
    P.crvq_sync()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,page,n_kv,group,lens,counts", [
    (128, 64, 2, 8, [300, 129, 16], [16, 16, 16]),             # (16-bit types: tiles of 128 rows)
    (64, 16, 3, 1, [40, 17, 65, 5, 130], [7, 0, 33, 9, 2]),     # more drafted tokens than places (9 of 5); none
    (256, 48, 1, 4, [1, 100, 63], [1, 5, 12]),
    (128, 16, 1, 1, [1500, 16], [3, 16]),                       # a unit in several shares, a tree that is all there is
])
def test_trees(fmt, dtype, d, page, n_kv, group, lens, counts):
    host, gpu = U.make(10, lens, page, n_kv, d, fmt, page_gap=1)
    q = _queries(11, sum(counts), n_kv * group, d, dtype, 2.0)
    mask, _ = C.tree_mask(_parents(12, counts), counts, -(-max(counts) // 32))
    _check(host, gpu, q, counts, mask, dtype, gap=5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 4, 20, 200])
@pytest.mark.parametrize("d,group,lens,counts", [
    (128, 4, [40, 70, 7], [3, 9, 9]),
    (64, 8, [400, 90], [64, 40]),
    (64, 1, [3000, 20], [6, 2]),
])
def test_windows_go_by_positions(dtype, window, d, group, lens, counts):
    host, gpu = U.make(13, lens, 32, 2, d, "int8")
    q = _queries(14, sum(counts), 2 * group, d, dtype)
    mask, pos = C.tree_mask(_parents(15, counts), counts, -(-max(counts) // 32), window, lens)
    _check(host, gpu, q, counts, mask, dtype, positions=pos, window=window)
    # positions of the caller's own, out of order and out of range: the nearest place counts
    pos = np.random.default_rng(16).integers(-5, max(lens) + 9, len(pos)).astype(np.int32)
    _check(host, gpu, q, counts, mask, dtype, positions=pos, window=window)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("d,group,lens,counts", [(64, 1, [70, 40, 9], [33, 40, 9]), (128, 8, [200, 90], [64, 50]),
                                                 (128, 2, [2000], [20])])
def test_masks_of_the_callers_own(dtype, d, group, lens, counts):
    """Random bits (also of tokens that come later), rows without a bit, bits past a sequence's tokens; one word more
    than the trees need, and fewer."""
    host, gpu = U.make(17, lens, 16, 1, d, "e4m3")
    q = _queries(18, sum(counts), group, d, dtype)
    rng = np.random.default_rng(19)
    for words in (1, -(-max(counts) // 32) + 1):
        mask = rng.integers(0, 1 << 32, (sum(counts), words), dtype=np.uint64).astype(np.uint32)
        mask[::5] = 0
        _check(host, gpu, q, counts, mask, dtype)


def test_rows_that_see_nothing():
    """A sequence that is its tree alone, and rows without bits: 0, and -inf in lse."""
    for dtype, group in (("bf16", 1), ("bf16", 64), ("f32", 2)):
        host, gpu = U.make(20, [6, 40], 16, 1, 64, "int8")
        q = _queries(21, 12, group, 64, dtype)
        mask, _ = C.tree_mask(_parents(22, [6, 6], "chain"), [6, 6], 1)
        mask[[0, 3, 11]] = 0
        out = _check(host, gpu, q, [6, 6], mask, dtype, ragged=False)
        assert (out[[0, 3]] == 0).all() and (out[11] != 0).any()


def test_a_chain_is_causal_attention():
    """Both calls take the same bar around the same numbers; and lse of the two is the same softmax's."""
    import paper_2412_09282_gb300 as P
    counts, lens = [9, 30], [500, 77]
    host, gpu = U.make(23, lens, 16, 2, 128, "int8")
    q = U.heads(_queries(24, 39, 4, 128, "f32"), "f32")
    off = U.offsets(counts)
    mask, _ = P.crvq_tree_mask(_ints(_parents(25, counts, "chain")), 2, off=off, max_new=30)
    a, la = P.crvq_cache_tree_attention(gpu, q, mask, q_off=off, want_lse=True)
    b, lb = P.crvq_cache_attention(gpu, q, q_off=off, want_lse=True)
    P.crvq_sync()
    assert torch.allclose(la, lb, rtol=0, atol=1e-4) and torch.allclose(a, b, rtol=1e-3, atol=1e-3 * float(b.abs().max()))


def test_not_finite_queries_stay_in_their_rows_and_results_repeat():
    import paper_2412_09282_gb300 as P
    for dtype, group, n in (("bf16", 8, 16), ("f32", 1, 5)):
        host, gpu = U.make(26, [300], 32, 1, 64, "int8")
        q = _queries(27, n, group, 64, dtype)
        mask = _bits(C.tree_mask(_parents(28, [n]), [n], 1)[0])
        ref = U.exactly(P.crvq_cache_tree_attention(gpu, U.heads(q, dtype), mask))
        q[2, 0, 7], q[4, group - 1, 1] = np.nan, np.inf
        out = U.exactly(P.crvq_cache_tree_attention(gpu, U.heads(q, dtype), mask))
        again = U.exactly(P.crvq_cache_tree_attention(gpu, U.heads(q, dtype), mask))
        P.crvq_sync()
        ok = np.ones((n, group), bool)
        ok[2, 0] = ok[4, group - 1] = False
        assert np.array_equal(out[ok], ref[ok]) and np.isnan(out[~ok]).all()
        assert np.array_equal(out, again, equal_nan=True)


def test_rows_behind_the_last_sequence_stay_as_they_were():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(29, [60, 20], 16, 1, 64, "int8")
    for dtype, group in (("bf16", 64), ("f32", 1)):
        q = U.heads(_queries(30, 9, group, 64, dtype), dtype)
        mask = torch.full((9, 1), -1, dtype=torch.int32, device="cuda")
        out = torch.full_like(q, 7.0)
        P.crvq_cache_tree_attention(gpu, q, mask, q_off=U.offsets([4, 3]), out=out)
        parents = _ints([-1] * 9)
        m, p = torch.full((9, 1), 5, dtype=torch.int32, device="cuda"), torch.full((9,), 5, dtype=torch.int32, device="cuda")
        P.crvq_tree_mask(parents, 2, off=U.offsets([4, 3]), max_new=4, mask_out=m, positions_out=p)
        P.crvq_sync()
        assert (out[7:] == 7).all() and (out[:7] != 7).any() and (m[7:] == 5).all() and (p[7:] == 5).all()
        assert (m[:7, 0].cpu() == torch.tensor([1, 2, 4, 8, 1, 2, 4])).all()


def test_bad_pages_are_reported():
    import paper_2412_09282_gb300 as P
    for dtype, group in (("bf16", 32), ("f32", 1)):
        host, _ = U.make(31, [40, 20], 16, 1, 64, "int8")
        host["pages"][0, 1] = 77
        gpu = U.on_gpu(host, "int8")
        q = _queries(32, 6, group, 64, dtype)
        out = P.crvq_cache_tree_attention(gpu, U.heads(q, dtype), torch.full((6, 1), 1, dtype=torch.int32, device="cuda"))
        with pytest.raises(P.CrvqError) as e:
            P.crvq_sync()
        assert e.value.status == -7
        assert np.isfinite(U.exactly(out)).all()


def test_refusals():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(33, [40, 20], 16, 2, 64, "int8")
    q = torch.ones((2, 4, 64), device="cuda")
    mask = torch.ones((2, 1), dtype=torch.int32, device="cuda")
    for bad in (dict(scale=float("nan")), dict(window=-1), dict(window=3), dict(out=q.bfloat16())):
        with pytest.raises(P.CrvqError) as e:
            P.crvq_cache_tree_attention(gpu, q, mask, **bad)
        assert e.value.status == -1
    with pytest.raises(P.CrvqError):                            # 80 drafted tokens a sequence, 32 bits a row
        P.crvq_cache_tree_attention(gpu, torch.ones((160, 4, 64), device="cuda"),
                                    torch.ones((160, 1), dtype=torch.int32, device="cuda"))
    for bad in (mask[:1], mask.long(), mask.t(), mask[:, :0]):
        with pytest.raises((TypeError, ValueError)):
            P.crvq_cache_tree_attention(gpu, q, bad)
    with pytest.raises(ValueError):
        P.crvq_cache_tree_attention(gpu, q, mask, positions=torch.zeros(3, dtype=torch.int32, device="cuda"))
    p = torch.zeros(4, dtype=torch.int32, device="cuda")
    for args, kw in (((p.long(), 2), {}), ((p.view(2, 2), 2), {}), ((p, 0), {}), ((p, 2), dict(lens=p)),
                     ((p, 2), dict(off=U.offsets([2, 2]))), ((p, 2), dict(mask_out=p.view(2, 2))),
                     ((torch.zeros(80, dtype=torch.int32, device="cuda"), 2), dict(max_new=32)),
                     ((p, 2), dict(positions_out=p[:3]))):
        with pytest.raises((TypeError, ValueError)):
            P.crvq_tree_mask(*args, **kw)
    with pytest.raises(P.CrvqError):
        P.crvq_tree_mask(p, 3, max_new=5)                       # 4 tokens for 3 sequences
    with pytest.raises(P.CrvqError):
        P.crvq_tree_mask(p, 2, window=-1)
    assert P.crvq_tree_mask(p[:0], 1, max_new=1)[0].shape == (0, 1)
    assert P.crvq_cache_tree_attention(gpu, q[:0], mask[:0], q_off=U.offsets([0, 0])).shape[0] == 0


def test_a_captured_step_replays_with_new_trees_and_lengths():
    """Mask and attention in one graph: parents, lengths and queries change between replays."""
    import paper_2412_09282_gb300 as P
    for dtype, group in (("bf16", 16), ("f32", 2)):
        host, gpu = U.make(34, [90, 200], 16, 1, 64, "int8")
        parents, q = torch.zeros(14, dtype=torch.int32, device="cuda"), torch.zeros((14, group, 64), device="cuda", dtype=U.TORCH[dtype])
        off = U.offsets([6, 8])

        def step():
            mask, pos = P.crvq_tree_mask(parents, 2, off=off, lens=gpu.lens, max_new=8, window=50)
            return P.crvq_cache_tree_attention(gpu, q, mask, q_off=off, positions=pos, window=50)

        parents.fill_(-1)
        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        for seed, lens in ((35, [90, 200]), (36, [7, 131])):
            parents.copy_(_ints(_parents(seed, [6, 8])))
            q.copy_(torch.from_numpy(_queries(seed, 14, group, 64, dtype)))
            gpu.lens.copy_(_ints(lens))
            g.replay()
            ref = step()
            P.crvq_sync()
            assert torch.equal(out, ref) and (ref != 0).any()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,page,n_kv,group,n", [(128, 64, 20, 1, 20), (64, 16, 24, 2, 12), (128, 48, 16, 4, 9), (64, 32, 32, 1, 40)])
def test_some_tens_of_queries_over_many_heads(fmt, dtype, d, page, n_kv, group, n):
    """Long and short sequences beside each other, trees that are all there is, none, and windows; not all full units.
    Weights below fp16's normal numbers are off by 2^-25 beside a largest one of 2^5 at least, so n of them by n 2^-30 of the
    largest's weight, whose token has at least half of its block's largest code in some channel: n 2^-29 of the row's
    largest sum of p |V|. It shows in a channel where that token's code is 0, as one of 20 x 128 x 84 here has."""
    lens, counts = [1400, 17, 333, n, 700, 128], [n, 9, max(1, n - 5), n, 0, n]
    host, gpu = U.make(40, lens, page, n_kv, d, fmt, page_gap=1)
    q = _queries(41, sum(counts), n_kv * group, d, dtype, 2.0)
    mask, pos = C.tree_mask(_parents(42, counts), counts, -(-max(counts) // 32), 0, lens)
    _check(host, gpu, q, counts, mask, dtype, gap=5, least=2.0 ** -29)
    mask, pos = C.tree_mask(_parents(42, counts), counts, -(-max(counts) // 32), 300, lens)
    _check(host, gpu, q, counts, mask, dtype, positions=pos, window=300, least=2.0 ** -29)


def test_growing_maxima_and_scales_far_apart_with_some_tens_of_queries():
    """Key scales that grow along the sequence (references move many times), value scales far apart (as far as fp16 outputs
    hold them, and 2^80), zeros among them, and not finite queries beside finite ones. What weights below fp16's normal
    numbers are off by, 2^-25 beside a largest one of 2^5 at least, is n 2^-29 of the row's largest sum of p |V| (see
    test_gpu_attention_scales.py)."""
    import paper_2412_09282_gb300 as P
    for fmt, dtype, low, high in (("int8", "f16", -12, 8), ("e4m3", "bf16", -40, 40)):
        host, _ = U.make(43, [2000, 900], 16, 16, 128, fmt)
        rng = np.random.default_rng(44)
        for b, n in enumerate((125, 57)):
            order = host["pages"][b, :n]
            host["k_scale"][order, :, 0] *= np.exp(np.linspace(-2.0, 1.5, n)).astype(np.float32)[:, None]
            host["v_scale"][order, :, 0] *= np.exp2(rng.uniform(low, high, (n, 16))).astype(np.float32)
            host["v_scale"][order[20], :, 0] = 0.0
        gpu = U.on_gpu(host, fmt)
        q = _queries(45, 40, 16, 128, dtype, 1.0)
        mask, _ = C.tree_mask(_parents(46, [20, 20]), [20, 20], 1)
        _check(host, gpu, q, [20, 20], mask, dtype, least=2.0 ** -29)
        ref = U.exactly(P.crvq_cache_tree_attention(gpu, U.heads(q, dtype), _bits(mask), q_off=U.offsets([20, 20])))
        q[7, 1, 3], q[30, 0, 5] = np.nan, np.inf
        out = U.exactly(P.crvq_cache_tree_attention(gpu, U.heads(q, dtype), _bits(mask), q_off=U.offsets([20, 20])))
        again = U.exactly(P.crvq_cache_tree_attention(gpu, U.heads(q, dtype), _bits(mask), q_off=U.offsets([20, 20])))
        P.crvq_sync()
        same = np.ones((40, 16), bool)
        same[7, 1] = same[30, 0] = False
        assert np.array_equal(out[same], ref[same]) and np.isnan(out[~same]).all()
        assert np.array_equal(out, again, equal_nan=True)
