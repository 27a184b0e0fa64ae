"""Moving kept tokens together in the paged 8-bit cache: codes and scales equal to the oracle's, which restates the fp32
steps; whatever is not written stays bit for bit."""
import numpy as np
import pytest
import torch

import decode_util as U
from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def _choice(seed, lens, start, counts, n_kv, each, wide=None):
    """count[b] places of every sequence (and head) from start[b] on, ascending; behind the last, places that do not exist."""
    rng = np.random.default_rng(seed)
    most = wide or max(1, max(counts))
    idx = np.full((len(lens), n_kv, most), 1 << 30, np.int32)
    for b, (n, a, c) in enumerate(zip(lens, start, counts)):
        for h in range(n_kv):
            idx[b, h, :c] = a + np.sort(rng.permutation(n - a)[:c])
    return idx if each else np.ascontiguousarray(idx[:, 0])


def _equal(host, gpu, fmt):
    """All codes, scales (NaN where none was written) and bytes of the pool."""
    for name in ("K", "V"):
        assert np.array_equal(U.exactly(getattr(gpu, name)), host[name], equal_nan=True), name
    for name in ("k_scale", "v_scale"):
        assert np.array_equal(U.exactly(getattr(gpu, name)), host[name], equal_nan=True), name


def _other(seed, host, start, counts, page, fmt, gap=0):
    """Another pool, of other pages, with tokens before start[b] in it."""
    return U.make(seed, [a + c for a, c in zip(start, counts)], page, host["K"].shape[1], host["K"].shape[3], fmt, page_gap=gap)


SHAPES = [
    # lens, start, counts
    ([40, 70, 33, 7, 150], [0, 0, 0, 0, 0], [17, 70, 1, 0, 99]),
    ([40, 70, 33, 7, 150], [30, 16, 32, 0, 149], [4, 31, 1, 7, 1]),            # in the middle of blocks, at their ends
    ([300, 17], [129, 15], [150, 2]),
]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d,page,n_kv,each", [(128, 64, 2, True), (64, 16, 3, True), (256, 48, 1, False), (128, 32, 2, False)])
@pytest.mark.parametrize("shape", SHAPES)
def test_in_place_and_into_other_pages(fmt, d, page, n_kv, each, shape):
    import paper_2412_09282_gb300 as P
    lens, start, counts = shape
    idx = _choice(80, lens, start, counts, n_kv, each, wide=max(counts) + 3)
    host, gpu = U.make(81, lens, page, n_kv, d, fmt, page_gap=1)
    other, to = _other(82, host, start, counts, 80 - page if page < 64 else page, fmt, gap=2)
    before = {k: v.copy() for k, v in host.items()}
    P.crvq_cache_keep(gpu, _ints(idx), _ints(counts), start=_ints(start), out=to)
    P.crvq_sync()
    C.keep(host, idx, counts, start, other, fmt)
    _equal(other, to, fmt)
    _equal(before, gpu, fmt)
    got = P.crvq_cache_keep(gpu, _ints(idx), _ints(counts), start=_ints(start))
    P.crvq_sync()
    assert got is gpu
    C.keep(host, idx, counts, start, host, fmt)
    _equal(host, gpu, fmt)


@pytest.mark.parametrize("d,n", [(64, 5000), (128, 3333), (256, 1200)])
def test_in_place_over_several_rounds(d, n):
    """More tokens than the CTAs of a (sequence, head) take at a time, of which most, few and all stay."""
    import paper_2412_09282_gb300 as P
    for counts in ([n - 900, 40, 300], [n, 60, 299], [n // 5, 1, 0]):
        lens = [n, 60, 300]
        idx = _choice(83, lens, [0, 0, 0], counts, 1, True)
        host, gpu = U.make(84, lens, 64, 1, d, "int8")
        P.crvq_cache_keep(gpu, _ints(idx), _ints(counts))
        P.crvq_sync()
        C.keep(host, idx, counts, [0, 0, 0], host, "int8")
        _equal(host, gpu, "int8")


def test_other_pages_of_the_same_pool_in_any_order():
    """Not ascending, one token twice, from shared source pages: all of which is open where pages differ."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(85, [40, 40], 16, 2, 64, "int8", spare=8)
    host["pages"][1] = host["pages"][0]
    gpu = U.on_gpu(host, "int8")
    free = np.setdiff1d(np.arange(host["K"].shape[0]), host["pages"][0])
    out = dict(host, pages=free[:6].reshape(2, 3).astype(np.int32), lens=np.asarray([20, 33], np.int32))
    to = P.KVCache(gpu.K, gpu.V, gpu.k_scale, gpu.v_scale, _ints(out["pages"]), _ints(out["lens"]))
    rng = np.random.default_rng(86)
    idx = rng.integers(0, 40, (2, 2, 33)).astype(np.int32)
    P.crvq_cache_keep(gpu, _ints(idx), _ints([20, 33]), out=to)
    P.crvq_sync()
    C.keep(host, idx, [20, 33], [0, 0], out, "int8")
    _equal(host, gpu, "int8")


def test_scales_far_apart_zeros_and_blocks_that_keep_their_bits():
    import paper_2412_09282_gb300 as P
    for fmt in ("int8", "e4m3"):
        host, _ = U.make(87, [200, 64], 16, 1, 64, fmt)
        rng = np.random.default_rng(88)
        host["k_scale"] *= np.exp(rng.uniform(-69, 69, host["k_scale"].shape)).astype(np.float32)
        host["v_scale"][host["pages"][0, :9]] = 0.0                # blocks of zeros
        host["K"][host["pages"][1]] = D_largest(fmt)
        host["k_scale"][host["pages"][1]] = 2.0 ** -149
        gpu = U.on_gpu(host, fmt)
        idx = _choice(89, [200, 64], [0, 0], [90, 64], 1, True)
        other, to = _other(90, host, [0, 0], [90, 64], 32, fmt)
        P.crvq_cache_keep(gpu, _ints(idx), _ints([90, 64]), out=to)
        P.crvq_sync()
        C.keep(host, idx, [90, 64], [0, 0], other, fmt)
        _equal(other, to, fmt)


def D_largest(fmt):
    return np.float32(127 if fmt == "int8" else 448)


def test_strided_indices_one_for_all_heads_and_none():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(91, [50, 60], 16, 3, 64, "int8")
    idx = _choice(92, [50, 60], [0, 0], [20, 31], 3, True, wide=40)
    buf = torch.full((3, 2, 50), -1, dtype=torch.int32, device="cuda")
    view = buf.transpose(0, 1)[:, :, 4:44]
    view.copy_(_ints(idx))
    P.crvq_cache_keep(gpu, view, _ints([20, 31]))
    P.crvq_sync()
    C.keep(host, idx, [20, 31], [0, 0], host, "int8")
    _equal(host, gpu, "int8")
    one = _ints(np.arange(5)[None].repeat(2, 0))
    P.crvq_cache_keep(gpu, one[:, None].expand(2, 3, 5), _ints([5, 0]))
    P.crvq_cache_keep(gpu, one[:, :0], _ints([0, 0]))
    P.crvq_sync()
    C.keep(host, np.arange(5, dtype=np.int32)[None].repeat(2, 0), [5, 0], [0, 0], host, "int8")
    _equal(host, gpu, "int8")


def _reports(call):
    import paper_2412_09282_gb300 as P
    call()
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -7


def test_bad_places_counts_and_pages_are_reported():
    import paper_2412_09282_gb300 as P
    lens = [40, 20]
    host, gpu = U.make(93, lens, 16, 1, 64, "int8")
    good = np.asarray([[3, 5, 7, 9], [0, 1, 18, 19]], np.int32)
    for bad in (-1, 40, 1 << 30, -(1 << 31)):
        idx = good.copy()
        idx[0, 1] = bad
        other, to = _other(94, host, [0, 0], [4, 4], 16, "int8")
        _reports(lambda: P.crvq_cache_keep(gpu, _ints(idx), _ints([4, 4]), out=to))
        C.keep(host, good, [4, 4], [0, 0], other, "int8")
        got = U.exactly(to.K)[other["pages"][0, 0], 0]
        assert (got[1] == 0).all()                              # the others lie in their places
        s = float(to.k_scale[int(other["pages"][0, 0]), 0, 0])
        for r, p in ((0, 3), (2, 7), (3, 9)):
            pg = host["pages"][0, 0]
            assert np.abs(got[r] * s - host["K"][pg, 0, p] * host["k_scale"][pg, 0, 0]).max() <= 0.5 * s * (1 + 1e-5)
        pg = other["pages"][1, 0]
        assert np.array_equal(U.exactly(to.K)[pg], other["K"][pg])
    # in place: a token that would move back
    idx = good.copy()
    idx[1, 2] = 1
    keep_host, g2 = U.make(93, lens, 16, 1, 64, "int8")
    _reports(lambda: P.crvq_cache_keep(g2, _ints(idx), _ints([4, 4])))
    # counts and starts: the sequence is left alone
    for counts, start in (([5, 4], None), ([-1, 4], None), ([4, 4], [-1, 0]), ([4, 4], [61, 0])):
        other, to = _other(95, host, [0, 0], [64, 4], 16, "int8")
        _reports(lambda: P.crvq_cache_keep(gpu, _ints(good), _ints(counts), start=None if start is None else _ints(start), out=to))
        C.keep(host, good, [0, 4], [0, 0], other, "int8")
        _equal(other, to, "int8")
    # pages of the source and of the destination
    b2 = {k: v.copy() for k, v in host.items()}
    b2["pages"][0, 0] = 99
    other, to = _other(96, host, [0, 0], [4, 4], 16, "int8")
    _reports(lambda: P.crvq_cache_keep(U.on_gpu(b2, "int8"), _ints(good), _ints([4, 4]), out=to))
    assert (U.exactly(to.K)[other["pages"][0, 0], 0, :4] == 0).all()
    other, to = _other(96, host, [0, 0], [4, 4], 16, "int8")
    to.pages[0, 0] = -1
    _reports(lambda: P.crvq_cache_keep(gpu, _ints(good), _ints([4, 4]), out=to))
    C.keep(host, good, [0, 4], [0, 0], other, "int8")
    _equal(other, to, "int8")
    # the same pages by another table: nothing is written
    same = P.KVCache(gpu.K, gpu.V, gpu.k_scale, gpu.v_scale, gpu.pages.clone(), gpu.lens)
    _reports(lambda: P.crvq_cache_keep(gpu, _ints(good), _ints([4, 4]), out=same))
    _equal(host, gpu, "int8")
    P.crvq_sync()


def test_refusals():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(97, [40, 20], 16, 2, 64, "int8")
    idx, count = torch.zeros((2, 2, 4), dtype=torch.int32, device="cuda"), _ints([4, 4])
    others = [U.make(97, [40, 20], 16, 1, 64, "int8")[1], U.make(97, [40], 16, 2, 64, "int8")[1],
              U.make(97, [40, 20], 16, 2, 128, "int8")[1], U.make(97, [40, 20], 16, 2, 64, "e4m3")[1],
              P.KVCache(gpu.K, gpu.V.clone(), gpu.k_scale, gpu.v_scale, gpu.pages, gpu.lens)]
    for out in others:
        with pytest.raises(P.CrvqError) as e:
            P.crvq_cache_keep(gpu, idx, count, out=out)
        assert e.value.status == -1
    with pytest.raises(P.CrvqError):
        P.crvq_cache_keep(gpu, idx.as_strided((2, 2, 4), (8, 2, 1)), count)
    for args in ((idx.long(), count), (idx[:1], count), (idx[:, :1], count), (idx.transpose(1, 2), count), (idx, count[:1]),
                 (idx, count.long()), (idx[0, 0], count), (idx.cpu(), count)):
        with pytest.raises((TypeError, ValueError)):
            P.crvq_cache_keep(gpu, *args)
    with pytest.raises(ValueError):
        P.crvq_cache_keep(gpu, idx, count, start=_ints([0]))


@pytest.mark.parametrize("in_place", [True, False])
def test_products_that_round_to_ties(in_place):
    """int8: c (their scale / its scale) is rounded to fp32, and that to a whole number: where the first rounding ends on
    k + 1/2 and the exact product does not, one rounding of both would give another code."""
    import paper_2412_09282_gb300 as P
    pairs = []
    for c in range(3, 128):
        for k in range(c):
            r = np.float32((k + 0.5) / c)
            exact = float(r) * c                                 # (31 bits: exact in fp64)
            if np.float32(c) * r == np.float32(k + 0.5) and exact != k + 0.5 and round(exact) != round(k + 0.5):
                pairs.append((c, r))
    assert len(pairs) > 1000
    pairs = pairs[:1500]
    blocks = 16 * (len(pairs) // 15)                             # of 16 tokens; every 16th has scale 1
    host, _ = U.make(150, [16 * blocks], 16, 1, 64, "int8")
    idx = 16 * np.arange(blocks, dtype=np.int32) + np.random.default_rng(151).integers(0, 16, blocks)
    idx[:16] = 16 * np.arange(16)
    at = 0
    for i in range(blocks):
        pg = host["pages"][0, i]
        for name, s in (("K", "k_scale"), ("V", "v_scale")):
            host[s][pg, 0, 0] = 1.0 if i % 16 == 0 else pairs[at][1]
            if i % 16:
                host[name][pg, 0, :, 5::16] = pairs[at][0] if name == "K" else -pairs[at][0]
        at += i % 16 != 0
    gpu = U.on_gpu(host, "int8")
    other, to = (host, gpu) if in_place else U.make(152, [blocks], 32, 1, 64, "int8")
    ref = {k: v.copy() for k, v in other.items()}
    C.keep(host, idx[None], [blocks], [0], ref, "int8")
    P.crvq_cache_keep(gpu, _ints(idx[None]), _ints([blocks]), out=to)
    P.crvq_sync()
    _equal(ref, to, "int8")


@pytest.mark.parametrize("d,fmt,page", [(64, "int8", 48), (128, "e4m3", 16), (256, "int8", 64)])
def test_in_place_over_several_rounds_from_the_middle_of_a_block(d, fmt, page):
    """Rounds whose codes are read while the ones before are written: dense selections (few tokens dropped, sources just
    behind their places), sparse ones, and a sequence that ends earlier."""
    import paper_2412_09282_gb300 as P
    lens, start = [9001, 4100, 9000], [1003, 17, 0]
    for seed, counts in ((160, [7990, 100, 8999]), (161, [2100, 4083, 1])):
        host, gpu = U.make(seed, lens, page, 2, d, fmt)
        idx = _choice(seed + 10, lens, start, counts, 2, True)
        P.crvq_cache_keep(gpu, _ints(idx), _ints(counts), start=_ints(start))
        P.crvq_sync()
        C.keep(host, idx, counts, start, host, fmt)
        _equal(host, gpu, fmt)
