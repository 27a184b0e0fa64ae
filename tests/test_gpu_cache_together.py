"""The calls around the cache as a serving program makes them: a tree of drafted tokens appended, attended to and cut to its
accepted path; a cache cut to a budget by the attention its tokens got; both captured in graphs and run beside one
another; pools and sums of more than 2^32 bytes; calls on a stream that the caller gives.
"""
import threading

import numpy as np
import pytest
import torch

import decode_util as U
import test_gpu_cache_weights as W
import test_gpu_tree as T
from oracle import cache_oracle as C
from oracle import decode_oracle as D
from test_gpu_decode_streams import SIZE, _again

pytestmark = pytest.mark.gpu


def _on_host(gpu, host):
    """The oracle's cache with what the GPU's holds now."""
    return dict(host, K=U.exactly(gpu.K), V=U.exactly(gpu.V), k_scale=U.exactly(gpu.k_scale), v_scale=U.exactly(gpu.v_scale),
                lens=gpu.lens.cpu().numpy())


@pytest.mark.parametrize("fmt,dtype,group", [("int8", "bf16", 8), ("e4m3", "f32", 2)])
def test_a_tree_is_drafted_verified_and_cut_to_its_path(fmt, dtype, group):
    """Append the tree, attend by its mask, keep one path behind the tokens before the tree, attend to what is left: both
    attentions against fp64 over what the cache then holds."""
    import paper_2412_09282_gb300 as P
    lens, counts = [130, 57], [12, 9]
    host, _ = U.make(60, lens, 32, 2, 64, fmt, wide=8, spare=20)
    free = sorted(set(range(host["K"].shape[0])) - set(host["pages"][0, :5].tolist() + host["pages"][1, :2].tolist()))
    host["pages"][0, 5:], host["pages"][1, 2:] = free[:3], free[3:9]   # (room for the drafted tokens)
    gpu = U.on_gpu(host, fmt)
    q = T._queries(62, sum(counts), 2 * group, 64, dtype)
    k, v = (U.heads(T._queries(s, sum(counts), 2, 64, dtype), dtype) for s in (63, 64))
    off, parents = U.offsets(counts), T._parents(65, counts)
    gpu.lens.add_(T._ints(counts))
    mask, pos = P.crvq_tree_mask(T._ints(parents), 2, off=off, lens=gpu.lens, max_new=12)
    P.crvq_cache_append(gpu, k, v, new_off=off)
    P.crvq_sync()
    now = _on_host(gpu, host)
    ref_mask, ref_pos = C.tree_mask(parents, counts, 1, 0, now["lens"])
    assert np.array_equal(mask.cpu().numpy().view(np.uint32), ref_mask) and np.array_equal(pos.cpu().numpy(), ref_pos)
    T._check(now, gpu, q, counts, ref_mask, dtype)
    # the path of the deepest token stays
    idx, kept = np.zeros((2, 12), np.int32), []
    for b, first in enumerate((0, counts[0])):
        path = max(C.ancestors(parents[first:first + counts[b]]), key=len)[::-1]
        idx[b, :len(path)] = lens[b] + np.asarray(path)
        kept.append(len(path))
    P.crvq_cache_keep(gpu, T._ints(idx), T._ints(kept), start=T._ints(lens))
    gpu.lens.copy_(T._ints(lens) + T._ints(kept))
    P.crvq_sync()
    want = {key: x.copy() for key, x in now.items()}
    C.keep(want, idx, kept, lens, want, fmt)
    want["lens"] = np.asarray(lens, np.int32) + np.asarray(kept, np.int32)
    got = _on_host(gpu, host)
    for b in range(2):
        for name in ("K", "V"):
            assert np.array_equal(D.values(got, name, b, 0, want["lens"][b]), D.values(want, name, b, 0, want["lens"][b]))
    T._check(want, gpu, q[[0, counts[0]]], [1, 1], np.ones((2, 1), np.uint32), dtype)


def _cut(gpu, q, keep, off=None, out=None):
    """Attention, the weights that its tokens got, and the cache cut to `keep` tokens by them."""
    import paper_2412_09282_gb300 as P
    o, lse = P.crvq_cache_attention(gpu, q, q_off=off, want_lse=True)
    w = P.crvq_cache_weights(gpu, q, lse, q_off=off)
    left = torch.empty_like(w)
    idx, count = P.crvq_cache_select(w, gpu.lens, keep, first=2, recent=9, weights_out=left)
    P.crvq_cache_keep(gpu, idx, count, out=out)
    return o, lse, w, idx, count, left


@pytest.mark.parametrize("fmt,dtype,group,counts", [("int8", "bf16", 8, [20, 20]), ("e4m3", "f32", 2, [1, 1]),
                                                    ("int8", "f16", 4, [30, 3])])
def test_a_cache_is_cut_to_a_budget(fmt, dtype, group, counts):
    import paper_2412_09282_gb300 as P
    for elsewhere in (False, True):
        host, gpu = U.make(66, [700, 60], 16, 2, 128, fmt)
        other = U.make(67, [100, 100], 64, 2, 128, fmt) if elsewhere else (host, gpu)
        q = T._queries(68, sum(counts), 2 * group, 128, dtype)
        _, lse, w, idx, count, left = _cut(gpu, U.heads(q, dtype), 64, U.offsets(counts), other[1] if elsewhere else None)
        other[1].lens.copy_(count)
        P.crvq_sync()
        W._check(host, U.on_gpu(host, fmt), q, counts, dtype, w.shape[2], decay=1.0, lse=U.exactly(lse))
        ref_idx, ref_count, ref_left = C.select(U.exactly(w), [700, 60], 64, 2, 9)
        assert np.array_equal(idx.cpu().numpy(), ref_idx) and np.array_equal(count.cpu().numpy(), ref_count)
        assert np.array_equal(U.exactly(left), ref_left)
        want = {key: x.copy() for key, x in other[0].items()}
        C.keep(host, ref_idx, ref_count, [0, 0], want, fmt)
        want["lens"] = ref_count
        got = _on_host(other[1], other[0])
        for b in range(2):
            for name in ("K", "V"):
                assert np.array_equal(D.values(got, name, b, 0, ref_count[b]), D.values(want, name, b, 0, ref_count[b]))
        T._check(want, other[1], q[[0, counts[0]]], [1, 1], np.ones((2, 1), np.uint32), dtype)


def _setting(seed, dtype, group, n):
    """A step's inputs: a cache, another one for what stays, a tree's queries, its parents."""
    host, gpu = U.make(seed, [2000, 900], 16, 2, 128, "int8")
    out = U.make(seed + 1, [256, 256], 16, 2, 128, "int8")[1]
    q = U.heads(T._queries(seed + 2, 2 * n, 2 * group, 128, dtype), dtype)
    return gpu, out, q, T._ints(T._parents(seed + 3, [n, n]))


def _step(gpu, out, q, parents, stream=None):
    import paper_2412_09282_gb300 as P
    kw = dict(stream=stream)
    mask, _ = P.crvq_tree_mask(parents, 2, lens=gpu.lens, **kw)
    o, lse = P.crvq_cache_tree_attention(gpu, q, mask, want_lse=True, **kw)
    o2, lse2 = P.crvq_cache_attention(gpu, q, want_lse=True, **kw)
    w = P.crvq_cache_weights(gpu, q, lse2, **kw)
    idx, count = P.crvq_cache_select(w, gpu.lens, 200, first=4, recent=40, **kw)
    P.crvq_cache_keep(gpu, idx, count, out=out, **kw)
    return o, lse, w, idx, count, out.K, out.k_scale


KINDS = [("bf16", 8, 16), ("f32", 1, 3), ("f16", 1, 1)]


def test_two_graphs_replayed_on_two_streams_and_eager_steps_beside_them():
    """Every graph has what it needs of memory to itself: replays of several at once give what one after another gives."""
    import paper_2412_09282_gb300 as P
    settings = [_setting(70 + 10 * i, *kind) for i, kind in enumerate(KINDS[:2])]
    refs = [[t.clone() for t in _step(*s)] for s in settings]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in settings:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_step(*s))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    eager = _setting(90, *KINDS[2])
    eager_ref = [t.clone() for t in _step(*eager)]
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        got = _step(*eager)
    P.crvq_sync()
    torch.cuda.synchronize()
    for ref, out in zip(refs + [eager_ref], outs + [got]):
        for a, b in zip(ref, out):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_steps_of_several_threads_at_once():
    import paper_2412_09282_gb300 as P
    settings = [_setting(100 + 10 * i, *KINDS[i % 3]) for i in range(4)]
    refs = [[t.clone() for t in _step(*s)] for s in settings]
    torch.cuda.synchronize()
    got, failed = [None] * 4, []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(10):
                    got[i] = _step(*settings[i])
            s.synchronize()
        except Exception as e:                                   # (reported below, by the main thread)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    P.crvq_sync()
    assert not failed
    for ref, out in zip(refs, got):
        for a, b in zip(ref, out):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_many_sequences_of_one_tile_with_many_columns():
    """Weights of a share that has several sequences, with tiles for one group of its warps or for both, columns that fill
    the queries' memory once or several times, and sequences without queries among them."""
    rng = np.random.default_rng(110)
    lens = [int(x) for x in rng.integers(1, 300, 90)]
    counts = [int(min(n, c)) for n, c in zip(lens, rng.integers(0, 40, 90))]
    counts[3], lens[3] = 150, 150                               # (1200 columns)
    host, gpu = U.make(111, lens, 16, 4, 64, "int8")
    q = T._queries(112, sum(counts), 32, 64, "bf16")
    import paper_2412_09282_gb300 as P
    lse = U.exactly(P.crvq_cache_attention(gpu, U.heads(q, "bf16"), q_off=U.offsets(counts), want_lse=True)[1])
    for _ in range(2):
        a = W._check(host, gpu, q, counts, "bf16", 320, lse=lse, seed=113)
    b = W._check(host, gpu, q, counts, "bf16", 320, lse=lse, seed=113, in_place=True)
    assert torch.equal(a, b)


def test_one_sequence_with_more_columns_than_the_average():
    """Single tokens, but one sequence has 40 columns: the queries that stay in registers come 8 at a time."""
    lens, counts = [300] + [20] * 15, [5] + [0] * 15
    host, gpu = U.make(114, lens, 16, 1, 128, "e4m3")
    for dtype in ("f32", "bf16"):
        q = T._queries(115, 5, 8, 128, dtype)
        a = W._check(host, gpu, q, counts, dtype, 304, seed=116)
        b = W._check(host, gpu, q, counts, dtype, 304, seed=116, in_place=True)
        assert torch.equal(a, b)


def _far(host, fmt, pages):
    """The cache in a pool of `pages` pages, its own at the end."""
    import paper_2412_09282_gb300 as P
    small = U.on_gpu(host, fmt)
    n = small.K.shape[0]
    t = {}
    for name in ("K", "V", "k_scale", "v_scale"):
        x = getattr(small, name)
        big = torch.empty((pages,) + tuple(x.shape[1:]), dtype=x.dtype, device="cuda")
        big[pages - n:].view(torch.uint8).copy_(x.contiguous().view(torch.uint8))
        t[name] = big
    table = torch.where(small.pages >= 0, small.pages + (pages - n), small.pages).contiguous()
    return small, P.KVCache(t["K"], t["V"], t["k_scale"], t["v_scale"], table, small.lens)


@pytest.mark.parametrize("dtype,group,counts", [("bf16", 8, [20, 9]), ("f32", 1, [2, 1])])
def test_offsets_past_32_bits(dtype, group, counts):
    """Pools of 4.5 GB and rows of sums 2^31 elements apart: the same results as in small ones."""
    import paper_2412_09282_gb300 as P
    host, _ = U.make(120, [333, 90], 64, 8, 128, "int8")
    small, big = _far(host, "int8", 70000)
    q = U.heads(T._queries(121, sum(counts), 8 * group, 128, dtype), dtype)
    off = U.offsets(counts)
    mask = T._bits(C.tree_mask(T._parents(122, counts), counts, 1)[0])
    rows = torch.empty((1 << 31) + 8 * 400, device="cuda")
    view = rows.as_strided((2, 8, 400), (1 << 31, 400, 1))
    results = []
    for c in (small, big):
        tree = P.crvq_cache_tree_attention(c, q, mask, q_off=off)
        out, lse = P.crvq_cache_attention(c, q, q_off=off, want_lse=True)
        w = P.crvq_cache_weights(c, q, lse, q_off=off, out=view if c is big else torch.empty((2, 8, 400), device="cuda"))
        idx, count = P.crvq_cache_select(w, c.lens, 70, recent=7)
        P.crvq_cache_keep(c, idx, count)
        n = small.K.shape[0]
        P.crvq_sync()
        results.append([tree, w.contiguous(), idx, count] + [getattr(c, x)[-n:].contiguous().view(torch.uint8)
                                                             for x in ("K", "V", "k_scale", "v_scale")])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def _stream_calls():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(130, [20], 16, 2, 64, "int8", wide=1100)
    n = SIZE // (2 * 64 * 4)
    off, one = U.offsets([1]), torch.ones(1, dtype=torch.int32, device="cuda")
    bits = torch.ones((n, 1), dtype=torch.int32, device="cuda")
    act = lambda: torch.ones((n, 2, 64), device="cuda")
    lse = torch.zeros((n, 2), device="cuda")
    sums = lambda: torch.zeros((1, 2, SIZE // 8), device="cuda")
    q1 = torch.ones((1, 2, 64), device="cuda")
    return {
        "tree": (act, lambda q, s: P.crvq_cache_tree_attention(gpu, q, bits, q_off=off, stream=s)),
        "mask": (lambda: torch.ones((1, SIZE // 4), dtype=torch.int32, device="cuda"),
                 lambda m, s: P.crvq_cache_tree_attention(gpu, q1, m, q_off=off, stream=s)),
        "parents": (lambda: torch.full((SIZE // 4,), -1, dtype=torch.int32, device="cuda"),
                    lambda p, s: P.crvq_tree_mask(p, 1, off=off, max_new=1, stream=s)),
        "weights q": (act, lambda q, s: P.crvq_cache_weights(gpu, q, lse, q_off=off, stream=s)),
        "weights before": (sums, lambda w, s: P.crvq_cache_weights(gpu, q1, lse[:1], q_off=off, weights=w, stream=s)),
        "select": (sums, lambda w, s: P.crvq_cache_select(w, gpu.lens, 5, stream=s)),
        "keep": (lambda: torch.zeros((1, 2, SIZE // 8), dtype=torch.int32, device="cuda"),
                 lambda i, s: P.crvq_cache_keep(gpu, i, one, stream=s)),
    }


@pytest.mark.parametrize("name", ["tree", "mask", "parents", "weights q", "weights before", "select", "keep"])
def test_inputs_outlive_a_call_on_a_stream_of_its_own(name):
    import paper_2412_09282_gb300 as P
    make, call = _stream_calls()[name]
    assert not _again(make, call)
    P.crvq_sync()
