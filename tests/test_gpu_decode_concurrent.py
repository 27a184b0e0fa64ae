"""The decode step's calls from several streams and host threads at once, over one cache and one matrix: bit for bit what they
return one after another. Each call's scratch is its own stream's."""
import threading

import numpy as np
import pytest
import torch

import decode_util as U
import test_gpu_attention as T

pytestmark = pytest.mark.gpu


def _work():
    """Calls without arguments, each of which returns new tensors: attention in every form, reads, products, a quantizer."""
    import paper_2412_09282_gb300 as P
    lens = [900, 3, 2000, 0, 513]
    _, bf = U.make(98, lens, 16, 2, 128, "int8", wide=1200)
    _, short = U.make(99, [300, 40], 16, 2, 64, "e4m3")
    one = U.heads(T._queries(100, 5, 8, 128, "f32"), "f32")
    chunk = U.heads(T._queries(101, 5 * 70, 8, 128, "bf16"), "bf16")
    few = U.heads(T._queries(102, 6, 4, 64, "f16"), "f16")
    start, off = torch.zeros(5, dtype=torch.int32, device="cuda"), U.offsets(lens)
    g = torch.Generator(device="cuda").manual_seed(103)
    W = torch.randn((2000, 1500), generator=g, device="cuda")
    m, _ = P.crvq_q4_quantize(W)
    X = torch.randn((20, 1500), generator=g, device="cuda")
    P.crvq_sync()
    return [lambda: P.crvq_cache_attention(bf, one), lambda: P.crvq_cache_attention(bf, chunk),
            lambda: P.crvq_cache_attention(short, few), lambda: P.crvq_cache_read(bf, start, off, sum(lens))[1],
            lambda: P.crvq_q4_matvec(X, m), lambda: P.crvq_q4_matvec(X[:1], m),
            lambda: P.crvq_q4_quantize(W, want_W_hat=True)[1]]


def test_streams_and_threads():
    calls = _work()
    ref = [f().clone() for f in calls]
    torch.cuda.synchronize()
    wrong, errors = [], []

    def lane(j):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for i in range(60):
                    k = (i * (j + 1) + j) % len(calls)
                    out = calls[k]()
                    if not torch.equal(out, ref[k]):
                        wrong.append((j, i, k))
        except Exception as e:  # (a thread's exception would be lost)
            errors.append(e)

    lanes = [threading.Thread(target=lane, args=(j,)) for j in range(4)]
    for t in lanes:
        t.start()
    for t in lanes:
        t.join()
    torch.cuda.synchronize()
    assert not errors and not wrong, (errors, wrong)


def test_appends_to_different_sequences_from_two_streams():
    """Two handles over one pool of pages, a sequence each."""
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(104, [5, 7], 16, 2, 64, "int8", wide=4, spare=8)
    used = set(host["pages"][:, 0].tolist())
    free = [p for p in range(10) if p not in used]
    pages = np.stack([np.array([host["pages"][b, 0]] + free[3 * b:3 * b + 3], np.int32) for b in range(2)])
    rng = np.random.default_rng(105)
    x = [U.heads(rng.standard_normal((40, 2, 64)).astype(np.float32), "f32") for _ in range(4)]

    def run(streams):
        K, V, ks, vs = (t.clone() for t in (gpu.K, gpu.V, gpu.k_scale, gpu.v_scale))
        caches = [P.KVCache(K, V, ks, vs, torch.from_numpy(pages[b:b + 1].copy()).cuda(),
                            torch.tensor([45 + 2 * b], dtype=torch.int32, device="cuda")) for b in range(2)]
        torch.cuda.synchronize()
        for _ in range(20):
            for b in range(2):
                with torch.cuda.stream(streams[b]):
                    P.crvq_cache_append(caches[b], x[2 * b], x[2 * b + 1])
        torch.cuda.synchronize()
        return [U.exactly(t) for t in (K, V, ks, vs)]

    main = torch.cuda.current_stream()
    for a, b in zip(run([main, main]), run([torch.cuda.Stream(), torch.cuda.Stream()])):
        assert np.array_equal(a, b, equal_nan=True)
