"""Calls on a stream that the caller gives: the memory of tensors that are dropped right after the call is not handed out
again before that stream has passed it. Inputs are made on the current stream, the given one is kept busy, and the
next tensor of an input's size has to lie elsewhere."""
import pytest
import torch

import decode_util as U

pytestmark = pytest.mark.gpu

SIZE = 1 << 22                                                   # (of a block of its own in the allocator's pool)


def _again(make, call):
    """Whether the memory of make()'s tensor is handed out again while call(tensor, stream) waits on its stream."""
    s = torch.cuda.Stream()
    call(make(), s)                                              # (a first call loads its kernel, which waits)
    torch.cuda.synchronize()
    x = make()
    at, n, dt = x.data_ptr(), x.untyped_storage().nbytes(), torch.uint8
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    out = call(x, s)
    del x
    pending = not s.query()
    new = [torch.empty(n, dtype=dt, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert pending and out is not None
    return any(t.data_ptr() == at for t in new)


def _calls():
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(106, [20], 16, 2, 64, "int8", wide=1100)
    n = SIZE // (2 * 64 * 4)
    m = P.Q4Matrix.empty(64, SIZE // 4, 128)
    m.codes.zero_(), m.scales.zero_()
    k = torch.ones((1, 2, 64), device="cuda")
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    act = lambda: torch.ones((n, 2, 64), device="cuda")
    off = U.offsets([1])

    def attend(q, s):
        return P.crvq_cache_attention(gpu, q, q_off=off, stream=s)

    def append(q, s):  # (queries beside one new token: rows past the sequence's stay as they are)
        kk = torch.ones((q.shape[0], 2, 64), device="cuda")
        return P.crvq_cache_append(gpu, kk, kk, new_off=off, q=q, q_out=q2, stream=s)

    q2 = act()
    return {
        "attention": (act, attend),
        "append q": (act, append),
        "append tables": (lambda: torch.ones((SIZE // 128, 32), device="cuda"),
                          lambda t, s: P.crvq_cache_append(gpu, k, k, cos=t, sin=t, positions=one, q=k, stream=s)),
        "matvec": (lambda: torch.ones((1, SIZE // 4), device="cuda"), lambda x, s: P.crvq_q4_matvec(x, m, stream=s)),
        "quantize": (lambda: torch.ones((1024, SIZE // 4096), device="cuda"), lambda w, s: P.crvq_q4_quantize(w, stream=s)),
        "read": (lambda: torch.zeros(SIZE // 4, dtype=torch.int32, device="cuda"),
                 lambda t, s: P.crvq_cache_read(gpu, t[:1], off, 1, stream=s)),
        "matrix": (lambda: torch.zeros((64, SIZE // 64), dtype=torch.uint8, device="cuda"),
                   lambda c, s: P.crvq_q4_matvec(torch.ones((1, SIZE // 32), device="cuda"), P.Q4Matrix(
                       c, torch.ones((64, SIZE // 32 // 128), device="cuda", dtype=torch.bfloat16), None, SIZE // 32, 128), stream=s)),
    }


@pytest.mark.parametrize("name", ["attention", "append q", "append tables", "matvec", "quantize", "read", "matrix"])
def test_inputs_outlive_the_call_on_its_stream(name):
    import paper_2412_09282_gb300 as P
    make, call = _calls()[name]
    assert not _again(make, call)
    P.crvq_sync()
