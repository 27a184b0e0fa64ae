"""Which tokens stay in a cache that is cut down to a budget: places, counts and their weights, equal to the oracle's."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as C

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).cuda()


def _same(a, b):
    return np.array_equal(np.asarray(a) + 0.0, np.asarray(b) + 0.0, equal_nan=True)


def _check(w, lens, keep, first=0, recent=0, out_width=None):
    import paper_2412_09282_gb300 as P
    idx_ref, count_ref, w_ref = C.select(w, lens, keep, first, recent)
    n_seq, n_kv, width = w.shape
    out = torch.full((n_seq, n_kv, out_width or width), np.nan, device="cuda")
    gw = torch.from_numpy(w).cuda()
    idx, count = P.crvq_cache_select(gw, _ints(lens), keep, first=first, recent=recent, weights_out=out)
    P.crvq_sync()
    assert np.array_equal(count.cpu().numpy(), count_ref)
    assert np.array_equal(idx.cpu().numpy(), idx_ref)
    ref = np.zeros(out.shape, np.float32)
    ref[:, :, :min(width, ref.shape[2])] = w_ref[:, :, :ref.shape[2]]
    assert _same(out.cpu().numpy(), ref)
    assert _same(gw.cpu().numpy(), w)
    return idx


def _sums(seed, shape):
    """A few tokens with most of it, some with nothing."""
    rng = np.random.default_rng(seed)
    return (np.exp(2.0 * rng.standard_normal(shape)) * (rng.random(shape) > 0.1)).astype(np.float32)


@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (7, 4, 3), (16, 4, 3), (100, 0, 90), (300, 4, 64), (500, 0, 0)])
def test_ragged_lengths(keep, first, recent):
    lens = [0, 1, 2, 6, 7, 8, 31, 33, 100, 127, 300, 301, 499]
    _check(_sums(1, (len(lens), 3, 500)), lens, keep, first, recent)


@pytest.mark.parametrize("width,keep", [(1025, 1000), (4096, 17), (4097, 2000), (8200, 1), (16500, 9000), (70001, 4096)])
def test_rows_of_one_to_eight_ctas(width, keep):
    """Rows of one, two, four and eight CTAs, of full length and shorter ones in the same call."""
    _check(_sums(2, (3, 2, width)), [width, width - 1, max(1, width // 9)], keep, min(4, keep // 2), keep // 3)


def test_rows_longer_than_shared_memory():
    rng = np.random.default_rng(3)
    w = rng.random((1, 1, 420000), np.float32)
    _check(w, [420000], 5000, 4, 1000)
    _check(w, [399999], 390000, 0, 7)


def test_ties_go_to_the_lowest_place():
    rng = np.random.default_rng(4)
    for width in (90, 5000, 40000):
        few = rng.integers(0, 3, (2, 2, width)).astype(np.float32)
        for keep in (1, width // 3, width // 2 + 1, width - 1):
            _check(few, [width, width - 2], keep, min(1, keep // 2), keep // 4)
        same = np.full((1, 2, width), 0.25, np.float32)
        idx = _check(same, [width], width // 2, 3, 10)
        assert idx[0, 0, -11].item() == width // 2 - 11         # the ones in front, and the 10 last


def test_neighbouring_values_signs_infinities_and_nan():
    rng = np.random.default_rng(5)
    for width in (200, 6000):
        base = rng.choice(np.float32([0.0, -0.0, 1e-45, -1e-45, 1.0, 1.0000001, 0.99999994, -1.0, -1.0000001, np.inf, -np.inf,
                                      np.nan, 3e38, -3e38, 1e-38]), (2, 2, width))
        for keep in (5, width // 4, width // 2, 3 * width // 4, width - 1):
            _check(base, [width, width - 5], keep, min(2, keep // 2), min(3, keep // 2))
        bits = (np.float32(1.0).view(np.uint32) + rng.integers(0, 4000, (2, 2, width))).astype(np.uint32).view(np.float32)
        _check(bits, [width, width], width // 3, 1, 1)


def test_nothing_between_the_first_and_the_recent():
    _check(_sums(6, (3, 2, 100)), [100, 20, 19], 20, 8, 12)
    _check(_sums(6, (1, 1, 5000)), [5000], 4000, 4000, 0)
    _check(_sums(6, (1, 1, 5000)), [5000], 4000, 0, 4000)


def test_more_to_keep_than_there_is_room_for_and_narrow_results():
    _check(_sums(7, (2, 2, 64)), [64, 10], 200, 100, 100)
    _check(_sums(7, (2, 2, 64)), [64, 10], 20, 4, 4, out_width=20)
    _check(_sums(7, (2, 2, 64)), [64, 10], 20, 4, 4, out_width=333)


def test_many_rows():
    rng = np.random.default_rng(8)
    _check(_sums(9, (70, 32, 260)), rng.integers(0, 261, 70).tolist(), 100, 4, 20)


def test_views_and_results_of_the_callers_own():
    import paper_2412_09282_gb300 as P
    w = _sums(10, (2, 3, 50))
    buf = torch.full((3, 2, 70), 5.0, device="cuda")
    view = buf.transpose(0, 1)[:, :, 3:53]
    view.copy_(torch.from_numpy(w))
    out = torch.full((2, 4, 60), 5.0, device="cuda")
    idx, count = torch.empty((2, 3, 9), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    a, b = P.crvq_cache_select(view, _ints([50, 41]), 9, first=1, recent=2, weights_out=out[:, :3, 1:41], idx_out=idx, count_out=count)
    P.crvq_sync()
    ri, rc, rw = C.select(w, [50, 41], 9, 1, 2)
    assert a is idx and b is count and np.array_equal(idx.cpu().numpy(), ri) and np.array_equal(count.cpu().numpy(), rc)
    assert np.array_equal(out[:, :3, 1:41].cpu().numpy(), rw[:, :, :40])
    assert (out[:, 3] == 5).all() and (out[:, :, 0] == 5).all() and (out[:, :, 41:] == 5).all()
    a, _ = P.crvq_cache_select(view, _ints([50, 41]), 9, first=1, recent=2)      # without weights
    P.crvq_sync()
    assert np.array_equal(a.cpu().numpy(), ri)


def test_bad_lengths_are_reported_and_count_as_zero():
    import paper_2412_09282_gb300 as P
    w = torch.from_numpy(_sums(11, (3, 1, 40))).cuda()
    idx, count = P.crvq_cache_select(w, _ints([41, 30, -1]), 8)
    with pytest.raises(P.CrvqError) as e:
        P.crvq_sync()
    assert e.value.status == -7
    assert count.tolist() == [0, 8, 0] and (idx[[0, 2]] == -1).all()
    assert np.array_equal(idx[1].cpu().numpy(), C.select(w.cpu().numpy(), [0, 30, 0], 8, 0, 0)[0][1])


def test_refusals():
    import paper_2412_09282_gb300 as P
    w, lens = torch.zeros((2, 2, 48), device="cuda"), _ints([40, 20])
    for kw in (dict(keep=0), dict(keep=-3), dict(keep=8, first=5, recent=4), dict(keep=8, first=-1), dict(keep=8, recent=-1),
               dict(keep=8, weights_out=w), dict(keep=8, weights_out=w[:, :, :7].clone()),
               dict(keep=8, weights_out=w.as_strided((2, 2, 48), (48, 48, 1)))):
        with pytest.raises(P.CrvqError) as e:
            P.crvq_cache_select(w, lens, **kw)
        assert e.value.status == -1
    for args in ((w.double(), lens), (w[0], lens), (w, lens[:1]), (w, lens.long()), (w.cpu(), lens), (w.transpose(1, 2), lens)):
        with pytest.raises((TypeError, ValueError)):
            P.crvq_cache_select(*args, 8)
    with pytest.raises(ValueError):
        P.crvq_cache_select(w, lens, 8, idx_out=torch.zeros((2, 2, 9), dtype=torch.int32, device="cuda"))


def test_a_captured_call_replays_with_new_weights_and_lengths():
    import paper_2412_09282_gb300 as P
    w, lens = torch.zeros((2, 2, 9000), device="cuda"), _ints([1, 1])
    P.crvq_cache_select(w, lens, 700, first=4, recent=9)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        idx, count = P.crvq_cache_select(w, lens, 700, first=4, recent=9)
    for seed, n in ((12, [9000, 300]), (13, [701, 8999])):
        x = _sums(seed, (2, 2, 9000))
        w.copy_(torch.from_numpy(x))
        lens.copy_(_ints(n))
        g.replay()
        P.crvq_sync()
        ref, rc, _ = C.select(x, n, 700, 4, 9)
        assert np.array_equal(idx.cpu().numpy(), ref) and np.array_equal(count.cpu().numpy(), rc)


@pytest.mark.parametrize("rows,width", [((1, 1), 3000), ((3, 70), 3001), ((2, 2), 30000), ((40, 4), 9001), ((1, 1), 400000)])
def test_weights_that_share_their_first_digits(rows, width):
    """Keys that agree in 11, 18 and 25 bits, more of them than a warp lists, beside rows where few do; of every number of
    tokens a warp takes (rows of SMs to themselves, and several on one)."""
    rng = np.random.default_rng(140)
    w = np.empty(rows + (width,), np.float32)
    flat = w.reshape(-1, width)
    for r in range(flat.shape[0]):
        near = [0.2, 2.0 ** -10, 2.0 ** -17, 2.0 ** -22, 0.0, 8.0][r % 6]
        flat[r] = (1 + near * rng.random(width)).astype(np.float32)
        if r % 4 == 3:
            flat[r, rng.integers(0, width, width // 3)] *= np.float32(0.01)
    lens = [width - 17 * b for b in range(rows[0])]
    for keep, first, recent in ((1000, 0, 0), (1500, 3, 200)):
        _check(w, lens, keep, first, recent)


def test_room_for_more_tokens_than_there_can_be():
    """The largest keep: 2^31 - 1 places a row, -1 behind the last token up to the end."""
    import paper_2412_09282_gb300 as P
    w = torch.rand((1, 1, 100), device="cuda")
    keep = 2 ** 31 - 1
    idx, count = P.crvq_cache_select(w, _ints([77]), keep)
    P.crvq_sync()
    assert count.item() == 77 and torch.equal(idx[0, 0, :77], torch.arange(77, dtype=torch.int32, device="cuda"))
    assert int(idx[0, 0, 77:].max()) == int(idx[0, 0, 77:].min()) == -1
