"""What crvq_cache_append refuses of its tables and positions, before anything is launched."""
import pytest
import torch

import decode_util as U

pytestmark = pytest.mark.gpu


def _call(**kw):
    import paper_2412_09282_gb300 as P
    host, gpu = U.make(90, [4, 4], 16, 2, 64, "int8")
    k = torch.ones((2, 2, 64), device="cuda")
    return P.crvq_cache_append(gpu, k, k, **kw)


@pytest.mark.parametrize("stride", [0, 1, 16, 31])
def test_tables_whose_rows_overlap_are_refused(stride):
    """n_pos rows of half entries, further apart than their length: a broadcast row has no such memory."""
    import paper_2412_09282_gb300 as P
    row = torch.ones(31 * 8 + 32, device="cuda")
    tab = row.as_strided((9, 32), (stride, 1))
    with pytest.raises(P.CrvqError) as e:
        _call(cos=tab, sin=tab)
    assert e.value.status == -1


def test_a_table_of_one_row_may_have_any_stride():
    import paper_2412_09282_gb300 as P
    tab = torch.ones((32,), device="cuda").expand(1, 32)
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    _call(cos=tab, sin=tab, positions=zero)
    P.crvq_sync()


def test_half_of_the_tables_and_positions_without_them_are_refused():
    tab = torch.ones((9, 32), device="cuda")
    for kw in (dict(cos=tab), dict(sin=tab), dict(positions=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            _call(**kw)
