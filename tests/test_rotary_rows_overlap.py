"""tpla_apply_rotary refuses queries whose rows share memory across tokens and heads (CPU)."""
import ctypes

import pytest

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import binding
from test_drafts_host import A, shape
from test_rows_overlap import LAYOUTS, shared


@pytest.mark.parametrize("ts,hs,T,heads", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_queries(ts, hs, T, heads, d):
    """Refused as what it is, or the next check's turn (positions that are not aligned)."""
    s = shape(H=heads, d_r=d)
    rc = binding.load_library().tpla_apply_rotary(ctypes.byref(s), tp.TPLA_ROTARY_HALF, 0, d, A, 1.0, A + 4, T, 8 * A, heads * d, d, A, int(ts * d), int(hs * d),
                                                  None, 0, None, 0, None)
    assert rc == (-2 if shared(d, ts, hs, T, heads) else -3), tp.tpla_last_error()
