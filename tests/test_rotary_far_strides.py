"""tpla_apply_rotary refuses strides whose byte offsets do not fit 64 bits (CPU)."""
import ctypes

import pytest

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import binding
from test_drafts_host import A, shape


@pytest.mark.parametrize("dtype,esz", [(tp.TPLA_BF16, 2), (tp.TPLA_F32, 4)])
@pytest.mark.parametrize("which", range(6))
def test_far_strides(dtype, esz, which):
    """Or the next check's turn (positions that are not aligned)."""
    s, d = shape(H=4, d_r=64, dtype=dtype), 64
    for stride in (2 ** 40, 2 ** 58 // esz, 2 ** 61, 2 ** 62, 2 ** 63 - 64):
        strides = [4 * d, d, 4 * d, d, d, d]
        strides[which] = stride
        q_ts, q_hs, qo_ts, qo_hs, k_ts, ko_ts = strides
        rc = binding.load_library().tpla_apply_rotary(ctypes.byref(s), tp.TPLA_ROTARY_HALF, 0, d, A, 1.0, A + 4, 2, 8 * A, q_ts, q_hs, A, qo_ts, qo_hs, 32 * A, k_ts, 64 * A,
                                                      ko_ts, None)
        assert rc == (-3 if stride < 2 ** 59 else -2), (stride, tp.tpla_last_error())
