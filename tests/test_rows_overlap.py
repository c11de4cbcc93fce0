"""Outputs whose rows share memory are refused, whichever of tokens and heads is the inner dimension (CPU)."""
import numpy as np
import pytest

import paper_2508_15881_amd as tp
from test_heads_limits import A, append, norm, shape

# token stride, head stride in rows of the width, tokens, heads
LAYOUTS = [(1, 1, 4, 8), (2, 1, 4, 8), (7, 1, 4, 8), (8, 1, 4, 8), (1, 4, 4, 8), (1, 3, 4, 8), (3, 2, 2, 2), (3, 2, 2, 4), (3, 2, 3, 2), (3, 2, 2, 3), (4, 6, 3, 2), (4, 6, 4, 4), (5, 5, 1, 8), (5, 5, 9, 1), (1, 9, 9, 2),
           (1.5, 1.25, 2, 2), (1.5, 2.5, 2, 2), (1.5, 2.5, 4, 3), (2.5, 6.25, 3, 2), (2.5, 6.25, 2, 2), (1000, 1, 4, 8), (1, 2 ** 40, 4, 8)]


def shared(width, ts, hs, T, heads):
    """Whether two rows share an element, by where each begins."""
    at = np.sort((np.arange(T)[:, None] * int(ts * width) + np.arange(heads) * int(hs * width)).ravel())
    return bool((np.diff(at) < width).any())


@pytest.mark.parametrize("ts,hs,T,heads", LAYOUTS)
@pytest.mark.parametrize("d", [64, 128])
def test_grouped_heads(ts, hs, T, heads, d):
    """Refused as what it is, or the next check's turn (a misaligned weight, a NULL pool)."""
    strides = (A, int(ts * d), int(hs * d))
    want = -2 if shared(d, ts, hs, T, heads) else -3
    s = shape(H=heads, H_kv=heads, d_k=d, d_v=d)
    dense = (8 * A, heads * d, d)
    assert norm(s, rot=d, T=T, q=dense, qo=strides, k=dense, ko=(A + 2, heads * d, d)) == want
    assert norm(s, rot=d, T=T, q=dense, qo=dense, k=(A + 2, heads * d, d), ko=strides) == -3              # (inputs first)
    if want == -2:
        assert norm(s, rot=d, T=T, q=(None, 0, 0), qo=(None, 0, 0), k=(8 * A, heads * d, d), ko=strides) == -2
    assert append(s, rot=d, T=T, q=dense, qo=strides, k=dense, v=dense, kp=A + 8) == want


def test_many_tokens_and_heads():
    """Decided without a walk over them where one dimension lies within a step of the other, and in steps of the smaller one otherwise."""
    d = 128
    s = shape(H=65535, H_kv=1, d_k=d, d_v=d)
    T = 2 ** 31 - 1
    big = lambda ts, hs: append(s, T=T, q=(8 * A, 65535 * d, d), qo=(A, ts, hs), k=(A, d, d), v=(A, d, d), kp=A + 8)  # noqa: E731
    assert big(65535 * d, d) == -3 and big(d, T * d) == -3 and big(65534 * d, d) == -2 and big(d, (T - 1) * d) == -2
    assert big(65535 * d, 65536 * d) == -3 and big(65534 * d, 65536 * d) == -2 and big(2 * d, (2 * T - 1) * d) == -3 and big(2 * d, 3 * d) == -2
    assert big(2 ** 62, 2 ** 62) == -2
