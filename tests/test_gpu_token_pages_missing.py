"""Calls that run out of pages: what the table says about tokens that have no place."""
import numpy as np
import pytest

from test_gpu_token_tables import assert_same, extend, extend_plain, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,n_free,in_place,add", [(9, 0, False, 60), (9, 1, False, 60), (9, 7, True, 60), (9, 12, True, 3000), (9, 200, False, 3000),
                                                   (1025, 300, False, 60), (1025, 300, True, 60)])
def test_entries_of_missing_pages_are_negative(B, n_free, in_place, add):
    """The rows hold old page ids behind the pages in use, as a table that is used again does."""
    r = np.random.default_rng([B, n_free, add])
    lens, adds, held, table, free = problem(r, B, 16, 50, add)
    table[table < 0] = 0
    args = (16, lens, adds, 0, None, free[:n_free], held, table, sum(adds))
    want = list(extend_plain(*args))
    stale = want[0].copy()
    for b in range(B):
        wanted = max(held[b], min(-(-(lens[b] + adds[b]) // 16), table.shape[1]))
        want[0][b, want[1][b]:wanted] = -1
    assert want[5][1] > 0 and (want[0] != stale).any()
    assert_same(extend(*args, in_place=in_place), want)
