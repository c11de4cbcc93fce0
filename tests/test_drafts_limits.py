"""Host side of the speculative step's entry points: sizes that the kernels' launches and index arithmetic do not hold are refused
before anything is launched."""
import pytest

import paper_2508_15881_amd as tp
from test_drafts_host import A, BIG, code, shape


@pytest.mark.parametrize("dtype,g", [(tp.TPLA_BF16, 1), (tp.TPLA_BF16, 2), (tp.TPLA_F32, 1)])
@pytest.mark.parametrize("pt,max_pages", [(1, 2 ** 31 - 1), (1, 2 ** 31 - 2 ** 17 + 1), (64, 2 ** 25 - 1), (2 ** 20, 2 ** 11 - 1)])
def test_rows_whose_token_numbers_pass_31_bits(dtype, g, pt, max_pages):
    s = shape(B=1, H=4, d_c=256 * g, g=g, page_tokens=pt, dtype=dtype)
    args = [s, 4, A, A, [A] * g, A, max_pages, A, A, A, A, BIG, A, A]
    most = 2 ** 31 - 2 ** 17
    assert (tp.tpla_workspace_bytes_tree(s, 4, max_pages) == 0) == (pt * max_pages > most)
    if pt * max_pages > most:
        assert code(tp.tpla_decode_shards_tree, *args) == -7
        assert code(tp.tpla_decode_shard_tree, *(args[:4] + [A] + args[5:])) == -7
    assert tp.tpla_workspace_bytes_tree(s, 4, most // pt) > 0
