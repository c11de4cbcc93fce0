"""Host side of the speculative step's entry points: sizes that the kernels' launches and index arithmetic do not hold are refused
before anything is launched."""
import numpy as np
import pytest

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import pipeline as pl
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


@pytest.mark.parametrize("dtype,d_v", [(tp.TPLA_F32, 32), (tp.TPLA_BF16, 12), (tp.TPLA_BF16, 128)])
def test_rows_that_the_combine_has_no_launch_for(dtype, d_v):
    """Refused ahead of the attention: the workspace is enough, so the only thing wrong is what follows."""
    s = shape(B=32768, H=1, d_c=64, g=1, d_v=d_v, d_r=64, dtype=dtype)
    need = tp.tpla_workspace_bytes_tree(s, 64, 4)
    assert need > 0
    both = [s, 64, A, A, [A], A, 4, A, A, A, A, need, A, A, dtype, A, A]
    assert code(tp.tpla_decode_shards_tree_combine, *both) == -7 and "grid" in tp.tpla_last_error()


def test_grids_of_more_threads_than_a_launch_has():
    # 2^24 items of 16 rows of the general kernel
    s = shape(B=65535, H=65, d_c=8, g=1, d_r=8, dtype=tp.TPLA_F32)
    assert tp.tpla_workspace_bytes_tree(s, 63, 4) > 0
    assert tp.tpla_workspace_bytes_tree(s, 64, 4) == 0
    assert code(tp.tpla_decode_shards_tree, s, 64, A, A, [A], A, 4, A, A, A, A, BIG, A, A) == -7
    # rows of one sequence
    for dtype in (tp.TPLA_BF16, tp.TPLA_F32):
        s = shape(B=1, H=65536, d_c=64, g=1, dtype=dtype)
        assert tp.tpla_workspace_bytes_tree(s, 64, 4) == 0
        assert code(tp.tpla_decode_shards_tree, s, 64, A, A, [A], A, 4, A, A, A, A, BIG, A, A) == -7
        assert tp.tpla_workspace_bytes_tree(shape(B=1, H=65535, d_c=64, g=1, dtype=dtype), 64, 4) > 0
    assert code(tp.tpla_commit_drafts, shape(B=1 << 22), 4, A, A, A, A, 8, [A, A], A) == -7


@pytest.mark.parametrize("parents", [np.arange(-1, 64), np.full((3, 65), -1), np.full(100, -1)])
def test_more_drafts_than_a_mask_has_bits(parents):
    """The 65th draft's own bit was lost, and with it what it sees of itself."""
    with pytest.raises(ValueError):
        pl.tree_masks(parents)
    masks, _ = pl.tree_masks(parents[..., :64])
    assert (masks[..., 63] >> np.uint64(63) == 1).all()


@pytest.mark.parametrize("original,base,fast,slow", [(4, 10000.0, 32.0, 1.0), (1, 10000.0, 32.0, 1.0), (6, 500.0, 32.0, 1.0), (7, 10000.0, 32.0, 1.0), (100, 1e6, 32.0, 16.0),
                                                     (64, 10000.0, 32.0, 1.0), (4096, 10000.0, 32.0, 1.0), (8192, 12.0, 4.0, 1.0), (2 ** 31 - 1, 1e4, 32.0, 1.0)])
def test_frequencies_of_pairs_that_turn_seldom_or_often(original, base, fast, slow):
    for rot in (2, 8, 64, 128):
        f = tp.tpla_rotary_frequencies(rot, base=base, factor=40.0, original_positions=original, beta_fast=fast, beta_slow=slow)
        want = base ** (-2.0 * np.arange(rot // 2) / rot)
        turns = original * want / (2 * np.pi)
        seldom, often = turns <= slow * (1 - 1e-12), turns >= fast * (1 + 1e-12)
        assert np.allclose(f[seldom], want[seldom] / 40, rtol=1e-14, atol=0) and np.allclose(f[often], want[often], rtol=1e-14, atol=0)
        assert (f <= want * (1 + 1e-14)).all() and (f >= want / 40 * (1 - 1e-14)).all()
