"""Attention of drafts whose pages were missing (negative entries of the block table): nobody sees them, and no read leaves the pools."""
import numpy as np
import pytest
import torch

from draft_common import TreeProblem, assert_close, run_all

pytestmark = pytest.mark.gpu

WIDE = 1 << 17


def without_pages(p):
    """Page 0 unused (NaN), the pages behind the one that holds the last committed token absent: masks as the definition then has them."""
    first = [-(-n // p.shape.page_tokens) for n in p.lens]
    used = {int(v) for b, (n, m) in enumerate(zip(p.lens, p.drafts)) for v in p.bt[b, :-(-(n + m) // p.shape.page_tokens)]}
    free = next(k for k in range(p.pools[0].shape[0]) if k not in used)
    if 0 in used:
        for pool in p.pools:
            pool[[0, free]] = pool[[free, 0]]
        p.bt = np.where(p.bt == 0, free, np.where(p.bt == free, 0, p.bt)).astype(np.int32)
    seen = p.masks.copy()
    for b, n in enumerate(p.lens):
        there = [j for j in range(p.drafts[b]) if n + j < first[b] * p.shape.page_tokens]
        p.masks[b] &= np.uint64(sum(1 << j for j in there))
    ref = p.expected()
    p.masks = seen
    return first, ref


@pytest.mark.parametrize("dtype,dl,g,H,T,lens,pt,wide", [
    # 64 rows on four waves
    ("bf16", 256, 2, 16, 4, [30, 32, 0, 127], 16, None), ("bf16", 256, 1, 5, 7, [62, 640, 64], 64, None), ("bf16", 128, 2, 1, 64, [32, 95, 0], 32, None),
    ("bf16", 512, 1, 16, 4, [31, 64, 0], 16, None), ("bf16", 64, 2, 16, 3, [30, 1, 46], 1, None),
    # two teams, up to 128 rows
    ("bf16", 256, 2, 16, 4, [30, 32, 0, 1000], 16, WIDE), ("bf16", 256, 1, 1, 64, [64, 0, 127], 64, WIDE), ("bf16", 256, 1, 16, 6, [95, 64, 0], 32, WIDE),
    ("bf16", 128, 2, 16, 8, [62, 513, 64], 64, WIDE), ("bf16", 64, 4, 16, 8, [30, 64, 0], 1, WIDE),
    # many rows
    ("bf16", 256, 1, 64, 3, [62, 64, 0, 900], 64, WIDE), ("bf16", 128, 1, 64, 4, [62, 64, 0], 64, WIDE), ("bf16", 64, 1, 64, 4, [30, 31, 0], 16, WIDE),
    # the general kernel, short and cut
    ("f32", 32, 2, 4, 5, [126, 60, 0], 64, None), ("f32", 256, 1, 3, 6, [900, 13, 0], 16, None), ("f32", 64, 8, 64, 16, [90, 32], 32, None),
    ("bf16", 72, 2, 6, 5, [62, 3], 64, None), ("f32", 32, 2, 4, 64, [1000, 64], 64, 64),
])
def test_drafts_without_a_page_are_not_seen(dtype, dl, g, H, T, lens, pt, wide):
    d_r = 64 if dtype == "bf16" and dl in (64, 128, 256, 512) else 16
    print("tree without pages", dtype, dl, g, H, T, lens, pt, wide, flush=True)
    p = TreeProblem(lens, [T] * len(lens), T, H=H, g=g, dl=dl, d_r=d_r, pt=pt, dtype=dtype, seed=dl + H + T, max_pages=wide)
    first, ref = without_pages(p)
    p.check_ids()
    d = p.device()
    for b in range(len(lens)):
        d["bt"][b, first[b]:] = -1 - b
    o, lse = run_all(p, d)
    assert_close(p, o, lse, ref)
    if 0 in lens:
        assert (o[:, lens.index(0)] == 0).all() and (lse[:, lens.index(0)] == -np.inf).all()


def test_a_negative_entry_between_pages_that_are_there():
    p = TreeProblem([30, 14], [20, 20], 20, H=4, pt=16, masks=np.full((2, 20), 2 ** 20 - 1, dtype=np.uint64), seed=3)
    keep = p.masks.copy()
    for b, n in enumerate(p.lens):                          # page 2 holds tokens 32 to 47
        p.masks[b] &= np.uint64(sum(1 << j for j in range(20) if (n + j) // 16 != 2))
    ref = p.expected()
    p.masks = keep
    d = p.device()
    d["bt"][:, 2] = torch.iinfo(torch.int32).min
    assert_close(p, *run_all(p, d), ref)
