"""tpla_commit_drafts where pages of drafts were missing (negative entries of the block table): the path ends before the first draft
that has no row, and nothing outside the pools is read or written."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from test_gpu_token_tables import shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,g,dl,pt,dtype", [(1, 1, 256, 64, "bf16"), (8, 2, 256, 4, "bf16"), (64, 4, 128, 16, "bf16"), (64, 1, 64, 1, "bf16"), (13, 2, 72, 3, "f32")])
@pytest.mark.parametrize("in_place", [False, True])
def test_the_path_ends_where_a_page_is_missing(T, g, dl, pt, dtype, in_place):
    B, d_r = 6, 64
    r = np.random.default_rng([T, g, pt])
    lens = [0, pt, 2 * pt + pt // 2, 5 * pt - 1, 7, 33]
    pages = [-(-(n + T) // pt) for n in lens]
    mp, n_pool = max(pages) + 1, sum(pages)
    order, k = r.permutation(n_pool), 0
    bt = np.full((B, mp), -1, dtype=np.int32)
    for b in range(B):
        bt[b, :pages[b]] = order[k:k + pages[b]]
        k += pages[b]
    bt[0, :] = -7                                              # no page at all
    bt[1, 1:] = np.iinfo(np.int32).min                         # none of the drafts
    bt[2, -(-lens[2] // pt):] = -1                             # those behind the committed page
    if pages[3] > 6:
        bt[3, 6] = -2                                          # one page in the middle
    acc, n_acc = np.zeros((B, T), dtype=np.int32), []
    for b in range(B):
        n = [T, T, T, T, max(1, T // 2), T // 3][b]
        acc[b, :n] = np.sort(r.choice(T, n, replace=False))
        acc[b, n:] = r.integers(-5, 2 * T, T - n)
        n_acc.append(n)
    st = torch.float32 if dtype == "f32" else torch.bfloat16
    guarded = [torch.from_numpy(r.standard_normal((n_pool + 2 * mp, pt, dl + d_r)).astype(np.float32)).cuda().to(st) for _ in range(g)]
    pools = [x[mp:mp + n_pool] for x in guarded]
    want = [x.cpu().clone() for x in guarded]
    new_want = []
    for b in range(B):
        n = 0
        while n < n_acc[b] and bt[b, (lens[b] + n) // pt] >= 0 and bt[b, (lens[b] + int(acc[b, n])) // pt] >= 0:
            n += 1
        new_want.append(lens[b] + n)
        at = lambda t: (mp + int(bt[b, t // pt]), t % pt)  # noqa: E731
        for w, x in zip(want, guarded):
            old = x.cpu()
            for j in range(n):
                w[at(lens[b] + j)] = old[at(lens[b] + int(acc[b, j]))]
    assert new_want[0] == 0 and new_want[1] == pt and new_want[4] == 7 + n_acc[4]
    dev = lambda v: torch.tensor(np.asarray(v, dtype=np.int32)).cuda()  # noqa: E731
    ln = dev(lens)
    new = ln if in_place else torch.full((B,), -7, dtype=torch.int32, device="cuda")
    print("commit without pages", T, g, dl, pt, dtype, in_place, flush=True)
    tp.tpla_commit_drafts(shape(B, pt, g, dl, d_r, tp.TPLA_F32 if dtype == "f32" else tp.TPLA_BF16), T, dev(acc), dev(n_acc), ln, dev(bt), mp, pools, new)
    torch.cuda.synchronize()
    assert new.tolist() == new_want
    bits = torch.int32 if dtype == "f32" else torch.int16
    for w, x in zip(want, guarded):
        assert torch.equal(w.view(bits), x.cpu().view(bits))
