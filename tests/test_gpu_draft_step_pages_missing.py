"""The speculative step when the free pages run out in its middle, eager and as one captured graph of placing, attention and commit:
what has no page is seen by nobody and not committed, and a later step with more pages goes on from there."""
import numpy as np
import pytest
import torch

from draft_common import TreeProblem
from paper_2508_15881_amd import pipeline as pl
from test_gpu_draft_step import Loop

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,T,pt,captured", [("bf16", 16, 20, 16, False), ("bf16", 16, 20, 16, True), ("bf16", 64, 12, 4, True), ("f32", 4, 12, 4, True)])
def test_a_step_that_runs_out_of_pages(dtype, H, T, pt, captured):
    s = Loop(dtype, H, T, pt, seed=11, dl=256 if dtype == "bf16" else 32, d_r=64 if dtype == "bf16" else 16) if pt == 16 else small_pages(dtype, H, T, pt)
    print("step without pages", dtype, H, T, pt, captured, flush=True)
    s.table[s.table < 0] = 0                                   # as a zeroed table is, or one that was used before
    step, x = s.step, s.inputs()
    chain = np.tile(np.arange(-1, T - 1), (3, 1))
    masks_np, depths = pl.tree_masks(chain)
    masks, depth_dev = torch.from_numpy(masks_np.view(np.int64)).cuda(), torch.from_numpy(depths).cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    n_dev, acc, n_acc = ints([T, T, T]), torch.arange(T, dtype=torch.int32, device="cuda").repeat(3, 1), ints([T, T, T])
    new = torch.zeros(3, dtype=torch.int32, device="cuda")
    free = s.free[:2].clone()                                  # too few
    lens, held, table, pools = s.lens.tolist(), s.held.clone(), s.table.clone(), [p.clone() for p in s.pools]

    def whole():
        step.place(s.lens, n_dev, depth_dev, free, free.numel(), s.held, s.table)
        o = step.run(x["q_nope"], x["q_pe"], x["c_t"], x["k_pe"], s.W_UK, s.W_UV, s.pools, s.table, s.lens, n_dev, masks)
        step.commit(acc, n_acc, s.lens, new, s.table, s.pools)
        return o

    if captured:
        whole()                                                # (kernel attributes are set on first use)
        torch.cuda.synchronize()
        s.held.copy_(held)
        s.table.copy_(table)
        for p, q in zip(s.pools, pools):
            p.copy_(q)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            whole()
        graph.replay()
    else:
        whole()
    torch.cuda.synchronize()
    assert step.counts.tolist()[0] == 2 and step.counts.tolist()[1] > 0
    placed = [min(T, h * pt - n) for h, n in zip(s.held.tolist(), lens)]
    assert min(placed) < T and new.tolist() == [n + k for n, k in zip(lens, placed)]
    assert (step.slots.cpu().numpy().reshape(3, T) >= 0).sum(1).tolist() == placed
    p = object.__new__(TreeProblem)
    p.shape, p.T, p.g, p.dtype, p.lens, p.drafts, p.max_pages = s.shape, T, 2, dtype, lens, [T] * 3, s.max_pages
    p.masks = np.stack([masks_np[b] & np.uint64((1 << placed[b]) - 1) for b in range(3)])
    p.q_lat, p.q_pe = pl.from_device_bits(step.q_lat), pl.from_device_bits(step.q_pe.reshape(3, T, H, s.d_r))
    p.pools, p.bt = [pl.from_device_bits(q) for q in s.pools], s.table.cpu().numpy()
    want, want_lse, off, lse_off = p.expected()
    fin = np.isfinite(want_lse)
    got, got_lse = step.o_lat.double().cpu().numpy(), step.lse.double().cpu().numpy()
    assert (np.abs(got - want) <= off).all()
    assert np.array_equal(np.isfinite(got_lse), fin) and (np.abs(got_lse[fin] - want_lse[fin]) <= lse_off[fin]).all()
    # nothing but the placed drafts' rows was written
    for q, old in zip(s.pools, pools):
        mine = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
        for b in range(3):
            for t in range(lens[b], lens[b] + placed[b]):
                mine[int(s.table[b, t // pt]), t % pt] = True
        bits = torch.int32 if dtype == "f32" else torch.int16
        assert torch.equal(q.view(bits)[~mine], old.view(bits)[~mine]) and not torch.isnan(q[mine]).any()
    # more pages: the next step places all of its drafts
    s.lens.copy_(new)
    more = s.free[2:].clone()
    step.place(s.lens, n_dev, depth_dev, more, more.numel(), s.held, s.table)
    torch.cuda.synchronize()
    assert step.counts.tolist()[1] == 0 and (step.slots >= 0).all() and len(set(step.slots.tolist())) == 3 * T


def small_pages(dtype, H, T, pt):
    """Loop has sixteen pages a row: contexts short enough for pages of four tokens."""
    s = Loop(dtype, H, T, 16, seed=12, dl=256 if dtype == "bf16" else 32, d_r=64 if dtype == "bf16" else 16)
    s.pt = pt
    s.shape.page_tokens = pt
    lens = [13, 0, 20]
    held = [-(-n // pt) for n in lens]
    n_pool = 48
    order = s.r.permutation(n_pool).astype(np.int32)
    table = np.full((3, s.max_pages), -1, dtype=np.int32)
    k = 0
    for b in range(3):
        table[b, :held[b]] = order[k:k + held[b]]
        k += held[b]
    s.free = torch.from_numpy(order[k:].copy()).cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    s.lens, s.held, s.table = ints(lens), ints(held), torch.from_numpy(table).cuda()
    s.pools = [torch.full((n_pool, pt, s.dl + s.d_r), float("nan"), device="cuda").to(s.st) for _ in range(2)]
    for b in range(3):
        for t in range(lens[b]):
            for p in s.pools:
                p[int(table[b, t // pt]), t % pt] = torch.from_numpy(s.r.standard_normal(s.dl + s.d_r)).cuda().to(s.st)
    s.step = pl.DraftStep(s.shape, T, s.max_pages, s.freq)
    return s
