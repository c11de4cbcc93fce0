"""The speculative step's operators together, as a serving loop uses them: several steps over the same caches, each checked against
64 bits from what the caches then hold, against the single-token decode, and captured into a graph."""
import math

import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import pipeline as pl
from paper_2508_15881_amd import workloads as wl
from draft_common import HALF, TreeProblem

pytestmark = pytest.mark.gpu


class Loop:
    """Three sequences with committed tokens in scattered pages, a list of free pages, weights."""

    def __init__(self, dtype, H, T, pt=16, seed=0, dl=256, d_r=64):
        self.dtype, self.H, self.T, self.pt, self.B, self.g, self.dl, self.d_r = dtype, H, T, pt, 3, 2, dl, d_r
        self.r = np.random.default_rng([seed, 63])
        self.shape = tp.TplaShape(3, H, 2 * dl, 2, d_r, 128, 128, pt, tp.TPLA_F32 if dtype == "f32" else tp.TPLA_BF16, 1 / math.sqrt(192))
        self.st = pl.torch_dtype(dtype)
        lens = [40, 0, 129]
        self.max_pages, n_pool = 16, 48
        held = [-(-n // pt) for n in lens]
        order = self.r.permutation(n_pool).astype(np.int32)
        table = np.full((3, self.max_pages), -1, dtype=np.int32)
        k = 0
        for b in range(3):
            table[b, :held[b]] = order[k:k + held[b]]
            k += held[b]
        self.free = torch.from_numpy(order[k:].copy()).cuda()
        self.taken = 0
        ints = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        self.lens, self.held, self.table = ints(lens), ints(held), torch.from_numpy(table).cuda()
        self.pools = [torch.full((n_pool, pt, dl + d_r), float("nan"), device="cuda").to(self.st) for _ in range(2)]
        for b in range(3):
            for t in range(lens[b]):
                for p in self.pools:
                    p[int(table[b, t // pt]), t % pt] = torch.from_numpy(self.r.standard_normal(dl + d_r)).cuda().to(self.st)
        draw = lambda *n, s=1.0: torch.from_numpy(self.r.standard_normal(n) * s).cuda().to(self.st)  # noqa: E731
        self.draw = draw
        self.W_UK, self.W_UV = draw(H, 128, 2 * dl, s=0.05), draw(H, 2 * dl, 128, s=0.02)
        self.freq = tp.tpla_rotary_frequencies(d_r, factor=4.0, original_positions=64)
        self.step = pl.DraftStep(self.shape, T, self.max_pages, self.freq)

    def inputs(self):
        n = 3 * self.T
        wide, kv = self.draw(n, self.H, 128 + self.d_r), self.draw(n, 2 * self.dl + self.d_r)
        return dict(q_nope=wide[:, :, :128].contiguous(), q_pe=wide[:, :, 128:], c_t=kv[:, :2 * self.dl].contiguous(), k_pe=kv[:, 2 * self.dl:])

    def trees(self, drafts):
        parents = np.array([[int(self.r.integers(-1, t)) if t else -1 for t in range(self.T)] for _ in range(3)])
        masks, depths = pl.tree_masks(parents)
        return (parents, torch.from_numpy(masks.view(np.int64)).cuda(), torch.from_numpy(depths).cuda(), masks, depths,
                torch.tensor(drafts, dtype=torch.int32).cuda())

    def row(self, i, b, t):
        return self.pools[i][int(self.table[b, t // self.pt]), t % self.pt].double().cpu().numpy()


@pytest.mark.parametrize("dtype,H,T,pt", [("bf16", 16, 6, 16), ("bf16", 64, 4, 64), ("f32", 4, 7, 16)])
def test_steps_of_a_serving_loop(dtype, H, T, pt):
    s = Loop(dtype, H, T, pt, dl=256 if dtype == "bf16" else 32, d_r=64 if dtype == "bf16" else 16)
    half, sh, step = HALF[dtype], s.shape, s.step
    for turn in range(3):
        print("draft step", dtype, H, T, pt, turn, flush=True)
        drafts = [T, max(1, T - 2 - turn), (T + turn) % T + 1]
        parents, masks, depth_dev, masks_np, depths, n_dev = s.trees(drafts)
        x = s.inputs()
        before, lens = s.table.cpu().numpy().copy(), s.lens.tolist()
        free = s.free[s.taken:].clone()
        step.place(s.lens, n_dev, depth_dev, free, free.numel(), s.held, s.table)
        o = step.run(x["q_nope"], x["q_pe"], x["c_t"], x["k_pe"], s.W_UK, s.W_UV, s.pools, s.table, s.lens, n_dev, masks)
        torch.cuda.synchronize()
        s.taken += int(step.counts[0])
        assert int(step.counts[1]) == 0
        table, pos = s.table.cpu().numpy(), step.positions.cpu().numpy().reshape(3, T)
        # the pages held stay, the new ones come off the list in order
        for b in range(3):
            assert (before[b][before[b] >= 0] == table[b][:(before[b] >= 0).sum()]).all()
        new = [int(v) for b in range(3) for v in table[b][(before[b] < 0) & (table[b] >= 0)]]
        assert new == free[:len(new)].tolist() and int(s.held.sum()) == (table >= 0).sum()
        # drafts in the cache: sliced norm of the latent, rotated key
        for b in range(3):
            for t in range(drafts[b]):
                assert pos[b, t] == lens[b] + depths[b, t]
                c, k = x["c_t"].double().cpu().numpy()[b * T + t], x["k_pe"].double().cpu().numpy()[b * T + t]
                a = pos[b, t] * s.freq
                kr = np.stack([k[0::2] * np.cos(a) - k[1::2] * np.sin(a), k[0::2] * np.sin(a) + k[1::2] * np.cos(a)], 1).reshape(-1)
                for i in range(2):
                    ci = c[i * s.dl:(i + 1) * s.dl]
                    want = np.concatenate([ci / np.sqrt(2 * (ci ** 2).sum() / (2 * s.dl) + 1e-6), kr])
                    got = s.row(i, b, lens[b] + t)
                    # float arithmetic over at most 256 terms, then one rounding to the storage type
                    assert (np.abs(got - want) <= half * np.abs(want) + 2.0 ** -18 * (1 + np.abs(want))).all()
        # attention from what is stored: the bound of TreeProblem, then through the value projection
        p = object.__new__(TreeProblem)
        p.shape, p.T, p.g, p.dtype, p.lens, p.drafts, p.masks, p.max_pages = sh, T, 2, dtype, lens, drafts, masks_np, s.max_pages
        p.q_lat, p.q_pe = pl.from_device_bits(step.q_lat), pl.from_device_bits(step.q_pe.reshape(3, T, H, s.d_r))
        p.pools, p.bt = [pl.from_device_bits(q) for q in s.pools], table
        want_lat, want_lse, lat_off, lse_off = p.expected()
        got_lat, got_lse = step.o_lat.double().cpu().numpy(), step.lse.double().cpu().numpy()
        assert (np.abs(got_lat - want_lat) <= lat_off).all()
        fin = np.isfinite(want_lse)
        assert np.array_equal(np.isfinite(got_lse), fin) and (np.abs(got_lse[fin] - want_lse[fin]) <= lse_off[fin]).all()
        W = s.W_UV.double().cpu().numpy()
        cat = lambda v: np.concatenate([v[0], v[1]], axis=-1)  # noqa: E731
        want_o = np.einsum("bthc,hcd->bthd", cat(want_lat), W)
        # the float product of d_c terms carries o_lat in 16 bits at least (2^-16), then the storage type
        off = np.einsum("bthc,hcd->bthd", cat(lat_off) + 2.0 ** -15 * np.abs(cat(want_lat)), np.abs(W)) + half * np.abs(want_o)
        assert (np.abs(o.double().cpu().numpy() - want_o) <= off + 1e-30).all()
        # a path of every tree is accepted
        acc, n_acc = np.zeros((3, T), dtype=np.int32), []
        for b in range(3):
            leaf, path = drafts[b] - 1 - turn % 2 if drafts[b] > 1 else 0, []
            while leaf >= 0:
                path.append(leaf)
                leaf = parents[b, leaf]
            acc[b, :len(path)] = path[::-1]
            n_acc.append(len(path))
        rows = [[[s.row(i, b, lens[b] + int(acc[b, k])) for k in range(n_acc[b])] for b in range(3)] for i in range(2)]
        step.commit(torch.from_numpy(acc).cuda(), torch.tensor(n_acc, dtype=torch.int32).cuda(), s.lens, s.lens, s.table, s.pools)
        torch.cuda.synchronize()
        assert s.lens.tolist() == [a + n for a, n in zip(lens, n_acc)]
        for i in range(2):
            for b in range(3):
                for k in range(n_acc[b]):
                    assert np.array_equal(s.row(i, b, lens[b] + k), rows[i][b][k])
        # the last accepted draft's attention is the single-token decode over the committed tokens
        last = [int(acc[b, n_acc[b] - 1]) for b in range(3)]
        q_lat = torch.stack([step.q_lat[:, b, last[b]] for b in range(3)], dim=1).contiguous()
        q_pe = torch.stack([step.q_pe.reshape(3, T, H, s.d_r)[b, last[b]] for b in range(3)]).contiguous()
        one = torch.empty((2, 3, H, s.dl), dtype=torch.float32, device="cuda")
        n_ws = tp.tpla_workspace_bytes_all(sh, s.max_pages, 0)
        tp.tpla_decode_shards(sh, q_lat, q_pe, s.pools, s.table, s.max_pages, s.lens, 0, torch.empty(n_ws, dtype=torch.uint8, device="cuda"),
                              n_ws, one, None)
        torch.cuda.synchronize()
        for b in range(3):
            # both are within their bound of the same sum in another order
            assert (np.abs(one[:, b].double().cpu().numpy() - got_lat[:, b, last[b]]) <= 2 * lat_off[:, b, last[b]]).all()


def test_captured_steps_with_drafts_of_changing_number():
    s = Loop("bf16", 16, 5, 16, seed=4)
    x = s.inputs()
    _, masks, depths, _, _, n_dev = s.trees([5, 3, 4])
    free = s.free.clone()
    args = (x["q_nope"], x["q_pe"], x["c_t"], x["k_pe"], s.W_UK, s.W_UV, s.pools, s.table, s.lens, n_dev, masks)

    def both():
        s.step.place(s.lens, n_dev, depths, free, free.numel(), s.held, s.table)
        return s.step.run(*args)

    both()                                           # (kernel attributes are set on first use; the pages are held from here on)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for n in ([5, 3, 4], [1, 5, 2], [0, 1, 5], [2, 0, 0]):
        n_dev.copy_(torch.tensor(n, dtype=torch.int32))
        s.step.o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = s.step.o.clone(), s.step.slots.clone(), s.step.lse.clone()
        both()
        torch.cuda.synchronize()
        for a, b in zip(replayed, (s.step.o, s.step.slots, s.step.lse)):
            assert torch.equal(a, b)
        assert not torch.isnan(s.step.o).any()


def test_two_calls_at_once_with_a_workspace_each():
    s, t = Loop("bf16", 16, 5, 16, seed=5), Loop("bf16", 64, 3, 16, seed=6)
    work = []
    for l in (s, t):
        x = l.inputs()
        _, masks, depths, _, _, n = l.trees([l.T, 1, 2])
        free = l.free.clone()
        l.step.place(l.lens, n, depths, free, free.numel(), l.held, l.table)
        work.append((l, (x["q_nope"], x["q_pe"], x["c_t"], x["k_pe"], l.W_UK, l.W_UV, l.pools, l.table, l.lens, n, masks)))
    alone = []
    for l, a in work:
        alone.append(l.step.run(*a).clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(4):
        for st, (l, a) in zip(streams, work):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                l.step.run(*a)
    torch.cuda.synchronize()
    for (l, _), want in zip(work, alone):
        assert torch.equal(l.step.o, want)
