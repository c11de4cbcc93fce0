"""Inputs and the 64-bit definition of the drafted tokens' attention (not collected by pytest)."""
import math

import numpy as np
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import pipeline as pl
from paper_2508_15881_amd import workloads as wl

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}     # half a step, relative to the value


def chain_masks(B, T):
    return np.tile(np.array([(2 << t) - 1 for t in range(T)], dtype=np.uint64), (B, 1)) if T < 64 else \
        np.tile(np.array([(1 << (t + 1)) - 1 for t in range(T)], dtype=np.uint64), (B, 1))


def random_masks(rng, B, T):
    """Masks of random trees: a draft sees what its parent sees, and itself."""
    m = np.zeros((B, T), dtype=np.uint64)
    for b in range(B):
        for t in range(T):
            p = int(rng.integers(-1, t)) if t else -1
            m[b, t] = (m[b, p] if p >= 0 else np.uint64(0)) | (np.uint64(1) << np.uint64(t))
    return m


class TreeProblem:
    """Seeded inputs of one call over all slices.  Rows that belong to no token are NaN."""

    def __init__(self, lens, drafts, T, H=16, g=2, dl=256, d_r=64, pt=64, dtype="bf16", d_v=128, seed=0, masks=None, spare_pages=3,
                 max_pages=None):
        self.lens, self.drafts, self.T, self.g, self.dtype = list(lens), list(drafts), T, g, dtype
        B = len(lens)
        r = np.random.default_rng([seed, 41])
        self.shape = tp.TplaShape(B, H, dl * g, g, d_r, 128, d_v, pt, tp.TPLA_F32 if dtype == "f32" else tp.TPLA_BF16,
                                  1.0 / math.sqrt(128 + d_r))
        pages = [-(-(a + b) // pt) for a, b in zip(lens, drafts)]
        self.max_pages = max_pages or max(1, max(pages))
        n_pool = sum(pages) + spare_pages
        order = r.permutation(n_pool)
        self.bt = np.full((B, self.max_pages), n_pool - 1, dtype=np.int32)
        k = 0
        for b, n in enumerate(pages):
            self.bt[b, :n] = order[k:k + n]
            k += n
        width = dl + d_r
        self.pools = [wl.nan_fill((n_pool, pt, width), dtype) for _ in range(g)]
        for b in range(B):
            n = lens[b] + drafts[b]
            for i in range(g):
                wl.place_rows(self.pools[i], self.bt[b, :max(1, pages[b])], wl.to_storage(r.standard_normal((n, width)), dtype))
        self.q_lat = wl.to_storage(r.standard_normal((g, B, T, H, dl)) * 0.35, dtype)
        self.q_pe = wl.to_storage(r.standard_normal((B, T, H, d_r)), dtype)
        self.W = wl.to_storage(r.standard_normal((H, dl * g, d_v)) * 0.02, dtype)
        self.masks = random_masks(r, B, T) if masks is None else np.asarray(masks, dtype=np.uint64)

    def row_of(self, b, t):
        pt = self.shape.page_tokens
        return self.bt[b, t // pt], t % pt

    def rows64(self, i, b):
        pt = self.shape.page_tokens
        t = np.arange(min(self.lens[b] + self.drafts[b], self.max_pages * pt))
        return wl.as_f64(self.pools[i][self.bt[b][t // pt], t % pt], self.dtype)

    def expected(self):
        """o_lat, lse, and how far each may be off: derived below."""
        s, T = self.shape, self.T
        dl = s.d_c // s.g
        o = np.zeros((s.g, s.B, T, s.H, dl))
        lse = np.full((s.g, s.B, T, s.H), -np.inf)
        o_off, lse_off = np.zeros_like(o), np.zeros_like(lse)
        q_lat, q_pe = wl.as_f64(self.q_lat, self.dtype), wl.as_f64(self.q_pe, self.dtype)
        for b in range(s.B):
            L, n = self.lens[b], min(self.drafts[b], T)
            for i in range(s.g):
                rows = self.rows64(i, b)
                for t in range(n):
                    sees = np.array([True] * L + [bool((int(self.masks[b, t]) >> j) & 1) for j in range(n)])[:len(rows)]
                    if not sees.any():
                        continue
                    x = rows[sees]
                    q = np.concatenate([q_lat[i, b, t], q_pe[b, t]], axis=1)
                    with np.errstate(invalid="ignore", over="ignore"):
                        sc = q @ x.T * s.sm_scale
                        top = sc.max(1, keepdims=True)
                        p = np.exp(sc - top)
                        l = p.sum(1, keepdims=True)
                        o[i, b, t] = p @ x[:, :dl] / l
                        lse[i, b, t] = (np.log(l) + top)[:, 0]
                        # a score is a float sum of dl + d_r exact products: off by (dl + d_r) half steps of the sum of their
                        # sizes at most, and as much again for scaling, reference and exponential (3 operations)
                        size = np.abs(q) @ np.abs(x.T) * s.sm_scale
                        ds = ((dl + s.d_r + 6) * 2.0 ** -24 * size.max(1) + 2.0 ** -21)[:, None]
                        # a weight is off by ds, by half a step of the type it is multiplied in, and by the float sum over
                        # the tokens; the sum of the weights by ds and its own float sum
                        each = 2 * ds + (HALF[self.dtype] if self.dtype == "bf16" else 0.0) + 2 * (x.shape[0] + 8) * 2.0 ** -24
                        o_off[i, b, t] = each * (p / l) @ np.abs(x[:, :dl])
                        lse_off[i, b, t] = (ds + (x.shape[0] + 8) * 2.0 ** -24)[:, 0] + np.abs(lse[i, b, t]) * 2.0 ** -22
        return o, lse, o_off, lse_off

    def device(self):
        return dict(q_lat=pl.to_device(self.q_lat, self.dtype), q_pe=pl.to_device(self.q_pe, self.dtype),
                    pools=[pl.to_device(p, self.dtype) for p in self.pools], bt=torch.from_numpy(self.bt).cuda(),
                    lens=torch.tensor(self.lens, dtype=torch.int32).cuda(), drafts=torch.tensor(self.drafts, dtype=torch.int32).cuda(),
                    masks=torch.from_numpy(self.masks.view(np.int64)).cuda(), W=pl.to_device(self.W, self.dtype))

    def check_ids(self):
        """On the host, before a launch: every page id that a kernel may read lies in the pool."""
        pt, P = self.shape.page_tokens, self.pools[0].shape[0]
        for b in range(self.shape.B):
            n = -(-min(self.lens[b] + self.drafts[b], self.max_pages * pt) // pt)
            assert n <= self.max_pages and (self.bt[b, :n] >= 0).all() and (self.bt[b, :n] < P).all()


def out_buffers(p, fill=float("nan")):
    s = p.shape
    return (torch.full((s.g, s.B, p.T, s.H, s.d_c // s.g), fill, dtype=torch.float32, device="cuda"),
            torch.full((s.g, s.B, p.T, s.H), fill, dtype=torch.float32, device="cuda"))


def workspace(p):
    n = tp.tpla_workspace_bytes_tree(p.shape, p.T, p.max_pages)
    assert n > 0
    return torch.empty(n, dtype=torch.uint8, device="cuda"), n


def run_all(p, d=None, drafts="given"):
    p.check_ids()
    d = d or p.device()
    o, lse = out_buffers(p)
    ws, n = workspace(p)
    tp.tpla_decode_shards_tree(p.shape, p.T, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"],
                               d["drafts"] if drafts == "given" else drafts, d["masks"], ws, n, o, lse)
    torch.cuda.synchronize()
    return o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)


def assert_close(p, o, lse, ref=None):
    want_o, want_lse, o_off, lse_off = ref or p.expected()
    nan = np.isnan(want_o)
    assert np.array_equal(np.isnan(o), nan)
    bad = np.abs(np.where(nan, 0, o - want_o)) > np.where(nan, 0, o_off)
    assert not bad.any(), "o_lat: %d of %d off, worst %.3g of what is allowed, first %r" % (
        bad.sum(), bad.size, np.nanmax(np.where(bad, np.abs(o - want_o) / np.maximum(o_off, 1e-300), 0)), np.argwhere(bad)[0].tolist())
    fin = np.isfinite(want_lse)
    assert np.array_equal(np.isfinite(lse), fin) and np.array_equal(lse[~fin & ~np.isnan(want_lse)], want_lse[~fin & ~np.isnan(want_lse)])
    assert (np.abs(lse[fin] - want_lse[fin]) <= lse_off[fin]).all(), np.max(np.abs(lse[fin] - want_lse[fin]) / lse_off[fin])
