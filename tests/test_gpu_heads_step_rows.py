"""HeadsStep: every row that a new token owns is computed, whatever the step was made for; rows that none owns are NaN; tokens without a page are neither
written nor seen.  Against 64 bits at every step."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import pipeline as pl
from heads_common import DTYPE, HALF_STEP, shape_of, stored
from test_gpu_heads_rows import turned
from test_gpu_heads_step import Reference

pytestmark = pytest.mark.gpu
ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731


class World:
    """A layer, its step, and the same in 64 bits."""

    def __init__(self, B, H, H_kv, d, page, dtype, most, n_pages, **kw):
        r = self.r = np.random.default_rng([H, d, page])
        self.B, self.H, self.H_kv, self.d, self.dtype = B, H, H_kv, d, dtype
        freq = tp.tpla_rotary_frequencies(d, 10000.0)
        (wq, wq64), (wk, wk64) = (stored(1 + 0.1 * r.standard_normal(d), dtype) for _ in range(2))
        self.wq, self.wk = wq.cuda(), wk.cuda()
        self.step = pl.HeadsStep(shape_of(B, H, H_kv, d, page=page, dtype=dtype), most, freq, **kw)
        self.pools = [torch.full((n_pages, H_kv, page, d), float("nan"), dtype=DTYPE[dtype], device="cuda") for _ in range(2)]
        self.table, self.held, self.free, self.lens = torch.zeros((B, most), dtype=torch.int32, device="cuda"), ints([0] * B), ints(r.permutation(n_pages).tolist()), ints([0] * B)
        self.ref = Reference(B, H, H_kv, d, dtype, freq, wq64, wk64)
        for x in (self.step.o, self.step.lse):
            x.fill_(7.0)

    def rows(self, T):
        x, x64 = stored(self.r.standard_normal((T, self.H + 2 * self.H_kv, self.d)) * 1.5, self.dtype)
        x = x.cuda()
        cut = lambda y: (y[:, :self.H], y[:, self.H:self.H + self.H_kv], y[:, self.H + self.H_kv:])  # noqa: E731
        return cut(x), cut(x64)

    def add(self, news, T=None, told=False, decode=False):
        """T: rows given (those behind sum(news) are padding)."""
        n = sum(news)
        (q, k, v), (q64, k64, v64) = self.rows(n if T is None else T)
        self.step.place(self.lens, ints(news), self.free, self.free.numel(), self.held, self.table, **(dict(news=news) if told else {}))
        after = self.lens + ints(news)
        o = self.step.run(q, k, v, self.wq, self.wk, *self.pools, self.table, after if decode else self.lens, decode=decode)
        taken, missing = self.step.counts.tolist()
        assert missing == 0
        self.free, self.lens = self.free[taken:].clone(), after
        got = o.double().cpu().numpy()
        assert np.isnan(got[n:]).all() and torch.isnan(self.step.lse[n:len(got)]).all()
        if n == 0:
            return
        want = self.ref.step(news, q64[:n], k64[:n], v64[:n])
        # o's rounding, for bf16 that of the weights, and a key or query on the other side of its rounding here than there: one score of many by
        # at most one step of one product
        tol = (HALF_STEP[self.dtype] + (3 * HALF_STEP["bf16"] if self.dtype == "bf16" else 2.0 ** -14)) * np.abs(want).max()
        assert np.abs(got[:n] - want).max() <= tol, news


SHAPES = [(8, 2, 128, 64, "bf16"), (4, 4, 64, 16, "bf16"), (6, 2, 96, 32, "f32")]


@pytest.mark.parametrize("H,H_kv,d,page,dtype", SHAPES)
@pytest.mark.parametrize("kw", [dict(max_tokens=200), dict(max_tokens=200, max_new=4)], ids=["room", "few"])
def test_sequences_of_more_tokens_than_the_step_was_made_for(H, H_kv, d, page, dtype, kw):
    w = World(3, H, H_kv, d, page, dtype, 256 // page + 4, 3 * (256 // page + 4), **kw)
    w.add([70, 5, 0])
    w.add([3, 40, 130])
    w.add([0, 2, 1])
    w.add([1, 1, 1], decode=True)


@pytest.mark.parametrize("H,H_kv,d,page,dtype", SHAPES)
def test_a_default_step_whose_tokens_are_one_sequences(H, H_kv, d, page, dtype):
    w = World(5, H, H_kv, d, page, dtype, 6, 30)
    w.add([0, 5, 0, 0, 0])
    w.add([1, 1, 1, 1, 1], decode=True)
    w.add([2, 0, 3, 0, 0])


@pytest.mark.parametrize("H,H_kv,d,page,dtype", SHAPES)
def test_counted_steps_and_padded_ones(H, H_kv, d, page, dtype):
    w = World(3, H, H_kv, d, page, dtype, 256 // page + 4, 3 * (256 // page + 4), max_tokens=200, max_new=130)
    w.add([70, 5, 0], told=True)
    w.add([2, 0, 3], T=64)
    w.add([0, 100, 30], told=True)
    w.add([1, 1, 1], told=True, decode=True)
    w.add([0, 0, 0], T=7)


@pytest.mark.parametrize("H,H_kv,d,page,dtype", SHAPES)
def test_tokens_without_a_page(H, H_kv, d, page, dtype):
    """Four pages short: the last sequence's tokens lose their pages from some page on, and later tokens find what was written."""
    B, news = 2, [2 * page + 3, 6 * page + 1]
    w = World(B, H, H_kv, d, page, dtype, 12, 6, max_tokens=9 * page)
    s, T = w.step, sum(news)
    (q, k, v), (q64, k64, v64) = w.rows(T)
    s.place(w.lens, ints(news), w.free, w.free.numel(), w.held, w.table)
    o = s.run(q, k, v, w.wq, w.wk, *w.pools, w.table, w.lens).double().cpu().numpy()
    assert s.counts.tolist() == [6, 4] and w.held.tolist() == [3, 3]                   # 3 + 7 pages wanted
    got = [o]
    w.lens = ints(news)
    s.place(w.lens, ints([1, 1]), w.free, 0, w.held, w.table)                          # the next tokens: one has room in its page, one does not
    (q1, k1, v1), (q164, k164, v164) = w.rows(2)
    got.append(s.run(q1, k1, v1, w.wq, w.wk, *w.pools, w.table, w.lens + 1, decode=True).double().cpu().numpy())
    assert s.counts.tolist() == [0, 4]
    eps, first = np.float64(np.float32(1e-6)), 0
    for b, n in enumerate(news):
        at = np.r_[first:first + n]
        turn = lambda x, y, weight: w.ref.rounded(turned(np.concatenate([x[at], y[b:b + 1]]), weight, eps, d, tp.TPLA_ROTARY_HALF, w.ref.freq, np.arange(n + 1), 1.0)[0])  # noqa: E731
        Q, K, V = turn(q64, q164, w.ref.wq), turn(k64, k164, w.ref.wk), np.concatenate([v64[at], v164[b:b + 1]])
        there = np.arange(n + 1) < 3 * page
        for h in range(H):
            score = Q[:, h] @ K[:, h // w.ref.G].T / np.sqrt(d)
            score[(np.arange(n + 1)[None] > np.arange(n + 1)[:, None]) | ~there[None]] = -np.inf
            p = np.exp(score - score.max(-1, keepdims=True))
            want = p / p.sum(-1, keepdims=True) @ V[:, h // w.ref.G]
            have = np.concatenate([got[0][at, h], got[1][b:b + 1, h]])
            tol = (HALF_STEP[dtype] + (3 * HALF_STEP["bf16"] if dtype == "bf16" else 2.0 ** -14)) * np.abs(want).max()
            assert np.abs(have - want).max() <= tol, (b, h)
        first += n
