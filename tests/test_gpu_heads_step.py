"""A serving run of a layer with grouped heads: prompts admitted, their next parts, then tokens one by one, against 64 bits at every step."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import pipeline as pl
from heads_common import DTYPE, HALF_STEP, shape_of, stored
from test_gpu_heads_rows import turned

pytestmark = pytest.mark.gpu


class Reference:
    """The cache as rows in storage precision, attention in 64 bits."""

    def __init__(self, B, H, H_kv, d, dtype, freq, wq, wk):
        self.K, self.V = [np.zeros((0, H_kv, d)) for _ in range(B)], [np.zeros((0, H_kv, d)) for _ in range(B)]
        self.H, self.G, self.d, self.dtype, self.freq, self.wq, self.wk = H, H // H_kv, d, dtype, freq, wq, wk

    def rounded(self, x):
        return torch.from_numpy(x).to(DTYPE[self.dtype]).double().numpy()

    def step(self, news, q, k, v):
        """New rows of every sequence, packed; o of each."""
        pos = np.concatenate([len(K) + np.arange(n) for K, n in zip(self.K, news)])
        eps = np.float64(np.float32(1e-6))
        q = self.rounded(turned(q, self.wq, eps, self.d, tp.TPLA_ROTARY_HALF, self.freq, pos, 1.0)[0])
        k = self.rounded(turned(k, self.wk, eps, self.d, tp.TPLA_ROTARY_HALF, self.freq, pos, 1.0)[0])
        out, at = np.zeros((len(pos), self.H, self.d)), 0
        for b, n in enumerate(news):
            L = len(self.K[b])
            self.K[b], self.V[b] = np.concatenate([self.K[b], k[at:at + n]]), np.concatenate([self.V[b], v[at:at + n]])
            for h in range(self.H):
                s = q[at:at + n, h] @ self.K[b][:, h // self.G].T / np.sqrt(self.d)
                s[np.arange(L + n)[None] > L + np.arange(n)[:, None]] = -np.inf
                p = np.exp(s - s.max(-1, keepdims=True)) if n else s
                out[at:at + n, h] = p / p.sum(-1, keepdims=True) @ self.V[b][:, h // self.G]
            at += n
        return out


@pytest.mark.parametrize("H,H_kv,d,page,dtype", [(8, 2, 128, 64, "bf16"), (4, 4, 64, 16, "bf16"), (6, 2, 96, 32, "f32"), (6, 2, 32, 8, "bf16")])
def test_prompts_parts_and_tokens(H, H_kv, d, page, dtype):
    B, steps = 3, [[70, 5, 0], [64, 0, 130], [1, 2, 3], "decode", "decode", [40, 1, 17], "decode"]
    r = np.random.default_rng([H, d, page])
    shape = shape_of(B, H, H_kv, d, page=page, dtype=dtype)
    most, n_pages = 256 // page + 4, 3 * (256 // page + 4)
    freq = tp.tpla_rotary_frequencies(d, 10000.0)
    wq, wq64 = stored(1 + 0.1 * r.standard_normal(d), dtype)
    wk, wk64 = stored(1 + 0.1 * r.standard_normal(d), dtype)
    wq, wk = wq.cuda(), wk.cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    step = pl.HeadsStep(shape, most, freq, max_tokens=200, max_new=130)
    pools = [torch.full((n_pages, H_kv, page, d), float("nan"), dtype=DTYPE[dtype], device="cuda") for _ in range(2)]
    table, held, free = torch.zeros((B, most), dtype=torch.int32, device="cuda"), ints([0] * B), ints(r.permutation(n_pages).tolist())
    ref, lens = Reference(B, H, H_kv, d, dtype, freq, wq64, wk64), ints([0] * B)
    for what in steps:
        news = [1] * B if what == "decode" else what
        T = sum(news)
        x, x64 = stored(r.standard_normal((T, H + 2 * H_kv, d)) * 1.5, dtype)
        x = x.cuda()
        step.place(lens, ints(news), free, free.numel(), held, table)
        after = lens + ints(news)
        o = step.run(x[:, :H], x[:, H:H + H_kv], x[:, H + H_kv:], wq, wk, *pools, table, after if what == "decode" else lens, decode=what == "decode")
        taken, missing = step.counts.tolist()
        assert missing == 0
        free, lens = free[taken:].clone(), after
        want = ref.step(news, x64[:, :H], x64[:, H:H + H_kv], x64[:, H + H_kv:])
        got = o.double().cpu().numpy()
        # the rounding of o; for bf16 that of the weights, and a key or query that fell on the other side of a rounding here than there (its
        # float value off by a few 2^-24) moves one score of many by at most one step of one product
        tol = (HALF_STEP[dtype] + (3 * HALF_STEP["bf16"] if dtype == "bf16" else 2.0 ** -14)) * np.abs(want).max()
        assert np.abs(got - want).max() <= tol, what
        assert step.cu.tolist() == [0, *np.cumsum(news).tolist()]


def test_decode_step_captured_and_replayed():
    """place and run of a decode step in one graph: lengths grow in place, every replay equals the eager step."""
    B, H, H_kv, d, page = 5, 16, 4, 128, 16
    r = np.random.default_rng(4)
    shape, most = shape_of(B, H, H_kv, d, page=page), 12
    freq = tp.tpla_rotary_frequencies(d, 10000.0)
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    free0 = ints(r.permutation(B * most).tolist())
    x = torch.zeros((B, H + 2 * H_kv, d), dtype=torch.bfloat16, device="cuda")
    add = ints([1] * B)

    def world():
        s = pl.HeadsStep(shape, most, freq)
        s.state = dict(pools=[torch.zeros((B * most, H_kv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                       table=torch.zeros((B, most), dtype=torch.int32, device="cuda"), held=ints([0] * B), lens=ints([0] * B), after=ints([0] * B),
                       free=free0.clone(), taken=ints([0]))
        return s

    def one(s):
        y = s.state
        # the list of free pages goes on behind those that are taken
        s.place(y["lens"], add, y["free"], y["free"].numel(), y["held"], y["table"])
        y["free"].copy_(torch.take(y["free"], (torch.arange(y["free"].numel(), device="cuda") + s.counts[0].long()) % y["free"].numel()))
        torch.add(y["lens"], add, out=y["after"])
        s.run(x[:, :H], x[:, H:H + H_kv], x[:, H + H_kv:], w, w, *y["pools"], y["table"], y["after"], decode=True)
        y["lens"].copy_(y["after"])

    eager, replayed, warm = world(), world(), world()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        one(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        one(replayed)
    for i in range(40):
        x.copy_(torch.from_numpy(r.standard_normal(tuple(x.shape))).cuda())
        one(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.o, replayed.o) and torch.isfinite(eager.o).all(), i
        assert torch.equal(eager.state["lens"], replayed.state["lens"]) and torch.equal(eager.state["table"], replayed.state["table"])
