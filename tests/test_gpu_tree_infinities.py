"""Drafts whose row holds an infinity: a head whose score becomes -inf gives it no weight, and 0 * inf is not a number in that column, as
for a committed token; heads whose score becomes inf, or all of whose scores are -inf, have no number anywhere; rows that do not see the draft do not notice."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import workloads as wl
from draft_common import TreeProblem, assert_close, out_buffers, run_all

pytestmark = pytest.mark.gpu

WIDE = 1 << 17
INF = {"f32": np.float32("inf"), "bf16": 0x7F80}


def with_infinity(p, b, j, column, negative=False):
    """Puts it into draft j of sequence b, slice 0; returns what the definition gives, from the call without that draft."""
    seen, whole = p.masks, p.expected()
    p.masks = seen.copy()
    p.masks[b] &= ~(np.uint64(1) << np.uint64(j))
    o, lse, o_off, lse_off = (np.concatenate([x[:1], y[1:]]) for x, y in zip(p.expected(), whole))      # (the other slices' rows stay as they are)
    p.masks = seen
    page, off = p.row_of(b, p.lens[b] + j)
    p.pools[0][page, off, column] = (-INF["f32"] if negative else INF["f32"]) if p.dtype == "f32" else INF["bf16"] | (0x8000 if negative else 0)
    q = wl.as_f64(p.q_lat, p.dtype)[0, b, :, :, column] * (-1.0 if negative else 1.0)
    kinds = set()
    for t in range(p.drafts[b]):
        if not (int(seen[b, t]) >> j) & 1:
            continue
        for h in range(p.shape.H):
            kinds.add(q[t, h] < 0)
            if q[t, h] < 0 and lse[0, b, t, h] > -np.inf:
                o[0, b, t, h, column] = np.nan
            else:
                o[0, b, t, h], lse[0, b, t, h] = np.nan, np.nan
    return (o, lse, o_off, lse_off), kinds


CASES = [  # rows on four waves, two teams, up to 128 rows, many rows; cut into several ranges where the context is long
    ("bf16", 256, 2, 16, 4, [50, 3], None), ("bf16", 256, 1, 16, 4, [9000, 0], None), ("bf16", 512, 1, 16, 3, [30, 700], None), ("bf16", 64, 2, 16, 4, [64, 1], None),
    ("bf16", 128, 2, 5, 40, [33, 0], None),
    ("bf16", 256, 2, 16, 4, [50, 64], WIDE), ("bf16", 256, 1, 16, 6, [95, 5000], WIDE), ("bf16", 128, 2, 16, 8, [63, 0], WIDE), ("bf16", 64, 4, 8, 3, [31, 500], WIDE),
    ("bf16", 256, 1, 64, 3, [90, 64], WIDE), ("bf16", 256, 1, 64, 3, [6000, 7], WIDE), ("bf16", 128, 1, 64, 4, [31, 0], WIDE), ("bf16", 64, 1, 64, 4, [30, 2000], WIDE),
]


@pytest.mark.parametrize("negative", [False, True])
@pytest.mark.parametrize("dtype,dl,g,H,T,lens,wide", CASES)
def test_an_infinity_in_one_column(dtype, dl, g, H, T, lens, wide, negative):
    d_r = 64 if dtype == "bf16" and dl in (64, 128, 256, 512) else 16
    masks = np.array([[(2 << t) - 1 for t in range(T)]] * 2, dtype=np.uint64)
    masks[:, T - 1] = 1 << (T - 1)                             # the last draft sees itself alone: not the one with the infinity
    for b, j, column in ((0, 1, 5), (1, 0, dl - 1), (0, T - 2, 0)):
        print("infinity", dtype, dl, g, H, T, lens, wide, negative, b, j, column, flush=True)
        p = TreeProblem(lens, [T, T], T, H=H, g=g, dl=dl, d_r=d_r, dtype=dtype, seed=dl + H + T + j, max_pages=wide, masks=masks)
        ref, kinds = with_infinity(p, b, j, column, negative)
        assert kinds == {True, False}
        o, lse = run_all(p)
        assert_close(p, o, lse, ref)
        assert np.array_equal(np.isnan(lse), np.isnan(ref[1]))


def test_drafts_of_many_tiles_and_several_infinities():
    T = 64
    p = TreeProblem([40, 100], [T, T - 9], T, H=16, g=1, pt=16, seed=4, masks=np.array([[(2 << t) - 1 for t in range(63)] + [2 ** 64 - 1]] * 2, dtype=np.uint64))
    p.masks[0, 63] = np.uint64(1) << np.uint64(63)
    ref, _ = with_infinity(p, 0, 47, 17)
    o, lse = run_all(p)
    assert_close(p, o, lse, ref)
    page, off = p.row_of(0, 40 + 50)                           # another one, in other columns: rows from 50 on
    p.pools[0][page, off, [1, 200]] = 0xFF80
    o2, _ = run_all(p)
    assert np.array_equal(o2[0, 0, :50], o[0, 0, :50], equal_nan=True) and np.array_equal(o2[0, 0, 63], o[0, 0, 63]) and np.array_equal(o2[0, 1], o[0, 1])
    assert np.isnan(o2[0, 0, 50:63][..., [1, 17, 200]]).all()


@pytest.mark.parametrize("dtype,H,L", [("bf16", 64, 63), ("bf16", 16, 0), ("bf16", 16, 3000)])
def test_committing_the_draft_changes_nothing(dtype, H, L):
    """The draft that sees itself is the decode of a sequence one longer: the same places are no numbers."""
    p = TreeProblem([L, 40], [1, 1], 1, H=H, masks=[[1], [1]], dtype=dtype, seed=6)
    ref, kinds = with_infinity(p, 0, 0, 9)
    assert kinds == {True, False}
    d = p.device()
    o, lse = run_all(p, d)
    assert_close(p, o, lse, ref)
    o2, lse2 = out_buffers(p)
    n = tp.tpla_workspace_bytes_all(p.shape, p.max_pages, 0)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    tp.tpla_decode_shards(p.shape, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"] + 1, 0, ws, n, o2, lse2)
    torch.cuda.synchronize()
    assert np.array_equal(np.isnan(o), np.isnan(o2.cpu().numpy())) and np.array_equal(np.isnan(lse), np.isnan(lse2.cpu().numpy()))


GENERAL = [("f32", 32, 2, 4, 5, [126, 0]), ("f32", 256, 1, 3, 6, [900, 13]), ("f32", 8, 2, 3, 3, [70, 1]), ("f32", 64, 8, 64, 16, [90, 32]), ("f32", 32, 1, 4, 5, [3001, 0]),
           ("bf16", 72, 2, 6, 5, [70, 3])]


@pytest.mark.parametrize("negative", [False, True])
@pytest.mark.parametrize("dtype,dl,g,H,T,lens", GENERAL)
def test_an_infinity_in_one_column_of_the_general_kernel(dtype, dl, g, H, T, lens, negative):
    masks = np.array([[(2 << t) - 1 for t in range(T)]] * 2, dtype=np.uint64)
    masks[:, T - 1] = 1 << (T - 1)
    both = set()
    for b, j, column in ((0, 1, 5), (1, 0, dl - 1), (0, T - 2, 0)):
        print("infinity, general", dtype, dl, g, H, T, lens, negative, b, j, column, flush=True)
        p = TreeProblem(lens, [T, T], T, H=H, g=g, dl=dl, d_r=16, dtype=dtype, seed=dl + H + T + j, masks=masks)
        ref, kinds = with_infinity(p, b, j, column, negative)
        both |= kinds
        o, lse = run_all(p)
        assert_close(p, o, lse, ref)
        assert np.array_equal(np.isnan(lse), np.isnan(ref[1]))
    assert both == {True, False}


@pytest.mark.parametrize("dtype,dl,H,L", [("f32", 32, 4, 71), ("f32", 256, 3, 71), ("bf16", 72, 6, 71), ("f32", 64, 4, 301), ("bf16", 256, 16, 71), ("bf16", 64, 16, 301)])
def test_an_infinity_of_a_committed_token_wherever_it_stands(dtype, dl, H, L):
    """In a group of tokens of its own kind, beside drafts, last before them."""
    T = 3
    for k in (0, L // 2, L - 3, L - 2, L - 1):
        print("infinity, committed", dtype, dl, H, L, k, flush=True)
        p = TreeProblem([L], [T], T, H=H, g=1, dl=dl, d_r=64 if dl in (64, 256) and dtype == "bf16" else 16, dtype=dtype, seed=dl + L)
        page, off = p.row_of(0, k)
        p.pools[0][page, off, 2] = INF[dtype]
        o, _ = run_all(p)
        q = wl.as_f64(p.q_lat, dtype)[0, 0, :, :, 2]
        want = np.zeros(o.shape, dtype=bool)
        want[0, 0][q >= 0] = True
        want[0, 0, ..., 2] = True
        assert (q < 0).any() and (q > 0).any() and np.array_equal(np.isnan(o), want)


@pytest.mark.parametrize("L", [0, 63, 600])
def test_committing_a_float_draft_changes_nothing(L):
    p = TreeProblem([L, 40], [1, 1], 1, H=4, dl=64, d_r=16, masks=[[1], [1]], dtype="f32", seed=6)
    ref, kinds = with_infinity(p, 0, 0, 9)
    assert kinds == {True, False}
    d = p.device()
    o, lse = run_all(p, d)
    assert_close(p, o, lse, ref)
    o2, lse2 = out_buffers(p)
    n = tp.tpla_workspace_bytes_all(p.shape, p.max_pages, 0)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    tp.tpla_decode_shards(p.shape, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"] + 1, 0, ws, n, o2, lse2)
    torch.cuda.synchronize()
    print(np.isnan(o).sum(), np.isnan(o2.cpu().numpy()).sum(), lse[0, 0], lse2[0, 0])
    assert np.array_equal(np.isnan(o), np.isnan(o2.cpu().numpy())) and np.array_equal(np.isnan(lse), np.isnan(lse2.cpu().numpy()))
