"""Attention of drafted tokens (tpla_decode_shard(s)_tree) against its 64-bit definition, at the sizes and masks where it can go
wrong.  Every bound is derived from the roundings in draft_common.TreeProblem.expected."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import workloads as wl
from draft_common import TreeProblem, assert_close, chain_masks, out_buffers, run_all, workspace

pytestmark = pytest.mark.gpu


# Which kernel a call takes depends on the rows of a sequence and on the width of the block table: a wide one is work for all of the chip.
WIDE = 1 << 17


@pytest.mark.parametrize("dtype,dl,g,H,T,lens,drafts,pt", [
    ("bf16", 256, 2, 16, 4, [130, 1, 64, 0, 1000], [4, 1, 3, 2, 4], 64),
    ("bf16", 256, 2, 64, 3, [33, 500], [3, 2], 64),                  # 192 rows
    ("bf16", 256, 1, 64, 8, [95, 96, 97], [8, 8, 8], 64),            # 512 rows, ends around a tile's edge
    ("bf16", 256, 2, 5, 7, [31, 62, 640], [7, 1, 5], 16),            # 35 rows, pages that end inside a tile
    ("bf16", 256, 1, 16, 64, [200, 3], [64, 61], 64),                # the most drafts
    ("bf16", 256, 1, 16, 2, [700, 77], [2, 2], 1),                   # one token a page: ids in several chunks
    ("bf16", 256, 1, 16, 2, [1500, 300], [2, 1], 3),
    ("bf16", 256, 2, 1, 1, [1, 0, 2049], [1, 1, 1], 128),            # one row
    ("bf16", 128, 4, 64, 4, [300, 65], [4, 4], 64),
    ("bf16", 128, 4, 16, 2, [31, 0, 1025], [2, 2, 0], 32),
    ("bf16", 64, 8, 16, 9, [257, 40], [9, 6], 64),
    ("bf16", 64, 8, 64, 4, [100], [4], 64),
    ("bf16", 512, 1, 16, 5, [129, 800], [5, 3], 64),
    ("bf16", 512, 1, 64, 2, [64, 31], [2, 1], 16),
    ("bf16", 72, 2, 6, 5, [70, 3], [5, 4], 16),                      # a width of the general kernel
    ("f32", 32, 2, 4, 5, [128, 60, 0], [5, 3, 2], 64),
    ("f32", 8, 2, 3, 2, [70, 1], [2, 1], 64),                        # eight columns
    ("f32", 16, 2, 3, 2, [70, 1], [2, 1], 64),
    ("f32", 256, 2, 3, 6, [900, 1], [6, 6], 64),
    ("f32", 64, 8, 64, 16, [90, 33], [16, 16], 64),                  # enough rows for four per wave
    ("f32", 1024, 1, 2, 3, [65], [3], 16),
])
def test_against_the_definition(dtype, dl, g, H, T, lens, drafts, pt):
    d_r = 64 if dtype == "bf16" and dl in (64, 128, 256, 512) else 16
    print("tree", dtype, dl, g, H, T, lens, drafts, pt, flush=True)
    p = TreeProblem(lens, drafts, T, H=H, g=g, dl=dl, d_r=d_r, pt=pt, dtype=dtype, seed=dl + H + T)
    assert_close(p, *run_all(p))


@pytest.mark.parametrize("dl,g,H,T,lens,drafts,pt", [
    # up to 64 rows: two teams
    (256, 2, 16, 4, [130, 1, 64, 0, 1000], [4, 1, 3, 2, 4], 64),
    (256, 2, 5, 7, [31, 62, 640], [7, 1, 5], 16),
    (256, 1, 16, 2, [700, 77, 64, 63], [2, 2, 1, 2], 1),
    (256, 1, 64, 1, [1500, 300, 32, 96], [1, 1, 1, 1], 3),
    (128, 4, 16, 3, [300, 65, 4000], [3, 1, 2], 32), (64, 8, 64, 1, [257, 40], [1, 1], 64),
    # up to 128 rows, and several blocks of 128
    (256, 2, 16, 5, [130, 1, 64, 0, 1000], [5, 1, 3, 2, 4], 64), (256, 1, 64, 4, [95, 96, 97, 31], [4, 3, 2, 4], 128),
    (256, 1, 16, 6, [700, 77], [6, 2], 1), (128, 2, 64, 2, [300, 65, 2500], [2, 1, 2], 16), (64, 4, 16, 8, [64, 63, 513], [8, 7, 8], 64),
    (128, 1, 64, 6, [333], [5], 64),
    # 192 rows (256-wide), 256 rows (narrower)
    (256, 2, 64, 3, [33, 500, 0, 1], [3, 2, 3, 1], 64), (256, 1, 64, 12, [95, 1200], [12, 7], 16), (256, 1, 24, 8, [64, 900, 32], [8, 8, 1], 3),
    (256, 1, 64, 3, [6000, 65], [3, 3], 64), (256, 1, 64, 3, [200, 90], [3, 2], 1),
    (128, 2, 64, 4, [300, 65, 31, 32], [4, 4, 1, 3], 64), (128, 1, 64, 16, [700, 3], [16, 11], 32),
    (64, 2, 64, 4, [257, 40], [4, 2], 64), (64, 1, 32, 16, [5, 1000], [16, 9], 16),
    # 512-wide slices
    (512, 1, 64, 2, [64, 31, 3000], [2, 1, 2], 64),
])
def test_against_the_definition_over_wide_tables(dl, g, H, T, lens, drafts, pt):
    print("tree, wide table", dl, g, H, T, lens, drafts, pt, flush=True)
    p = TreeProblem(lens, drafts, T, H=H, g=g, dl=dl, pt=pt, seed=dl + H + T, max_pages=WIDE)
    assert_close(p, *run_all(p))


@pytest.mark.parametrize("dtype,H,wide", [("bf16", 16, None), ("f32", 16, None), ("bf16", 16, WIDE), ("bf16", 32, WIDE), ("bf16", 48, WIDE)])
def test_empty_masks_and_drafts_that_do_not_exist(dtype, H, wide):
    lens, drafts, T = [0, 0, 70, 5], [3, 0, 4, 2], 4
    masks = np.zeros((4, T), dtype=np.uint64)
    masks[0] = [0, 2, 4, 0]                                  # draft 0 of an empty sequence sees nothing
    masks[2] = [0, np.uint64(0xFFFFFFFFFFFFFFFF), 1, 8]      # bits beyond the drafts are ignored
    masks[3] = [np.uint64(1) << np.uint64(63), 3, 3, 3]
    p = TreeProblem(lens, drafts, T, H=H, masks=masks, dtype=dtype, seed=5, max_pages=wide)
    o, lse = run_all(p)
    assert_close(p, o, lse)
    assert (o[:, 0, 0] == 0).all() and (lse[:, 0, 0] == -np.inf).all()
    assert (o[:, 1] == 0).all() and (lse[:, 1] == -np.inf).all()
    assert (o[:, 3, 2:] == 0).all() and (lse[:, 3, 2:] == -np.inf).all()


@pytest.mark.parametrize("dtype,H,wide", [("bf16", 16, None), ("f32", 16, None), ("bf16", 8, WIDE), ("bf16", 16, WIDE), ("bf16", 32, WIDE)])
@pytest.mark.parametrize("L", [0, 50, 64, 95])
def test_what_a_masked_draft_holds_reaches_nobody_else(dtype, H, wide, L):
    T = 6
    p = TreeProblem([L, 40], [T, T], T, H=H, masks=chain_masks(2, T), dtype=dtype, seed=7, max_pages=wide)
    p.masks[0] = [1, 2, 5, 9, 17, 33]                        # draft 1 is seen by itself alone
    clean = p.expected()
    nan, inf = (np.float32("nan"), np.float32("inf")) if dtype == "f32" else (0x7FC0, 0x7F80)
    page, off = p.row_of(0, L + 1)
    for i in range(2):
        p.pools[i][page, off, ::2] = nan
        p.pools[i][page, off, 1::2] = inf
    o, lse = run_all(p)
    assert np.isnan(o[:, 0, 1]).all() and np.isnan(lse[:, 0, 1]).all()
    o[:, 0, 1], lse[:, 0, 1] = clean[0][:, 0, 1], clean[1][:, 0, 1]
    assert_close(p, o, lse, clean)


def test_a_committed_row_that_is_not_a_number_is_seen_by_all_of_its_sequence():
    p = TreeProblem([300, 40], [2, 2], 2, seed=8)
    clean = p.expected()
    page, off = p.row_of(0, 11)
    p.pools[1][page, off, 3] = 0x7FC0
    o, lse = run_all(p)
    assert np.isnan(o[1, 0]).all() and np.isnan(lse[1, 0]).all()
    o[1, 0], lse[1, 0] = clean[0][1, 0], clean[1][1, 0]
    assert_close(p, o, lse, clean)


@pytest.mark.parametrize("H,wide", [(16, None), (16, WIDE), (40, WIDE), (64, WIDE)])
def test_a_reference_that_moves(H, wide):
    p = TreeProblem([200], [3], 3, H=H, seed=9, max_pages=wide)
    p.q_lat = wl.to_storage(wl.as_f64(p.q_lat, "bf16") * 400.0, "bf16")    # a few tokens carry everything, the reference moves
    assert_close(p, *run_all(p))


def test_lengths_out_of_range_are_clipped():
    T = 4
    p = TreeProblem([120, 64], [4, 4], T, masks=chain_masks(2, T), seed=10)
    d = p.device()
    ref = p.expected()
    d["drafts"] = torch.tensor([9, 4], dtype=torch.int32).cuda()         # more than T count as T
    assert_close(p, *run_all(p, d), ref)
    d["drafts"] = torch.tensor([-1, 4], dtype=torch.int32).cuda()
    o, lse = run_all(p, d)
    assert (o[:, 0] == 0).all() and (lse[:, 0] == -np.inf).all()
    d["drafts"] = torch.tensor([4, 4], dtype=torch.int32).cuda()
    d["lens"] = torch.tensor([-5, 64], dtype=torch.int32).cuda()         # fewer than none count as none
    p.lens = [0, 64]
    assert_close(p, *run_all(p, d))


def test_drafts_beyond_the_table_row_are_not_seen():
    T = 4
    p = TreeProblem([124], [4], T, masks=chain_masks(1, T), seed=10)
    assert p.max_pages * 64 == 128
    d = p.device()
    p.lens = [126]                                             # drafts 2 and 3 would be tokens 128 and 129
    d["lens"] = torch.tensor([126], dtype=torch.int32).cuda()
    assert_close(p, *run_all(p, d))
    p.lens, p.drafts = [128], [4]
    d["lens"] = torch.tensor([500], dtype=torch.int32).cuda()  # clipped to the row; no draft is seen
    assert_close(p, *run_all(p, d))


def test_no_draft_lengths_means_all():
    p = TreeProblem([100, 7], [5, 5], 5, seed=11)
    assert_close(p, *run_all(p, drafts=None))


@pytest.mark.parametrize("wide", [None, WIDE])
@pytest.mark.parametrize("H,T,lens", [(16, 2, [9000, 40, 3000]), (64, 4, [5003, 1200]), (64, 16, [700, 3000]), (16, 1, [20000]), (64, 3, [4000])])
def test_long_contexts_are_cut_and_joined(H, T, lens, wide):
    p = TreeProblem(lens, [T] * len(lens), T, H=H, g=1, seed=12, max_pages=wide)
    assert_close(p, *run_all(p))


@pytest.mark.parametrize("H,wide", [(32, None), (8, WIDE), (20, WIDE), (32, WIDE)])
def test_same_bits_every_time_and_on_another_stream(H, wide):
    p = TreeProblem([3000, 77, 512], [6, 2, 5], 6, H=H, seed=13, max_pages=wide)
    d = p.device()
    a = run_all(p, d)
    b = run_all(p, d)
    o, lse = out_buffers(p)
    ws, n = workspace(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tp.tpla_decode_shards_tree(p.shape, p.T, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"], d["drafts"],
                                   d["masks"], ws, n, o, lse)
    side.synchronize()
    for x, y, z in zip(a, b, (o, lse)):
        assert np.array_equal(x, y) and np.array_equal(x, z.cpu().numpy().astype(np.float64))


def test_one_slice_is_that_slice():
    p = TreeProblem([400, 90], [5, 3], 5, H=64, g=4, dl=128, seed=14)
    d = p.device()
    ref = p.expected()
    ws, n = workspace(p)
    for i in range(4):
        o, lse = out_buffers(p)
        tp.tpla_decode_shard_tree(p.shape, p.T, d["q_lat"][i], d["q_pe"], d["pools"][i], d["bt"], p.max_pages, d["lens"], d["drafts"],
                                  d["masks"], ws, n, o[i], lse[i])
        torch.cuda.synchronize()
        both = o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        for k in range(2):
            both[k][[j for j in range(4) if j != i]] = ref[k][[j for j in range(4) if j != i]]
        assert_close(p, *both, ref)


def test_one_draft_that_sees_itself_is_the_decode_of_a_sequence_one_longer():
    p = TreeProblem([640, 63], [1, 1], 1, H=64, masks=[[1], [1]], seed=15)
    d = p.device()
    o, lse = run_all(p, d)
    o2, lse2 = out_buffers(p)
    n = tp.tpla_workspace_bytes_all(p.shape, p.max_pages, 0)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    tp.tpla_decode_shards(p.shape, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"] + 1, 0, ws, n, o2, lse2)
    torch.cuda.synchronize()
    _, _, o_off, lse_off = p.expected()
    assert (np.abs(o - o2.cpu().numpy()) <= 2 * o_off).all()          # both round their weights to bf16
    # (the sum of the decode kernel is that of its rounded weights)
    assert (np.abs(lse - lse2.cpu().numpy()) <= 2 * lse_off + 2.0 ** -8).all()


def test_pools_beyond_32_bit_offsets():
    """Pages behind 4 GiB and 2^31 elements; only the pages in use are written."""
    p = TreeProblem([100, 30], [4, 4], 4, H=16, g=1, spare_pages=0, seed=16)
    d = p.device()
    used = p.pools[0].shape[0]
    n_pool = 120000                                            # 64 x 320 elements each: 2.46e9 elements, 4.9 GB
    big = torch.empty((n_pool, 64, 320), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([n_pool - 1 - 7001 * k for k in range(used)])
    assert int(ids.min()) >= 0
    for k in range(used):
        big[int(ids[k])] = d["pools"][0][k]
    p.bt = ids.numpy().astype(np.int32)[np.minimum(p.bt, used - 1)]
    d["pools"], d["bt"] = [big], torch.from_numpy(p.bt).cuda()
    o, lse = out_buffers(p)
    ws, n = workspace(p)
    tp.tpla_decode_shards_tree(p.shape, p.T, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"], d["drafts"], d["masks"],
                               ws, n, o, lse)
    torch.cuda.synchronize()
    back = {int(v): k for k, v in enumerate(ids)}
    p.bt = np.vectorize(lambda v: back[int(v)])(p.bt).astype(np.int32)
    assert_close(p, o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64))


def test_captured_into_a_graph():
    p = TreeProblem([2100, 65], [4, 3], 4, H=64, seed=17)
    q = TreeProblem([900, 33], [2, 4], 4, H=64, seed=18, max_pages=p.max_pages)
    d, e = p.device(), q.device()
    want_p, want_q = run_all(p, d), run_all(q, e)
    o, lse = out_buffers(p)
    ws, n = workspace(p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tp.tpla_decode_shards_tree(p.shape, p.T, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"], d["drafts"],
                                   d["masks"], ws, n, o, lse)
    keep = {k: d[k].clone() for k in ("q_lat", "q_pe", "lens", "drafts", "masks")}
    for it in range(4):
        o.fill_(float("nan"))
        if it % 2:                                             # same lengths' table, other queries, lengths and masks
            d["lens"].copy_(keep["lens"] // 2)
        else:
            d["lens"].copy_(keep["lens"])
        graph.replay()
        torch.cuda.synchronize()
        if it % 2 == 0:
            assert np.array_equal(o.cpu().numpy(), want_p[0].astype(np.float32)) and np.array_equal(lse.cpu().numpy(), want_p[1].astype(np.float32))
        else:
            h = TreeProblem([2100, 65], [4, 3], 4, H=64, seed=17)
            h.lens = [v // 2 for v in h.lens]
            assert_close(h, o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64))
    again = run_all(q, e)
    assert all(np.array_equal(x, y) for x, y in zip(again, want_q))


@pytest.mark.parametrize("dl,g", [(256, 2), (128, 2), (64, 4)])
@pytest.mark.parametrize("lens", [[63, 64, 65, 0, 31, 32, 33, 95], [1500, 700, 1100, 333, 64, 2000, 129, 905]])
def test_every_number_of_row_blocks(dl, g, lens):
    """Blocks of 16 rows 1 to 8 of an item: a block alone has both halves of a round, one with a second wave half of it."""
    p = TreeProblem(lens, [1, 2, 3, 4, 5, 6, 7, 8], 8, H=16, g=g, dl=dl, seed=dl + len(lens) + lens[0], max_pages=WIDE)
    o, lse = run_all(p)
    assert_close(p, o, lse)


@pytest.mark.parametrize("T", [3, 5, 6, 7])
def test_masked_infinities_where_blocks_have_one_or_two_waves(T):
    for L in (0, 37, 63, 64, 90):
        p = TreeProblem([L, 40, 700], [T, T - 1, T], T, H=16, masks=chain_masks(3, T), seed=L + T, max_pages=WIDE)
        p.masks[:, 1:] &= ~np.uint64(1)                          # draft 0 is seen by itself alone
        clean = p.expected()
        for b in range(3):
            page, off = p.row_of(b, [L, 40, 700][b])
            for i in range(2):
                p.pools[i][page, off, ::2] = 0x7FC0
                p.pools[i][page, off, 1::2] = 0x7F80
        o, lse = run_all(p)
        assert np.isnan(o[:, :, 0]).all() and np.isnan(lse[:, :, 0]).all()
        o[:, :, 0], lse[:, :, 0] = clean[0][:, :, 0], clean[1][:, :, 0]
        assert_close(p, o, lse, clean)


@pytest.mark.parametrize("H,T", [(16, 3), (16, 7), (64, 3)])
def test_long_tables_in_pools_beyond_32_bit_offsets(H, T):
    p = TreeProblem([300, 30], [T, T], T, H=H, g=1, spare_pages=0, seed=19 + T, max_pages=WIDE)
    d = p.device()
    used, n_pool = p.pools[0].shape[0], 120000
    big = torch.empty((n_pool, 64, 320), dtype=torch.bfloat16, device="cuda")
    ids = np.array([n_pool - 1 - 7001 * k for k in range(used)], dtype=np.int32)
    assert ids.min() >= 0
    for k in range(used):
        big[int(ids[k])] = d["pools"][0][k]
    table = torch.from_numpy(ids[np.clip(p.bt, 0, used - 1)]).cuda()
    o, lse = out_buffers(p)
    ws, n = workspace(p)
    tp.tpla_decode_shards_tree(p.shape, p.T, d["q_lat"], d["q_pe"], [big], table, p.max_pages, d["lens"], d["drafts"], d["masks"], ws, n, o, lse)
    torch.cuda.synchronize()
    assert_close(p, o.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64))


@pytest.mark.parametrize("H,T,wide", [(16, 3, WIDE), (16, 7, WIDE), (64, 3, WIDE), (64, 4, None)])
def test_two_graphs_that_share_a_workspace(H, T, wide):
    """Replayed one after the other on a stream, with other work in between: each has the eager call's bits every time."""
    problems = [TreeProblem([2100, 65, 500], [T, 1, T], T, H=H, seed=23, max_pages=wide or 64),
                TreeProblem([90, 1333, 4000], [1, T, T - 1], T, H=H, seed=24, max_pages=wide or 64)]
    devs = [p.device() for p in problems]
    want = [run_all(p, d) for p, d in zip(problems, devs)]
    ws, n = workspace(problems[0])
    assert n >= workspace(problems[1])[1]
    outs, graphs = [out_buffers(p) for p in problems], []
    for p, d, (o, lse) in zip(problems, devs, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            tp.tpla_decode_shards_tree(p.shape, p.T, d["q_lat"], d["q_pe"], d["pools"], d["bt"], p.max_pages, d["lens"], d["drafts"],
                                       d["masks"], ws, n, o, lse)
        graphs.append(graph)
    for it in range(4):
        for k in ((0, 1), (1, 0), (0, 0), (1, 1))[it]:
            o, lse = outs[k]
            o.fill_(float("nan"))
            lse.fill_(float("nan"))
            graphs[k].replay()
            graphs[1 - k].replay()                           # the other one uses the workspace right behind it
            torch.cuda.synchronize()
            assert np.array_equal(o.cpu().numpy(), want[k][0].astype(np.float32)) and np.array_equal(lse.cpu().numpy(), want[k][1].astype(np.float32))
