"""Attention of grouped heads over paged keys and values against 64 bits: single tokens and prompts, every kernel."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from heads_common import CODE, DTYPE, HALF_STEP, Cached, check, decode_parity, prefill_parity, run_decode, run_prefill

pytestmark = pytest.mark.gpu

# H, H_kv, d_k, d_v, page, dtype
SHAPES = [(8, 2, 128, 128, 64, "bf16"), (48, 1, 128, 128, 64, "bf16"), (130, 1, 64, 64, 32, "bf16"), (4, 4, 64, 64, 16, "bf16"), (16, 1, 128, 128, 32, "bf16"), (5, 1, 64, 64, 64, "bf16"), (40, 2, 128, 128, 128, "bf16"),
          (35, 1, 64, 64, 48, "bf16"), (6, 2, 96, 96, 16, "bf16"), (4, 2, 128, 64, 64, "bf16"), (4, 2, 128, 128, 24, "bf16"), (3, 1, 256, 256, 64, "bf16"),
          (6, 2, 96, 96, 16, "f32"), (4, 1, 64, 64, 64, "f32"), (2, 2, 24, 8, 7, "f32"), (12, 1, 128, 128, 64, "f32"), (2, 1, 256, 200, 64, "f32"), (1, 1, 8, 32, 5, "f32")]
IDS = ["-".join(map(str, s)) for s in SHAPES]


@pytest.mark.parametrize("H,H_kv,d_k,d_v,page,dtype", SHAPES, ids=IDS)
def test_decode_lengths(H, H_kv, d_k, d_v, page, dtype):
    lens = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 300, 1025]
    c = Cached(lens, H, H_kv, d_k, d_v, page, dtype)
    c.queries(len(lens))
    decode_parity(c, lens)
    decode_parity(c, lens, "f32")


@pytest.mark.parametrize("H,H_kv,d_k,d_v,page,dtype", SHAPES, ids=IDS)
@pytest.mark.parametrize("B", [5, 150])
def test_decode_short_sequences_in_narrow_and_wide_tables(H, H_kv, d_k, d_v, page, dtype, B):
    """How the work is cut follows from the width of the block table and the number of items, which the lengths do not tell."""
    lens = [(37 * b) % 301 for b in range(B)]
    for width in (-(-301 // page), -(-1500 // page), -(-20000 // page)):
        c = Cached(lens, H, H_kv, d_k, d_v, page, dtype, max_pages=width, seed=width)
        c.queries(B)
        decode_parity(c, lens)


@pytest.mark.parametrize("H,H_kv,d_k,d_v,page,dtype", SHAPES, ids=IDS)
@pytest.mark.parametrize("new", [1, 3, 12, 40])
def test_a_few_new_tokens_in_narrow_and_wide_tables(H, H_kv, d_k, d_v, page, dtype, new):
    news, lens = [new, 1, new, new - 1, new], [0, 130, 255, 17, 300]
    for width in (-(-400 // page), -(-5000 // page)):
        c = Cached([a + b for a, b in zip(news, lens)], H, H_kv, d_k, d_v, page, dtype, max_pages=width, seed=width)
        c.queries(sum(news))
        prefill_parity(c, news, lens)


@pytest.mark.parametrize("H,H_kv,d_k,d_v,page,dtype", SHAPES, ids=IDS)
def test_decode_one_long_sequence(H, H_kv, d_k, d_v, page, dtype):
    c = Cached([5003], H, H_kv, d_k, d_v, page, dtype, sharp=2.0)
    c.queries(1)
    decode_parity(c, [5003])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_lengths_out_of_range_and_missing_pages(dtype):
    c = Cached([256, 256, 200, 200, 130, 64], 8, 2, 128, page=64, dtype=dtype, missing={2: [1], 3: [0, 3], 4: [0, 1, 2], 5: [0]}.items())
    c.queries(6)
    decode_parity(c, [1000, -5, 200, 200, 130, 64])


def test_decode_writes_no_lse_and_repeats_to_the_bit():
    c = Cached([3000, 1, 700], 32, 8, 128)
    c.queries(3)
    a, _ = run_decode(c, [3000, 1, 700], with_lse=False)
    b, _ = run_decode(c, [3000, 1, 700])
    assert np.array_equal(a, b)


PROMPTS = [([1], [0]), ([1, 1, 1], [0, 5, 200]), ([17, 64, 3, 100], None), ([130, 1, 65], [0, 64, 37]), ([0, 40, 0, 9], [10, 0, 0, 300]), ([257], [1000]), ([2, 2], [0, 1500])]


@pytest.mark.parametrize("H,H_kv,d_k,d_v,page,dtype", SHAPES, ids=IDS)
@pytest.mark.parametrize("news,lens", PROMPTS, ids=["one", "ones", "prompts", "parts", "empty", "long_part", "few_rows"])
def test_prefill(H, H_kv, d_k, d_v, page, dtype, news, lens):
    keys = [a + (lens[b] if lens else 0) for b, a in enumerate(news)]
    c = Cached(keys, H, H_kv, d_k, d_v, page, dtype)
    c.queries(sum(news))
    prefill_parity(c, news, lens)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_long_prompt(dtype):
    c = Cached([1500], 4, 1, 128, dtype=dtype, sharp=1.5)
    c.queries(1500)
    prefill_parity(c, [1500], [0], "f32", rows=[0, 1, 31, 32, 63, 64, 127, 128, 500, 511, 512, 1000, 1498, 1499])


@pytest.mark.parametrize("H,H_kv,d,page,dtype", [(4, 2, 128, 64, "bf16"), (6, 1, 64, 16, "bf16"), (2, 1, 32, 16, "f32")])
def test_prefill_many_sequences(H, H_kv, d, page, dtype):
    news, lens = [(7 * b) % 23 for b in range(150)], [(b * b) % 61 for b in range(150)]
    c = Cached([a + b for a, b in zip(news, lens)], H, H_kv, d, page=page, dtype=dtype)
    c.queries(sum(news))
    prefill_parity(c, news, lens)


def wanted(q, k_pool, v_pool, ids, seen, G, scale):
    """o of one row of q [H, d] over the first `seen` tokens of pages `ids`, and the sum of weight |value|, in 64 bits on the GPU."""
    d = q.shape[1]
    K, V = (p[ids].double().transpose(0, 1).reshape(p.shape[1], -1, d)[:, :seen] for p in (k_pool, v_pool))
    s = (K @ q.double().reshape(-1, G, d).transpose(1, 2)).transpose(1, 2) * scale
    p = torch.softmax(s, -1)
    return (p @ V).reshape(-1, d), (p @ V.abs()).reshape(-1, d)


def test_more_pages_than_are_held_at_once():
    """Tokens of more than a thousand small pages in one workgroup: a long prompt that is not split, and ranges of many long sequences."""
    d, page, n = 64, 16, 17003
    pages = -(-n // page)
    pools = [torch.randn((pages, 4, page, d), device="cuda").to(torch.bfloat16) for _ in range(2)]
    table = torch.randperm(pages, device="cuda").to(torch.int32)[None].contiguous()
    shape = tp.TplaHeads(1, 8, 4, d, d, page, tp.TPLA_BF16, d ** -0.5)
    q = (4 * torch.randn((n, 8, d), device="cuda")).to(torch.bfloat16)            # few tokens weigh: a lost one is seen
    o = torch.empty((n, 8, d), device="cuda")
    size = tp.tpla_workspace_bytes_prefill_heads(shape, n, n, pages)
    ws, cu = torch.empty(max(16, size), dtype=torch.uint8, device="cuda"), torch.tensor([0, n], dtype=torch.int32, device="cuda")
    tp.tpla_prefill_heads(shape, q, *pools, table, pages, None, cu, n, n, ws, size, o, tp.TPLA_F32, None)
    for row in (0, 5000, 16300, 16367, 16368, 16400, 17002):
        want, span = wanted(q[row], *pools, table[0].long(), row + 1, 2, d ** -0.5)
        assert ((o[row].double() - want).abs() <= (2 * HALF_STEP["bf16"] + 2.0 ** -11) * span).all(), row       # the weights' roundings (see check), floats
    B, n, G = 520, 16700, 2
    pages = -(-n // page)
    pools = [torch.randn((4000, 1, page, d), device="cuda").to(torch.bfloat16) for _ in range(2)]          # sequences share pages: legal for reading
    table = torch.randint(0, 4000, (B, pages), device="cuda").to(torch.int32)
    shape = tp.TplaHeads(B, G, 1, d, d, page, tp.TPLA_BF16, d ** -0.5)
    q, o = (4 * torch.randn((B, G, d), device="cuda")).to(torch.bfloat16), torch.empty((B, G, d), device="cuda")
    size = tp.tpla_workspace_bytes_heads(shape, pages)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    tp.tpla_decode_heads(shape, q, *pools, table, pages, torch.full((B,), n, dtype=torch.int32, device="cuda"), ws, size, o, tp.TPLA_F32, None)
    for b in (0, 1, 259, 518, 519):
        want, span = wanted(q[b], *pools, table[b].long(), n, G, d ** -0.5)
        assert ((o[b].double() - want).abs() <= (2 * HALF_STEP["bf16"] + 2.0 ** -11) * span).all(), b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_missing_pages_and_the_end_of_the_table(dtype):
    c = Cached([230, 300, 90], 8, 2, 64, page=64, dtype=dtype, missing={0: [0], 1: [1, 4], 2: [0, 1]}.items())
    c.queries(230 + 100 + 90)
    prefill_parity(c, [230, 100, 90], [0, 200, 0])            # whole rows of the first and third see nothing
    # tokens beyond the table's row are not there: sequence 1 has room for 320 tokens
    c = Cached([320], 8, 2, 64, page=64, dtype=dtype)
    c.queries(60)
    prefill_parity(c, [60], [290])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prefill_rows_that_are_left_alone(dtype):
    c = Cached([50, 30], 4, 2, 128, dtype=dtype)
    c.queries(100)
    got, lse = run_prefill(c, [50, 30], None, "f32", max_new=40, T=100, cu=[0, 50, 80])
    full, full_lse = run_prefill(c, [50, 30], None, "f32", T=100, cu=[0, 50, 80])
    rows = list(range(40)) + list(range(50, 80))
    assert np.allclose(got[rows], full[rows], atol=2e-2 if dtype == "bf16" else 1e-5)
    assert np.isnan(got[40:50]).all() and np.isnan(got[80:]).all() and np.isnan(full[80:]).all() and np.isnan(lse[80:]).all()
    # malformed row ranges are clipped: nothing outside the buffers is touched
    run_prefill(c, [50, 30], None, "f32", max_new=100, T=100, cu=[-7, 60, 1000])
    run_prefill(c, [50, 30], None, "f32", max_new=100, T=100, cu=[70, 20, 90])


@pytest.mark.parametrize("H,H_kv,d,page,dtype", [(8, 2, 128, 64, "bf16"), (4, 4, 64, 16, "bf16"), (16, 1, 64, 64, "bf16"), (4, 2, 96, 16, "bf16"), (4, 2, 128, 64, "f32"), (32, 1, 64, 16, "f32")])
@pytest.mark.parametrize("new,cached", [(150, 0), (3, 120), (70, 333)])
def test_values_that_are_not_finite_reach_no_row_that_does_not_see_them(H, H_kv, d, page, dtype, new, cached):
    at = [cached + new // 2, cached + new - 1]                # two new tokens

    def edit(b, k, v):
        v[:, at[0], 3] = float("inf")
        v[:, at[0], d - 1] = float("nan")
        v[:, at[1]] = -float("inf")
        k[:, at[1], 0] = float("nan")

    c = Cached([cached + new], H, H_kv, d, page=page, dtype=dtype, edit=edit)
    c.queries(new)
    got, lse = run_prefill(c, [new], [cached])
    for i in range(new):
        if i >= new // 2 and i < new - 1:
            o, want_lse, span = c.want(0, i, cached + i + 1)
            cols = [x for x in range(d) if x not in (3, d - 1)]
            assert np.isposinf(got[i][:, 3]).all() and np.isnan(got[i][:, d - 1]).all()
            check(dtype, dtype, d, got[i][:, cols], lse[i], o[:, cols], want_lse, span[:, cols])
        elif i == new - 1:
            assert np.isnan(got[i]).all()
        else:
            o, want_lse, span = c.want(0, i, cached + i + 1)
            check(dtype, dtype, d, got[i], lse[i], o, want_lse, span, "new token %d" % i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_that_are_not_finite(dtype):
    lens = [700, 700, 700, 700, 3, 700]

    def edit(b, k, v):
        if b == 0:
            k[:, 650, 1] = float("nan")                       # one score is NaN
        if b == 1:
            k[:, :, 0] = -float("inf")                        # all scores are -inf
        if b == 2:
            k[:, 100:400, 0] = -float("inf")                  # some are: those tokens weigh nothing
        if b == 3:
            k[:, 17, 0] = float("inf")
        if b == 4:
            k[:, :, 0] = -float("inf")

    c = Cached(lens, 8, 2, 64, dtype=dtype, edit=edit)
    c.queries(len(lens))
    c.q[:, :, 0] = 1.0
    c.q64[:, :, 0] = 1.0
    got, lse = run_decode(c, lens)
    for b in (0, 1, 3, 4):
        assert np.isnan(got[b]).all(), b
    assert np.isneginf(lse[1]).all() and np.isneginf(lse[4]).all()
    c.there[2][100:400] = False
    for b in (2, 5):
        o, want_lse, span = c.want(b, b, 700)
        check(dtype, dtype, 64, got[b], lse[b], o, want_lse, span)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 96)])
def test_captured_calls_on_another_stream_share_a_workspace(dtype, d):
    """Two graphs over one workspace, replayed in turn with eager calls between them."""
    B, news = 3, [40, 1, 77]
    c = Cached([2500, 90, 700], 8, 2, d, dtype=dtype)
    c.queries(sum(news))
    lens = [2500, 90, 700]
    before = [a - b for a, b in zip(lens, news)]
    x = c.on()
    T = sum(news)
    n = max(tp.tpla_workspace_bytes_heads(c.shape, c.max_pages), tp.tpla_workspace_bytes_prefill_heads(c.shape, T, max(news), c.max_pages))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    cu, all_lens, first = x["ints"]([0, 40, 41, 118]), x["ints"](lens), x["ints"](before)
    out = lambda rows: (torch.zeros((rows, 8, d), dtype=DTYPE[dtype], device="cuda"), torch.zeros((rows, 8), device="cuda"))  # noqa: E731
    od, op = out(B), out(T)
    q1 = x["q"][:B].contiguous()

    def decode():
        tp.tpla_decode_heads(c.shape, q1, x["k_pool"], x["v_pool"], x["table"], c.max_pages, all_lens, ws, n, od[0], CODE[dtype], od[1])

    def prefill():
        tp.tpla_prefill_heads(c.shape, x["q"], x["k_pool"], x["v_pool"], x["table"], c.max_pages, first, cu, T, max(news), ws, n, op[0], CODE[dtype], op[1])

    decode()
    prefill()
    torch.cuda.synchronize()
    want = [t.clone() for t in (*od, *op)]
    graphs, stream = [], torch.cuda.Stream()
    for fn in (decode, prefill):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            fn()
        graphs.append(g)
    for _ in range(3):
        for t in (*od, *op):
            t.zero_()
        ws.fill_(0xFF)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*od, *op), want))
        for t in (*od, *op):
            t.zero_()
        prefill()
        decode()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*od, *op), want))
