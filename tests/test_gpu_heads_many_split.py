"""Rows of more than 64 sequences whose tokens are split in the 128-row kernel: parts, their slots and the merge across groups of 64 sequences, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from heads_common import CODE, DTYPE, Cached, check

pytestmark = pytest.mark.gpu


def lengths(B, long, seed):
    """Mostly short, empty ones among them, the long ones in every group of 64."""
    r = np.random.default_rng(seed)
    n = r.integers(0, 400, B)
    n[r.random(B) < 0.15] = 0
    n[[3, 70, B - 1, B - 2, 66, 64, 63]] = [long, long - 517, long + 3, 513, 1024, 1025, 2049]
    return n.tolist()


def part_tokens(workspace):
    """Tokens of a part, which the first workgroup notes behind the partial results: the last 16 bytes of a workspace of this call's size."""
    return int(workspace[-16:-12].view(torch.int32).item())


@pytest.mark.parametrize("H,H_kv,d,page,dtype_o", [(48, 1, 128, 64, "f32"), (130, 1, 64, 32, "bf16"), (144, 3, 64, 16, "f32"), (40, 1, 128, 48, "bf16")])
@pytest.mark.parametrize("B", [100, 150])
def test_decode(H, H_kv, d, page, dtype_o, B):
    lens = lengths(B, 3301, B + H)
    c = Cached(lens, H, H_kv, d, page=page, seed=B, sharp=1.5)
    c.queries(B)
    x = c.on()
    n = tp.tpla_workspace_bytes_heads(c.shape, c.max_pages)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    o = torch.full((B, H, d), float("nan"), dtype=DTYPE[dtype_o], device="cuda")
    lse = torch.full((B, H), float("nan"), device="cuda")
    tp.tpla_decode_heads(c.shape, x["q"], x["k_pool"], x["v_pool"], x["table"], c.max_pages, x["ints"](lens), ws, n, o, CODE[dtype_o], lse)
    torch.cuda.synchronize()
    assert 512 <= part_tokens(ws) < max(lens)
    o, lse = o.double().cpu().numpy(), lse.double().cpu().numpy()
    for b, k in enumerate(lens):
        check("bf16", dtype_o, d, o[b], lse[b], *c.want(b, b, k), "sequence %d, %d tokens" % (b, k))


@pytest.mark.parametrize("H,H_kv,d,page", [(8, 2, 128, 64), (6, 1, 64, 16)])
def test_prefill(H, H_kv, d, page):
    B = 90
    lens = lengths(B, 2600, H)
    news = [(5 * b) % 13 for b in range(B)]
    news[1], news[65], news[70], news[B - 1] = 75, 101, 60, 40
    c = Cached([a + b for a, b in zip(news, lens)], H, H_kv, d, page=page, seed=H, sharp=1.5)
    T = sum(news)
    c.queries(T)
    x = c.on()
    n = tp.tpla_workspace_bytes_prefill_heads(c.shape, T, max(news), c.max_pages)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    o = torch.full((T, H, d), float("nan"), device="cuda")
    lse = torch.full((T, H), float("nan"), device="cuda")
    cu = x["ints"]([sum(news[:b]) for b in range(B + 1)])
    tp.tpla_prefill_heads(c.shape, x["q"], x["k_pool"], x["v_pool"], x["table"], c.max_pages, x["ints"](lens), cu, T, max(news), ws, n, o, tp.TPLA_F32, lse)
    torch.cuda.synchronize()
    assert 512 <= part_tokens(ws) < max(c.keys)
    o, lse, first = o.double().cpu().numpy(), lse.double().cpu().numpy(), 0
    for b, k in enumerate(news):
        for i in range(k):
            check("bf16", "f32", d, o[first + i], lse[first + i], *c.want(b, first + i, lens[b] + i + 1), "sequence %d, new token %d of %d" % (b, i, k))
        first += k
