"""Norm, position and cache append of grouped heads against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from heads_common import CODE, DTYPE, HALF_STEP, shape_of, stored

pytestmark = pytest.mark.gpu
EPS = 1e-6


def turned(x, weight, eps, rot, layout, freq, positions, amplitude):
    """Rows [T, heads, d] in 64 bits, and the length of every column's pair (what float errors are relative to)."""
    if eps >= 0:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * weight
    y, size, n = x.copy(), np.abs(x), rot // 2
    if n:
        a = positions[:, None, None] * freq
        i, j = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if layout == tp.TPLA_ROTARY_INTERLEAVED else (np.arange(n), np.arange(n) + n)
        u, v = x[..., i], x[..., j]
        y[..., i], y[..., j] = amplitude * (u * np.cos(a) - v * np.sin(a)), amplitude * (u * np.sin(a) + v * np.cos(a))
        size[..., i] = size[..., j] = abs(amplitude) * np.hypot(u, v)
    return y, size


def close(dtype, got, want, size):
    """One rounding of the result, and floats: 13 additions and a root and a quotient in the norm, two products for the weight, the sine (its argument
    is off by half a step of up to pi) and the turn: below 32 half steps of a float relative to the pair."""
    got = got.double().cpu().numpy()
    slop = 32 * 2.0 ** -24 * size
    off = np.abs(got - want) - (HALF_STEP[dtype] * (np.abs(want) + slop) + slop)
    assert not np.any(off > 0), float(off.max())


CASES = [(1, 32, 8, 128, 128, "half", "bf16"), (7, 5, 1, 64, 64, "interleaved", "bf16"), (300, 6, 2, 96, 48, "half", "bf16"), (33, 4, 4, 128, 64, "interleaved", "f32"),
         (65, 3, 1, 64, 60, "half", "bf16"), (9, 3, 3, 40, 26, "half", "f32"), (5, 2, 1, 256, 256, "half", "bf16"), (12, 2, 2, 8, 8, "half", "f32"), (700, 17, 1, 24, 0, "half", "bf16"),
         (1100, 8, 2, 32, 32, "half", "bf16"), (3, 200, 100, 128, 128, "half", "bf16"), (4, 6, 2, 200, 200, "half", "f32"),
         (31, 5, 5, 64, 36, "interleaved", "bf16"), (2100, 24, 3, 64, 64, "half", "bf16"), (2049, 3, 1, 32, 20, "interleaved", "f32")]


def problem(T, H, H_kv, d, rot, layout, dtype, seed=3, d_v=None):
    r = np.random.default_rng([seed, T, H, d])
    d_v = d_v or d
    wide = torch.full((T, H + H_kv + 1, d), float("nan"), dtype=DTYPE[dtype])
    x, x64 = stored(r.standard_normal((T, H + H_kv, d)) * 2, dtype)
    wide[:, 1:] = x
    p = dict(qk=wide.cuda(), q64=x64[:, :H], k64=x64[:, H:], freq=tp.tpla_rotary_frequencies(rot, 500000.0) if rot else np.zeros(0),
             positions=r.integers(0, 300000, T).astype(np.int32), layout=tp.TPLA_ROTARY_HALF if layout == "half" else tp.TPLA_ROTARY_INTERLEAVED)
    p["q"], p["k"] = p["qk"][:, 1:1 + H], p["qk"][:, 1 + H:]
    p["wq"], p["wq64"] = stored(1 + 0.2 * r.standard_normal(d), dtype)
    p["wk"], p["wk64"] = stored(1 + 0.2 * r.standard_normal(d), dtype)
    v, p["v64"] = stored(r.standard_normal((T, H_kv, d_v)), dtype)
    p["v"], p["wq"], p["wk"] = v.cuda(), p["wq"].cuda(), p["wk"].cuda()
    p["freq_gpu"] = torch.from_numpy(p["freq"]).cuda() if rot else None
    p["pos_gpu"] = torch.from_numpy(p["positions"]).cuda() if rot else None
    return p


@pytest.mark.parametrize("T,H,H_kv,d,rot,layout,dtype", CASES)
def test_norm_and_rotary(T, H, H_kv, d, rot, layout, dtype):
    p = problem(T, H, H_kv, d, rot, layout, dtype)
    shape = shape_of(1, H, H_kv, d, dtype=dtype)
    for eps, wq, wk, wq64, wk64, amplitude in ((EPS, p["wq"], p["wk"], p["wq64"], p["wk64"], 1.0), (0.5, None, p["wk"], None, p["wk64"], 1.3), (-1.0, None, None, None, None, -0.7)):
        q_out, k_out = (torch.full((T, n, d), float("nan"), dtype=DTYPE[dtype], device="cuda") for n in (H, H_kv))
        tp.tpla_norm_rotary_heads(shape, p["layout"], rot, p["freq_gpu"], amplitude, wq, wk, eps, p["pos_gpu"], T, p["q"], q_out, p["k"], k_out)
        for got, x, w in ((q_out, p["q64"], wq64), (k_out, p["k64"], wk64)):
            close(dtype, got, *turned(x, w, np.float64(np.float32(eps)), rot, p["layout"], p["freq"], p["positions"], np.float64(np.float32(amplitude))))
    # one of the pairs alone, in place
    before = p["qk"].clone()
    tp.tpla_norm_rotary_heads(shape, p["layout"], rot, p["freq_gpu"], 1.0, None, p["wk"], EPS, p["pos_gpu"], T, None, None, p["k"], p["k"])
    close(dtype, p["k"], *turned(p["k64"], p["wk64"], np.float64(np.float32(EPS)), rot, p["layout"], p["freq"], p["positions"], 1.0))
    assert torch.equal(p["qk"][:, :1 + H].nan_to_num(), before[:, :1 + H].nan_to_num())


@pytest.mark.parametrize("T,H,H_kv,d,rot,layout,dtype", CASES)
@pytest.mark.parametrize("page,wider", [(64, 0), (5, 16)])
def test_append(T, H, H_kv, d, rot, layout, dtype, page, wider):
    if d + wider > 256:
        wider = 0
    p = problem(T, H, H_kv, d, rot, layout, dtype, d_v=d + wider)
    shape = shape_of(1, H, H_kv, d, d + wider, page, dtype)
    r = np.random.default_rng(T)
    n_pages = -(-T // page) + 2
    slots = r.permutation(n_pages * page)[:T].astype(np.int32)
    slots[r.random(T) < 0.2] = -1
    pools = [torch.full((n_pages, H_kv, page, w), 7.0, dtype=DTYPE[dtype], device="cuda") for w in (d, d + wider)]
    q_out = torch.full((T, H, d), float("nan"), dtype=DTYPE[dtype], device="cuda")
    tp.tpla_append_heads(shape, p["layout"], rot, p["freq_gpu"], 1.0, p["wq"], p["wk"], EPS, p["pos_gpu"], T, p["q"], q_out, p["k"], p["v"],
                         torch.from_numpy(slots).cuda(), *pools)
    eps = np.float64(np.float32(EPS))
    close(dtype, q_out, *turned(p["q64"], p["wq64"], eps, rot, p["layout"], p["freq"], p["positions"], 1.0))
    k, size = turned(p["k64"], p["wk64"], eps, rot, p["layout"], p["freq"], p["positions"], 1.0)
    used = np.nonzero(slots >= 0)[0]
    rows = [x.transpose(1, 2).reshape(n_pages * page, H_kv, -1) for x in pools]
    at = torch.from_numpy(slots[used]).long().cuda()
    close(dtype, rows[0][at], k[used], size[used])
    assert np.array_equal(rows[1][at].double().cpu().numpy(), p["v64"][used])
    rest = np.setdiff1d(np.arange(n_pages * page), slots[used])
    assert all((x[torch.from_numpy(rest).cuda()] == 7.0).all() for x in rows)
    # without queries: the same cache
    more = [torch.full_like(x, 7.0) for x in pools]
    tp.tpla_append_heads(shape, p["layout"], rot, p["freq_gpu"], 1.0, None, p["wk"], EPS, p["pos_gpu"], T, None, None, p["k"], p["v"],
                         torch.from_numpy(slots).cuda(), *more)
    assert all(torch.equal(a, b) for a, b in zip(pools, more))


def test_values_that_are_not_finite_stay_in_their_row():
    T, H, H_kv, d = 6, 4, 2, 64
    p = problem(T, H, H_kv, d, d, "half", "bf16")
    p["q"][2, 1, 5] = float("inf")
    p["q"][3, 0, 7] = float("nan")
    p["q"][4, 2] = 0
    q_out = torch.full((T, H, d), 3.0, dtype=torch.bfloat16, device="cuda")
    tp.tpla_norm_rotary_heads(shape_of(1, H, H_kv, d), p["layout"], d, p["freq_gpu"], 1.0, p["wq"], None, EPS, p["pos_gpu"], T, p["q"], q_out, None, None)
    odd = ~torch.isfinite(q_out).all(-1)
    want = torch.zeros((T, H), dtype=torch.bool, device="cuda")
    want[2, 1] = want[3, 0] = True
    assert torch.equal(odd, want) and (q_out[4, 2] == 0).all()


def test_more_tokens_than_a_launch_has():
    """Tokens around the borders of the parts that a long call goes in, on other rows than theirs if a stride were lost."""
    T, H, d = (1 << 20) * 2 + 77, 2, 8
    shape = shape_of(1, H, 1, d)
    x = torch.randn((T, H + 1, d), device="cuda").to(torch.bfloat16)
    pos = torch.arange(T, dtype=torch.int32, device="cuda") % 5000
    freq = torch.from_numpy(tp.tpla_rotary_frequencies(d, 10000.0)).cuda()
    q_out, k_out = torch.empty((T, H, d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 1, d), dtype=torch.bfloat16, device="cuda")
    tp.tpla_norm_rotary_heads(shape, tp.TPLA_ROTARY_HALF, d, freq, 1.0, None, None, EPS, pos, T, x[:, :H], q_out, x[:, H:], k_out)
    page, slots = 64, torch.arange(T, dtype=torch.int32, device="cuda")
    pools = [torch.zeros((T // page + 1, 1, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    q2 = torch.empty_like(q_out)
    tp.tpla_append_heads(shape, tp.TPLA_ROTARY_HALF, d, freq, 1.0, None, None, EPS, pos, T, x[:, :H], q2, x[:, H:], x[:, H:], slots, *pools)
    at = torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 21) - 1, 1 << 21, T - 1], device="cuda")
    rows = x[at].double().cpu().numpy()
    want, size = turned(rows, None, np.float64(np.float32(EPS)), d, tp.TPLA_ROTARY_HALF, freq.cpu().numpy(), pos[at].cpu().numpy(), 1.0)
    close("bf16", q_out[at], want[:, :H], size[:, :H])
    close("bf16", k_out[at], want[:, H:], size[:, H:])
    assert torch.equal(q_out, q2) and torch.equal(pools[0].reshape(-1, d)[:T], k_out[:, 0]) and torch.equal(pools[1].reshape(-1, d)[:T], x[:, H])


def test_pools_beyond_32_bit_offsets():
    """Slots behind 2^32 bytes of a pool (and 2^31 elements)."""
    H_kv, d, page = 8, 128, 64
    n_pages = (2 ** 31 // (H_kv * page * d)) + 40
    pools = [torch.empty((n_pages, H_kv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    T = 70
    p = problem(T, 8, H_kv, d, d, "half", "bf16")
    slots = torch.arange(T, dtype=torch.int32, device="cuda") * 3 + (n_pages - 6) * page
    tp.tpla_append_heads(shape_of(1, 8, H_kv, d), p["layout"], d, p["freq_gpu"], 1.0, None, p["wk"], EPS, p["pos_gpu"], T, None, None, p["k"], p["v"], slots, *pools)
    s = slots.long()
    assert np.array_equal(pools[1][s // page, :, s % page].double().cpu().numpy(), p["v64"])
    close("bf16", pools[0][s // page, :, s % page], *turned(p["k64"], p["wk64"], np.float64(np.float32(EPS)), d, p["layout"], p["freq"], p["positions"], 1.0))
    # and the attention that reads them: the 70 tokens lie every third slot, so a sequence of 1 token per page entry
    table = torch.arange(n_pages - 6, n_pages, dtype=torch.int32, device="cuda")[None]
    for x in pools:
        x[n_pages - 6:] = torch.randn_like(x[n_pages - 6:])
    shape, low = shape_of(1, 8, H_kv, d), [x[n_pages - 6:].clone() for x in pools]
    q = torch.randn((1, 8, d), device="cuda").to(torch.bfloat16)
    n = tp.tpla_workspace_bytes_heads(shape, 6)
    ws, lens = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.tensor([6 * page - 3], dtype=torch.int32, device="cuda")
    out = []
    for k_pool, v_pool, t in ((*pools, table), (*low, table - (n_pages - 6))):
        o = torch.empty((1, 8, d), dtype=torch.float32, device="cuda")
        tp.tpla_decode_heads(shape, q, k_pool, v_pool, t.contiguous(), 6, lens, ws, n, o, CODE["f32"], None)
        o2 = torch.empty((1, 8, d), dtype=torch.float32, device="cuda")
        cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
        n2 = tp.tpla_workspace_bytes_prefill_heads(shape, 1, 1, 6)
        ws2 = torch.empty(max(n2, 16), dtype=torch.uint8, device="cuda")
        tp.tpla_prefill_heads(shape, q, k_pool, v_pool, t.contiguous(), 6, lens - 1, cu, 1, 1, ws2, n2, o2, CODE["f32"], None)
        out.append((o, o2))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and torch.isfinite(out[0][0]).all()
