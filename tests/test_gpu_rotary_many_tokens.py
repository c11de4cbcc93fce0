"""Rotary positions of more tokens than one launch has threads for: keys alone, and narrow heads."""
import pytest
import torch

import paper_2508_15881_amd as tp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H,d_r,queries", [(2 ** 25 + 3, 1, 8, False), (2 ** 26 + 1, 1, 8, False), (2 ** 23 + 1, 2, 16, True)])
def test_every_token_is_turned(T, H, d_r, queries):
    print("rotary of", T, "tokens", flush=True)
    s = tp.TplaShape(1, H, 64, 1, d_r, 16, 16, 64, tp.TPLA_BF16, 0.1)
    freq = tp.tpla_rotary_frequencies(d_r)
    f = torch.from_numpy(freq).cuda()
    period = 1000                                              # rows and positions repeat: a few rows to compare with, all of them compared
    pos = (torch.arange(T, dtype=torch.int32, device="cuda") % period)
    rows = torch.randn((period, d_r), device="cuda").to(torch.bfloat16)
    k = torch.empty((T, d_r), dtype=torch.bfloat16, device="cuda")      # (in parts: one indexing call over 2^29 elements gathered wrong rows)
    for t0 in range(0, T, period * 1000):
        n = min(T, t0 + period * 1000) - t0
        k[t0:t0 + n] = rows[torch.arange(t0, t0 + n, device="cuda") % period]
    k_out = torch.full((T, d_r), float("nan"), dtype=torch.bfloat16, device="cuda")
    q = k[:, None].expand(T, H, d_r).contiguous() if queries else None
    q_out = torch.full_like(q, float("nan")) if queries else None
    tp.tpla_apply_rotary(s, tp.TPLA_ROTARY_HALF, 0, d_r, f, 1.0, pos, T, q, q_out, k, k_out)
    torch.cuda.synchronize()
    want = torch.empty_like(rows)
    tp.tpla_apply_rotary(s, tp.TPLA_ROTARY_HALF, 0, d_r, f, 1.0, pos[:period], period, None, None, rows, want)
    a, half = torch.arange(period, device="cuda")[:, None] * f, d_r // 2
    x, y = rows[:, :half].double(), rows[:, half:].double()
    exact = torch.cat([x * a.cos() - y * a.sin(), x * a.sin() + y * a.cos()], 1)
    # angle, sine, products in float (2^-21 of the size), then half a step of bfloat16
    assert ((want.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 2.0 ** -20 * (x.abs() + y.abs()).repeat(1, 2)).all()
    want = want.view(torch.int16)
    for t0 in range(0, T, period * 1000):
        n = min(T, t0 + period * 1000) - t0
        idx = torch.arange(t0, t0 + n, device="cuda") % period
        assert torch.equal(k_out[t0:t0 + n].view(torch.int16), want[idx])
        if queries:
            assert torch.equal(q_out[t0:t0 + n].view(torch.int16), want[idx][:, None].expand(n, H, d_r))
