"""What the prefill of grouped heads writes, with guards around its buffers; and the general kernel's arithmetic, which is float for bf16 too."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp
from heads_common import Cached, check, run_decode, run_prefill

pytestmark = pytest.mark.gpu
GUARD = 4096


class Guarded:
    """A buffer of n elements in the middle of one whose borders are known."""

    def __init__(self, shape, dtype, fill, border):
        n = int(np.prod(shape))
        self.all = torch.full((n + 2 * GUARD,), border, dtype=dtype, device="cuda")
        self.x = self.all[GUARD:GUARD + n].view(shape)
        self.x.fill_(fill)
        self.border = border

    def intact(self):
        return bool((self.all[:GUARD] == self.border).all() and (self.all[-GUARD:] == self.border).all())


@pytest.mark.parametrize("H,H_kv,d,page,dtype,width", [(8, 2, 128, 64, "bf16", 2), (8, 2, 128, 64, "bf16", 40), (4, 4, 64, 16, "bf16", 200), (6, 2, 96, 16, "bf16", 200),
                                                       (4, 2, 128, 64, "f32", 40)])
@pytest.mark.parametrize("cu,max_new", [([-7, 60, 1000], 100), ([70, 20, 90], 100), ([0, 50, 80], 100), ([0, 50, 80], 30), ([0, 0, 100], 5), ([0, 3, 6], 3)])
def test_row_ranges_are_clipped(H, H_kv, d, page, dtype, width, cu, max_new):
    T, lens = 100, [30, 500] if width > 2 else [0, 0]
    c = Cached([lens[0] + 100, lens[1] + 100], H, H_kv, d, page=page, dtype=dtype, max_pages=width)
    c.queries(T)
    x = c.on()
    st = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    n = tp.tpla_workspace_bytes_prefill_heads(c.shape, T, max_new, c.max_pages)
    o, lse, ws = Guarded((T, H, d), st, float("nan"), 5.0), Guarded((T, H), torch.float32, float("nan"), 5.0), Guarded((max(n, 16),), torch.uint8, 0xFF, 0x5A)
    tp.tpla_prefill_heads(c.shape, x["q"], x["k_pool"], x["v_pool"], x["table"], c.max_pages, x["ints"](lens), x["ints"](cu), T, max_new, ws.x if n else None, n, o.x,
                          c.shape.dtype, lse.x)
    torch.cuda.synchronize()
    assert o.intact() and lse.intact() and ws.intact()
    got, got_lse = o.x.double().cpu().numpy(), lse.x.double().cpu().numpy()
    mine = np.zeros(T, dtype=bool)
    for b in range(2):
        first = min(max(cu[b], 0), T)
        k = min(min(max(cu[b + 1], first), T) - first, max_new)
        mine[first:first + k] = True
        for i in range(k):
            check(dtype, dtype, d, got[first + i], got_lse[first + i], *c.want(b, first + i, lens[b] + i + 1), "row %d" % (first + i))
    assert np.isnan(got[~mine]).all() and np.isnan(got_lse[~mine]).all()


@pytest.mark.parametrize("H,H_kv,d_k,d_v,page", [(6, 2, 96, 96, 16), (4, 2, 128, 64, 64), (4, 2, 128, 128, 24), (3, 1, 256, 256, 64), (40, 1, 80, 80, 16), (2, 2, 192, 128, 64)])
def test_other_widths_of_bf16_keep_their_weights_in_float(H, H_kv, d_k, d_v, page):
    """The tolerance of float arithmetic alone (see check): a rounding of the weights to bf16 would be seen, most of all where few tokens are."""
    lens = [0, 1, 2, 3, 5, 17, 64, 65, 300, 1500]
    c = Cached(lens, H, H_kv, d_k, d_v, page, "bf16")
    c.queries(len(lens))
    o, lse = run_decode(c, lens, "f32")
    for b, n in enumerate(lens):
        check("f32", "f32", d_k, o[b], lse[b], *c.want(b, b, n), "%d tokens" % n)
    news, before = [70, 2, 33], [0, 1, 600]
    c = Cached([a + b for a, b in zip(news, before)], H, H_kv, d_k, d_v, page, "bf16")
    c.queries(sum(news))
    o, lse = run_prefill(c, news, before, "f32")
    first = 0
    for b, n in enumerate(news):
        for i in range(n):
            check("f32", "f32", d_k, o[first + i], lse[first + i], *c.want(b, first + i, before[b] + i + 1), "sequence %d, new token %d" % (b, i))
        first += n
