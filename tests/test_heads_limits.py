"""Refusals of the grouped-head calls: nothing is launched, every check names its error (CPU)."""
import ctypes

import pytest
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import binding, pipeline as pl

A, F, H, K = 4096, tp.TPLA_F32, tp.TPLA_ROTARY_HALF, 1 << 40


def shape(**kw):
    base = dict(B=2, H=8, H_kv=2, d_k=128, d_v=128, page_tokens=64, dtype=tp.TPLA_BF16, sm_scale=0.09)
    base.update(kw)
    return tp.TplaHeads(*[base[n] for n, _ in tp.TplaHeads._fields_])


def code(name, s, *args):
    c = getattr(binding.load_library(), name)(ctypes.byref(s) if s else None, *args)
    if c < 0:
        assert tp.tpla_last_error() != ""
    return c


def norm(s=None, layout=H, rot=128, freq=A, amp=1.0, wq=A, wk=A, eps=1e-6, pos=A, T=4, q=(A, 1024, 128), qo=(A, 1024, 128), k=(A, 256, 128), ko=(A, 256, 128)):
    return code("tpla_norm_rotary_heads", s or shape(), layout, rot, freq, amp, wq, wk, eps, pos, T, *q, *qo, *k, *ko, None)


def append(s=None, rot=128, freq=A, eps=1e-6, wk=A, pos=A, T=4, q=(A, 1024, 128), qo=(A, 1024, 128), k=(A, 256, 128), v=(A, 256, 128), slots=A, kp=A, vp=A):
    return code("tpla_append_heads", s or shape(), H, rot, freq, 1.0, A if eps >= 0 else None, wk, eps, pos, T, *q, *qo, *k, *v, slots, kp, vp, None)


def decode(s=None, q=A, kp=A, vp=A, table=A, pages=4, lens=A, ws=A, n=K, o=A, o_dtype=F, lse=A):
    return code("tpla_decode_heads", s or shape(), q, kp, vp, table, pages, lens, ws, n, o, o_dtype, lse, None)


def prefill(s=None, q=A, kp=A, vp=A, table=A, pages=4, lens=A, cu=A, T=9, most=9, ws=A, n=K, o=A, o_dtype=F, lse=A):
    return code("tpla_prefill_heads", s or shape(), q, kp, vp, table, pages, lens, cu, T, most, ws, n, o, o_dtype, lse, None)


BAD_SHAPES = [(dict(dtype=7), -5), (dict(B=0), -2), (dict(H=9), -2), (dict(H_kv=0), -2), (dict(d_k=100), -2), (dict(d_v=60), -2), (dict(page_tokens=0), -2),
              (dict(sm_scale=0.0), -2), (dict(sm_scale=float("nan")), -2), (dict(d_k=264), -7), (dict(d_v=512), -7), (dict(H=1 << 17, H_kv=1 << 17), -7), (dict(H=1 << 15, H_kv=1 << 15, page_tokens=1 << 17), -7)]


@pytest.mark.parametrize("kw,want", BAD_SHAPES)
def test_shapes(kw, want):
    s = shape(**kw)
    assert norm(s) == want and append(s) == want and decode(s) == want and prefill(s) == want
    assert prefill(s, T=0, most=0) == want
    assert tp.tpla_workspace_bytes_heads(s, 4) == 0 and tp.tpla_workspace_bytes_prefill_heads(s, 9, 9, 4) == 0


def test_norm_rotary():
    assert code("tpla_norm_rotary_heads", None, H, 128, A, 1.0, A, A, 1e-6, A, 4, *4 * (A, 1024, 128), None) == -1
    assert norm(layout=2) == -2 and norm(rot=127) == -2 and norm(rot=130) == -2 and norm(rot=-2) == -2 and norm(T=-1) == -2 and norm(T=1 << 31) == -2
    assert norm(amp=float("inf")) == -2 and norm(eps=float("nan")) == -2 and norm(eps=-1.0) == -2 and norm(eps=-1.0, wq=None) == -2
    assert norm(freq=None) == -1 and norm(pos=None) == -1 and norm(q=(None, 0, 0)) == -1 and norm(ko=(None, 0, 0)) == -1
    assert norm(q=(None, 0, 0), qo=(None, 0, 0), k=(None, 0, 0), ko=(None, 0, 0)) == -1
    assert norm(freq=A + 8) == -3 and norm(pos=A + 4) == -3 and norm(wk=A + 2) == -3
    assert norm(q=(A + 2, 1024, 128)) == -3 and norm(k=(A, 250, 128)) == -3 and norm(qo=(A, 1024, 132)) == -3
    assert norm(q=(A, -8, 128)) == -2 and norm(qo=(A, 1024, 120)) == -2 and norm(ko=(A, 120, 128)) == -2
    assert norm(q=(2 * A, 1032, 128), qo=(2 * A, 1024, 128)) == -2 and norm(k=(2 * A, 512, 256), ko=(2 * A, 256, 128)) == -2       # in place
    assert norm(T=0, freq=None, pos=None, q=(None, 0, 0), qo=(None, 0, 0)) == 0


def test_append():
    for kw in (dict(q=(None, 0, 0)), dict(qo=(None, 0, 0)), dict(k=(None, 0, 0)), dict(v=(None, 0, 0)), dict(slots=None), dict(kp=None), dict(vp=None)):
        assert append(**kw) == -1, kw
    assert append(slots=A + 4) == -3 and append(kp=A + 2) == -3 and append(vp=A + 8) == -3 and append(v=(A, 251, 128)) == -3 and append(k=(A + 2, 256, 128)) == -3
    assert append(v=(A, -256, 128)) == -2 and append(eps=-1.0) == -2 and append(rot=3) == -2 and append(qo=(A, 8, 128)) == -2
    assert append(T=0, slots=None) == 0


def test_decode():
    for kw in (dict(q=None), dict(kp=None), dict(vp=None), dict(table=None), dict(lens=None), dict(o=None)):
        assert decode(**kw) == -1, kw
    big = shape(B=1, H=8, H_kv=8)
    assert tp.tpla_workspace_bytes_heads(big, 1024) > 16
    assert decode(big, ws=None, pages=1024) == -1 and decode(big, n=16, pages=1024) == -4
    for kw in (dict(q=A + 2), dict(kp=A + 8), dict(vp=A + 8), dict(table=A + 4), dict(lens=A + 4), dict(ws=A + 8), dict(o=A + 4), dict(lse=A + 4)):
        assert decode(**kw) == -3, kw
    assert decode(pages=0) == -2 and decode(o_dtype=2) == -5 and decode(pages=1 << 25) == -7 and decode(shape(B=1 << 24, H=16)) == -7


def test_prefill():
    for kw in (dict(q=None), dict(kp=None), dict(vp=None), dict(table=None), dict(cu=None), dict(o=None)):
        assert prefill(**kw) == -1, kw
    for kw in (dict(q=A + 2), dict(kp=A + 8), dict(vp=A + 8), dict(table=A + 4), dict(lens=A + 4), dict(cu=A + 4), dict(ws=A + 8), dict(o=A + 4), dict(lse=A + 4)):
        assert prefill(**kw) == -3, kw
    assert prefill(T=-1) == -2 and prefill(most=0) == -2 and prefill(most=-1) == -2 and prefill(pages=0) == -2 and prefill(pages=0, T=0) == -2
    assert prefill(o_dtype=9) == -5 and prefill(T=1 << 25, most=5) == -7 and prefill(pages=1 << 25) == -7 and prefill(T=1 << 40, most=5) == -7
    need = tp.tpla_workspace_bytes_prefill_heads(shape(), 9, 9, 1024)
    assert need > 0 and prefill(pages=1024, n=1024) == -4 and prefill(pages=1024, ws=None, n=need) == -1
    for s in (shape(), shape(H_kv=8), shape(dtype=F), shape(B=1, H=1, H_kv=1, d_k=64, d_v=64), shape(d_v=64)):         # room for fewer tokens too
        sizes = [tp.tpla_workspace_bytes_prefill_heads(s, t, min(t, 100), 1024) for t in (1, 5, 9, 64, 200, 1000, 4000, 20000)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    assert tp.tpla_workspace_bytes_prefill_heads(shape(), 9, 50, 1024) == need              # no more new tokens than there are rows
    assert tp.tpla_workspace_bytes_prefill_heads(shape(), 0, 9, 4) == 0 and tp.tpla_workspace_bytes_prefill_heads(shape(), 9, 0, 4) == 0
    assert prefill(T=0, most=0, q=None, cu=None, o=None) == 0


def test_binding_checks_views():
    s = shape()
    q = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        tp.tpla_norm_rotary_heads(s, H, 128, A, 1.0, None, None, 1e-6, A, 4, q.transpose(1, 2), q, None, None)
    with pytest.raises(ValueError):
        tp.tpla_norm_rotary_heads(s, H, 128, A, 1.0, None, None, 1e-6, A, 5, q, q, None, None)


def test_step_refuses_tokens_that_it_has_no_rows_for():
    step = pl.HeadsStep(shape(B=3), 4, [1.0] * 64, max_tokens=5, device="cpu")
    rows = lambda T, h: torch.zeros((T, h, 128), dtype=torch.bfloat16)  # noqa: E731
    pool = torch.zeros((12, 2, 64, 128), dtype=torch.bfloat16)
    table, lens = torch.zeros((3, 4), dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    for T, decode in ((6, False), (2, True), (4, True)):
        with pytest.raises(ValueError, match="new tokens"):
            step.run(rows(T, 8), rows(T, 2), rows(T, 2), None, None, pool, pool, table, lens, decode=decode)
