"""tpla_apply_rotary against the definition in 64 bits, and its transpose against the gradient and against differences."""
import numpy as np
import pytest
import torch

import paper_2508_15881_amd as tp

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def shape(H, d_r, st):
    return tp.TplaShape(1, H, 64, 1, d_r, 32, 32, 64, tp.TPLA_F32 if st == torch.float32 else tp.TPLA_BF16, 0.1)


def rotate64(x, pos, freq, rot, layout, amplitude=1.0, inverse=False):
    """x [T, ..., d_r] float64."""
    a = pos.double()[:, None] * torch.as_tensor(freq)
    a = (-a if inverse else a).reshape((len(pos),) + (1,) * (x.dim() - 2) + (rot // 2,))
    i = torch.arange(0, rot, 2) if layout == tp.TPLA_ROTARY_INTERLEAVED else torch.arange(rot // 2)
    j = i + (1 if layout == tp.TPLA_ROTARY_INTERLEAVED else rot // 2)
    y = x.clone()
    y[..., i] = amplitude * (x[..., i] * a.cos() - x[..., j] * a.sin())
    y[..., j] = amplitude * (x[..., i] * a.sin() + x[..., j] * a.cos())
    size = x.abs().clone()
    size[..., i] = size[..., j] = abs(amplitude) * (x[..., i].abs() + x[..., j].abs())
    return y, size


def assert_close(got, want, size, st):
    # sine and cosine: 4 units of 2^-24 of the angle's own rounding (2 pi 2^-25) and the function; then amplitude, product
    # and sum: 3 half steps.  All relative to |x| + |y|.  One rounding of the result on the way out.
    tol = 8 * 2.0 ** -24 * size + (HALF[st] * want.abs() if st == torch.bfloat16 else 0.0)
    assert ((got.double().cpu() - want).abs() <= tol).all(), float(((got.double().cpu() - want).abs() / tol.clamp(min=1e-300)).max())


@pytest.mark.parametrize("T,H,d_r,rot,layout,st,far", [
    (1, 64, 64, 64, 0, torch.bfloat16, 10), (1, 64, 64, 64, 1, torch.bfloat16, 100000), (3, 5, 64, 62, 0, torch.bfloat16, 5000),
    (17, 3, 64, 32, 1, torch.bfloat16, 5000), (300, 7, 48, 36, 1, torch.bfloat16, 300), (1500, 16, 64, 64, 0, torch.bfloat16, 2 ** 31 - 1),
    (1300, 2, 128, 128, 1, torch.float32, 2 ** 31 - 1), (5, 1, 16, 2, 0, torch.float32, 1000000), (9, 4, 16, 10, 1, torch.float32, 1000000),
    (257, 128, 64, 64, 1, torch.float32, 131072), (2, 1, 8, 8, 1, torch.bfloat16, 50),
])
def test_against_the_definition(T, H, d_r, rot, layout, st, far):
    print("rotary", T, H, d_r, rot, layout, st, flush=True)
    g = torch.Generator().manual_seed(T + d_r)
    q, k = torch.randn((T, H, d_r), generator=g).to(st), torch.randn((T, d_r), generator=g).to(st)
    pos = torch.randint(0, far, (T,), generator=g).to(torch.int32)
    pos[0] = far - 1
    freq = tp.tpla_rotary_frequencies(rot)
    qd, kd = q.cuda(), k.cuda()
    qo, ko = torch.full_like(qd, float("nan")), torch.full_like(kd, float("nan"))
    tp.tpla_apply_rotary(shape(H, d_r, st), layout, 0, rot, torch.from_numpy(freq).cuda(), 1.25, pos.cuda(), T, qd, qo, kd, ko)
    torch.cuda.synchronize()
    for got, x in ((qo, q), (ko, k)):
        want, size = rotate64(x.double(), pos, freq, rot, layout, 1.25)
        assert_close(got, want, size, st)
        assert torch.equal(got.cpu()[..., rot:], x[..., rot:])
    assert torch.equal(qd.cpu(), q)
    # in place, each alone
    tp.tpla_apply_rotary(shape(H, d_r, st), layout, 0, rot, torch.from_numpy(freq).cuda(), 1.25, pos.cuda(), T, qd, qd, None, None)
    tp.tpla_apply_rotary(shape(H, d_r, st), layout, 0, rot, torch.from_numpy(freq).cuda(), 1.25, pos.cuda(), T, None, None, kd, kd)
    torch.cuda.synchronize()
    assert torch.equal(qd, qo) and torch.equal(kd, ko)


@pytest.mark.parametrize("layout", [0, 1])
def test_columns_of_a_projection_into_rows_of_another(layout):
    T, H, st = 37, 6, torch.bfloat16
    wide = torch.randn((T, H, 192)).to(st).cuda()
    kv = torch.randn((T, 576)).to(st).cuda()
    out = torch.zeros((T, H, 96), dtype=st, device="cuda")
    before = wide.clone()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 991
    freq = tp.tpla_rotary_frequencies(64, factor=32.0, original_positions=4096)
    tp.tpla_apply_rotary(shape(H, 64, st), layout, 0, 64, torch.from_numpy(freq).cuda(), 1.0, pos, T, wide[:, :, 128:], out[:, :, 16:80], kv[:, 512:], kv[:, 512:])
    torch.cuda.synchronize()
    want, size = rotate64(before[:, :, 128:].double().cpu(), pos.cpu(), freq, 64, layout)
    assert_close(out[:, :, 16:80], want, size, st)
    assert (out[:, :, :16] == 0).all() and (out[:, :, 80:] == 0).all() and torch.equal(wide, before)


@pytest.mark.parametrize("layout", [0, 1])
def test_inverse_is_the_gradient(layout):
    """<R x, w> has the gradient R^T w; and in 64 bits the central difference of a linear function is exact up to rounding."""
    T, H, d_r, rot, st = 6, 3, 32, 24, torch.float32
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn((T, H, d_r), generator=g), torch.randn((T, H, d_r), generator=g)
    pos = torch.randint(0, 100000, (T,), generator=g).to(torch.int32)
    freq = tp.tpla_rotary_frequencies(rot)
    got = torch.empty_like(x).cuda()
    tp.tpla_apply_rotary(shape(H, d_r, st), layout, 1, rot, torch.from_numpy(freq).cuda(), 0.75, pos.cuda(), T, w.cuda(), got, None, None)
    torch.cuda.synchronize()
    want, size = rotate64(w.double(), pos, freq, rot, layout, 0.75, inverse=True)
    assert_close(got, want, size, st)
    leaf = x.double().requires_grad_()
    a = pos.double()[:, None, None] * torch.as_tensor(freq)
    p, q = (leaf[..., 0:rot:2], leaf[..., 1:rot:2]) if layout == 0 else (leaf[..., :rot // 2], leaf[..., rot // 2:rot])
    wp, wq = (w[..., 0:rot:2], w[..., 1:rot:2]) if layout == 0 else (w[..., :rot // 2], w[..., rot // 2:rot])
    loss = 0.75 * ((p * a.cos() - q * a.sin()) * wp + (p * a.sin() + q * a.cos()) * wq).sum() + (leaf[..., rot:] * w[..., rot:]).sum()
    loss.backward()
    assert_close(got, leaf.grad, size, st)
    f = lambda z: float((rotate64(z, pos, freq, rot, layout, 0.75)[0] * torch.where(torch.arange(d_r) < rot, 1.0, 1.0) * w.double()).sum())  # noqa: E731
    for t, h, c in ((0, 0, 0), (2, 1, 5), (5, 2, 23), (3, 0, 30)):
        e = torch.zeros_like(x, dtype=torch.float64)
        e[t, h, c] = 0.5
        # the sums have 576 terms below 10: rounding below 576 * 10 * 2^-52
        assert abs(f(x.double() + e) - f(x.double() - e) - float(got[t, h, c])) <= 1e-11 + 8 * 2.0 ** -24 * float(size[t, h, c])


def test_captured_and_replayed_on_a_side_stream():
    T, H, st = 70, 8, torch.bfloat16
    x = torch.randn((T, H, 64), device="cuda").to(st)
    pos = torch.zeros(T, dtype=torch.int32, device="cuda")
    freq = tp.tpla_rotary_frequencies(64)
    f = torch.from_numpy(freq).cuda()
    y = torch.empty_like(x)
    call = lambda: tp.tpla_apply_rotary(shape(H, 64, st), 0, 0, 64, f, 1.0, pos, T, x, y, None, None)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(3):
        pos.copy_(torch.arange(T) * (k + 1) * 77)
        graph.replay()
        torch.cuda.synchronize()
        want, size = rotate64(x.double().cpu(), pos.cpu(), freq, 64, 0)
        assert_close(y, want, size, st)


@pytest.mark.parametrize("layout", [0, 1])
def test_widest_rows(layout):
    T, d_r, st = 1100, 8192, torch.bfloat16
    g = torch.Generator().manual_seed(layout)
    k = torch.randn((T, d_r), generator=g).to(st)
    pos = torch.randint(0, 100000, (T,), generator=g).to(torch.int32)
    freq = tp.tpla_rotary_frequencies(d_r)
    kd = k.cuda()
    tp.tpla_apply_rotary(shape(1, d_r, st), layout, 0, d_r, torch.from_numpy(freq).cuda(), 1.0, pos.cuda(), T, None, None, kd, kd)
    torch.cuda.synchronize()
    want, size = rotate64(k.double(), pos, freq, d_r, layout)
    assert_close(kd, want, size, st)


@pytest.mark.parametrize("T,H", [(1, 6), (5, 1), (1, 1)])
def test_strides_of_single_tokens_and_heads_mean_nothing(T, H):
    st = torch.bfloat16
    wide = torch.randn((T, H, 64)).to(st).cuda()
    q = torch.as_strided(wide, (T, H, 64), (3 if T == 1 else H * 64, 1 if H == 1 else 64, 1))
    k = torch.as_strided(torch.randn((T, 64)).to(st).cuda(), (T, 64), (7 if T == 1 else 64, 1))
    before, kb = q.clone(), k.clone()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") + 41
    freq = tp.tpla_rotary_frequencies(64)
    qo, ko = torch.empty((T, H, 64), dtype=st, device="cuda"), torch.empty((T, 64), dtype=st, device="cuda")
    call = lambda *t: tp.tpla_apply_rotary(shape(H, 64, st), 0, 0, 64, torch.from_numpy(freq).cuda(), 1.0, pos, T, *t)  # noqa: E731
    call(q, qo, k, ko)
    call(q, q, k, k)
    torch.cuda.synchronize()
    for got, x in ((qo, before), (ko, kb), (q, before), (k, kb)):
        want, size = rotate64(x.double().cpu(), pos.cpu(), freq, 64, 0)
        assert_close(got, want, size, st)


@pytest.mark.parametrize("T,H,d_r,rot,st", [
    (33, 5, 64, 62, torch.bfloat16), (1100, 3, 64, 60, torch.bfloat16), (700, 9, 16, 6, torch.bfloat16), (5, 2, 128, 124, torch.float32),
    (1031, 4, 64, 28, torch.float32), (50, 3, 24, 2, torch.float32), (50, 3, 24, 12, torch.float32), (7, 1, 1024, 1022, torch.bfloat16),
])
def test_halves_of_odd_and_even_numbers_of_columns(T, H, d_r, rot, st):
    g = torch.Generator().manual_seed(T + rot)
    wide = torch.randn((T, H, d_r + 8), generator=g).to(st)
    q, k = wide[:, :, 8:], torch.randn((T, d_r), generator=g).to(st)
    pos = torch.randint(0, 90000, (T,), generator=g).to(torch.int32)
    freq = tp.tpla_rotary_frequencies(rot)
    wd, kd = wide.cuda(), k.cuda()
    tp.tpla_apply_rotary(shape(H, d_r, st), tp.TPLA_ROTARY_HALF, 0, rot, torch.from_numpy(freq).cuda(), 0.5, pos.cuda(), T, wd[:, :, 8:], wd[:, :, 8:], kd, kd)
    torch.cuda.synchronize()
    for got, x in ((wd[:, :, 8:], q), (kd, k)):
        want, size = rotate64(x.double(), pos, freq, rot, tp.TPLA_ROTARY_HALF, 0.5)
        assert_close(got, want, size, st)
        assert torch.equal(got.cpu()[..., rot:], x[..., rot:])
    assert torch.equal(wd.cpu()[:, :, :8], wide[:, :, :8])
