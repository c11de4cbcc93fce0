"""Host side of the speculative step's entry points: refusals before any launch, the workspace, the rotary frequencies."""
import math

import numpy as np
import pytest

import paper_2508_15881_amd as tp

A = 4096   # a 16-byte aligned fake address: validation must fail before it is ever used
BIG = 1 << 40


def shape(**kw):
    base = dict(B=2, H=64, d_c=512, g=2, d_r=64, d_n=128, d_v=128, page_tokens=64, dtype=tp.TPLA_BF16, sm_scale=0.07)
    base.update(kw)
    return tp.TplaShape(**base)


def code(fn, *args):
    with pytest.raises(tp.TplaError) as e:
        fn(*args)
    assert tp.tpla_last_error() != ""
    return e.value.code


def swapped(good, **kw):
    return [kw.get("a%d" % i, v) for i, v in enumerate(good)]


def test_tree_refusals():
    s = shape()
    good = [s, 4, A, A, [A, A], A, 8, A, A, A, A, BIG, A, A]
    fn = tp.tpla_decode_shards_tree
    for i in (2, 3, 5, 7, 9, 10, 12):
        assert code(fn, *swapped(good, **{"a%d" % i: None})) == -1, i
    for i in (2, 3, 5, 7, 8, 9, 10, 12, 13):
        assert code(fn, *swapped(good, **{"a%d" % i: A + 4})) == -3, i
    assert code(fn, *swapped(good, a4=[A, None])) == -1 and code(fn, *swapped(good, a4=[A, A + 2])) == -3
    assert code(fn, *swapped(good, a4=None)) == -1
    assert code(fn, *swapped(good, a1=0)) == -2 and code(fn, *swapped(good, a1=65)) == -2
    assert code(fn, *swapped(good, a6=0)) == -2 and code(fn, *swapped(good, a6=2 ** 31 - 1)) == -2
    assert code(fn, *swapped(good, a11=16)) == -4
    assert code(fn, *swapped(good, a0=shape(dtype=3))) == -5 and code(fn, *swapped(good, a0=shape(g=3))) == -2
    assert code(fn, *swapped(good, a0=shape(B=40000))) == -7                              # g * B above 65535
    assert code(fn, *swapped(good, a0=shape(B=30000, H=2000), a1=64)) == -7
    assert code(fn, *swapped(good, a0=shape(d_c=2064, g=1, dtype=tp.TPLA_F32), a4=[A])) == -7
    one = [s, 4, A, A, A, A, 8, A, A, A, A, BIG, A, A]
    assert code(tp.tpla_decode_shard_tree, *swapped(one, a4=None)) == -1
    assert code(tp.tpla_decode_shard_tree, *swapped(one, a11=16)) == -4
    both = [s, 4, A, A, [A, A], A, 8, A, A, A, A, BIG, A, A, tp.TPLA_BF16, A, A]
    fn = tp.tpla_decode_shards_tree_combine
    assert code(fn, *swapped(both, a12=None)) == -1 and code(fn, *swapped(both, a13=None)) == -1
    assert code(fn, *swapped(both, a12=A + 8)) == -3 and code(fn, *swapped(both, a14=7)) == -5
    assert code(fn, *swapped(both, a15=None)) == -1 and code(fn, *swapped(both, a11=16)) == -4


def test_tree_workspace():
    s = shape()
    n = tp.tpla_workspace_bytes_tree(s, 4, 512)
    assert n > 0 and tp.tpla_workspace_bytes_tree(s, 4, 512) == n
    assert tp.tpla_workspace_bytes_tree(s, 0, 512) == 0 and tp.tpla_workspace_bytes_tree(s, 4, 0) == 0
    assert tp.tpla_workspace_bytes_tree(shape(H=0), 4, 512) == 0
    assert tp.tpla_workspace_bytes_tree(shape(d_c=64, H=2, d_r=16, dtype=tp.TPLA_F32), 1, 1) >= 16


def test_extend_refusals():
    s = shape()
    good = [s, A, A, 3, A, A, 9, A, A, A, 8, A, A, A, 6, A]
    fn = tp.tpla_extend_sequences
    for i in (1, 2, 5, 7, 8, 9, 11, 12, 13, 15):
        assert code(fn, *swapped(good, **{"a%d" % i: None})) == -1, i
    for i in (1, 2, 4, 5, 7, 8, 9, 11, 12, 13, 15):
        assert code(fn, *swapped(good, **{"a%d" % i: A + 4})) == -3, i
    assert code(fn, *swapped(good, a3=-1)) == -2 and code(fn, *swapped(good, a6=-1)) == -2 and code(fn, *swapped(good, a10=0)) == -2
    assert code(fn, *swapped(good, a14=7)) == -2                # not B rows of 3
    assert code(fn, *swapped(good, a3=0)) == -2                 # depths without rows
    assert code(fn, *swapped(good, a3=0, a4=None, a14=-1)) == -2 and code(fn, *swapped(good, a3=0, a4=None, a14=1 << 31)) == -2


def test_commit_refusals():
    s = shape()
    good = [s, 4, A, A, A, A, 8, [A, A], A]
    fn = tp.tpla_commit_drafts
    for i in (2, 3, 4, 5, 7, 8):
        assert code(fn, *swapped(good, **{"a%d" % i: None})) == -1, i
    for i in (2, 3, 4, 5, 8):
        assert code(fn, *swapped(good, **{"a%d" % i: A + 4})) == -3, i
    assert code(fn, *swapped(good, a7=[A, None])) == -1 and code(fn, *swapped(good, a7=[A + 2, A])) == -3
    assert code(fn, *swapped(good, a1=0)) == -2 and code(fn, *swapped(good, a1=65)) == -2 and code(fn, *swapped(good, a6=0)) == -2


def test_rotary_refusals():
    """The C call itself: strides and addresses as numbers."""
    import ctypes
    lib = tp.load_library()
    s = shape(H=4)

    def rc(sh=s, layout=0, rot=64, freq=A, amp=1.0, pos=A, T=5, q=A, qs=(256, 64), qo=A, qos=(256, 64), k=A, ks=64, ko=A, kos=64):
        return lib.tpla_apply_rotary(ctypes.byref(sh), layout, 0, rot, freq, amp, pos, T, q, *qs, qo, *qos, k, ks, ko, kos, None)

    assert rc(freq=None) == -1 and rc(pos=None) == -1 and rc(q=None) == -1 and rc(ko=None) == -1
    assert rc(q=None, qo=None, k=None, ko=None) == -1
    assert rc(layout=2) == -2 and rc(rot=63) == -2 and rc(rot=0) == -2 and rc(rot=66) == -2 and rc(T=-1) == -2 and rc(T=1 << 31) == -2
    assert rc(amp=math.inf) == -2 and rc(amp=math.nan) == -2
    assert rc(qs=(257, 64)) == -3 and rc(qs=(256, 60)) == -3 and rc(kos=68) == -3 and rc(qs=(-256, 64)) == -2
    assert rc(qos=(56, 64)) == -2 and rc(qos=(256, 56)) == -2 and rc(kos=56) == -2        # rows written twice
    assert rc(qos=(512, 64)) == -2 and rc(ks=128) == -2                                   # in place with other strides
    assert rc(q=A + 2, qo=A + 2) == -3 and rc(freq=A + 8) == -3
    assert rc(T=0) == 0
    with pytest.raises(ValueError):
        import torch
        x = torch.zeros((5, 4, 64), dtype=torch.bfloat16)
        tp.tpla_apply_rotary(s, 0, 0, 64, A, 1.0, A, 5, x.transpose(1, 2), x, None, None)


def test_rotary_frequencies():
    f = tp.tpla_rotary_frequencies(64)
    want = np.array([10000.0 ** (-2 * j / 64) for j in range(32)])
    assert np.max(np.abs(f / want - 1)) <= 4 * 2.0 ** -52
    assert np.allclose(tp.tpla_rotary_frequencies(64, factor=8.0), want / 8, rtol=1e-15, atol=0)
    g = tp.tpla_rotary_frequencies(64, base=10000.0, factor=40.0, original_positions=4096, beta_fast=32.0, beta_slow=1.0)
    turns = 4096 * want / (2 * math.pi)
    assert np.allclose(g[turns > 40], want[turns > 40], rtol=1e-15) and np.allclose(g[turns < 0.8], want[turns < 0.8] / 40, rtol=1e-14)
    # pair numbers at which a pair turns 32 times and once: 10.25 and 22.51 -> the ramp goes from pair 10 to pair 23
    ramp = np.clip((np.arange(32) - 10) / 13.0, 0, 1)
    assert np.allclose(g, want * (1 - ramp) + want / 40 * ramp, rtol=1e-14)
    assert (np.diff(g) < 0).all()
    for bad in (dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=64, base=1.0), dict(rot_dim=64, factor=0.5), dict(rot_dim=64, factor=math.inf),
                dict(rot_dim=64, original_positions=-1), dict(rot_dim=64, original_positions=10, beta_slow=0.0),
                dict(rot_dim=64, original_positions=10, beta_fast=0.5)):
        with pytest.raises(tp.TplaError) as e:
            tp.tpla_rotary_frequencies(**bad)
        assert e.value.code == -2


def test_tree_masks():
    from paper_2508_15881_amd import pipeline as pl
    masks, depths = pl.tree_masks([-1, 0, 0, 1, -1])
    assert masks.tolist() == [1, 3, 5, 11, 16] and depths.tolist() == [0, 1, 1, 2, 0]
    masks, depths = pl.tree_masks(np.stack([np.arange(-1, 63), np.full(64, -1)]))
    assert masks[0, 63] == 2 ** 64 - 1 and masks[1, 63] == 2 ** 63 and depths[0].tolist() == list(range(64)) and not depths[1].any()
    for bad in ([0], [-1, 1], [-1, -2]):
        with pytest.raises(ValueError):
            pl.tree_masks(bad)


def test_rotary_of_no_tokens_does_nothing():
    """Empty tensors have no address: that is not a missing pointer."""
    import torch
    s = shape()
    freq, pos = torch.zeros(s.d_r // 2, dtype=torch.float64), torch.zeros(0, dtype=torch.int32)
    st = torch.bfloat16 if s.dtype == tp.TPLA_BF16 else torch.float32
    q, k = torch.zeros((0, s.H, s.d_r), dtype=st), torch.zeros((0, s.d_r), dtype=st)
    assert q.data_ptr() == 0 and pos.data_ptr() == 0
    tp.tpla_apply_rotary(s, tp.TPLA_ROTARY_HALF, 0, s.d_r, freq, 1.0, pos, 0, q, q.clone(), k, k.clone(), stream=0)
    tp.tpla_apply_rotary(s, tp.TPLA_ROTARY_HALF, 0, s.d_r, freq, 1.0, pos, 0, None, None, k, k, stream=0)
    with pytest.raises(tp.TplaError):
        tp.tpla_apply_rotary(s, 7, 0, s.d_r, freq, 1.0, pos, 0, q, q, None, None, stream=0)
