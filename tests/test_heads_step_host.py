"""HeadsStep on the host: no row that a new token owns is left out by the bound of its prefill, counts that the host knows are held to the step's room (CPU:
the library's calls are recorded, not made)."""
import pytest
import torch

import paper_2508_15881_amd as tp
from paper_2508_15881_amd import pipeline as pl

H, H_KV, D, PAGE = 8, 2, 64, 16


@pytest.fixture
def calls(monkeypatch):
    made = {}
    for name in ("tpla_extend_sequences", "tpla_append_heads", "tpla_decode_heads", "tpla_prefill_heads"):
        monkeypatch.setattr(pl.B, name, lambda *a, _n=name: made.setdefault(_n, []).append(a))
    return made


def step(B=3, **kw):
    return pl.HeadsStep(tp.TplaHeads(B, H, H_KV, D, D, PAGE, tp.TPLA_BF16, 0.1), 40, [1.0] * (D // 2), device="cpu", **kw)


def place(s, add=None, **kw):
    B = s.shape.B
    ints = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    s.place(ints(B), ints(B) if add is None else torch.tensor(add, dtype=torch.int32), ints(8), 8, ints(B), ints((B, 40)), **kw)


def run(s, T, decode=False):
    rows = lambda h: torch.zeros((T, h, D), dtype=torch.bfloat16)  # noqa: E731
    pool = torch.zeros((8, H_KV, PAGE, D), dtype=torch.bfloat16)
    return s.run(rows(H), rows(H_KV), rows(H_KV), None, None, pool, pool, torch.zeros((s.shape.B, 40), dtype=torch.int32), torch.zeros(s.shape.B, dtype=torch.int32), decode=decode)


def bound(calls):
    """T, max_new and the room of the last prefill."""
    a = calls["tpla_prefill_heads"][-1]
    return a[8], a[9], a[11]


@pytest.mark.parametrize("kw", [dict(max_tokens=200), dict(max_tokens=200, max_new=8), dict(max_tokens=200, max_new=130)])
@pytest.mark.parametrize("T", [1, 8, 150, 200])
def test_one_sequence_may_have_all_new_tokens_that_nobody_counted(calls, kw, T):
    s = step(**kw)
    place(s)
    run(s, T)
    rows, most, room = bound(calls)
    assert rows == T and most >= T
    assert room >= tp.tpla_workspace_bytes_prefill_heads(s.shape, T, most, s.max_pages) and room <= s.workspace.numel()


def test_counts_of_the_host_are_the_bound(calls):
    s = step(max_tokens=200, max_new=130)
    place(s, [70, 130, 0], news=[70, 130, 0])
    run(s, 200)
    assert bound(calls)[:2] == (200, 130)
    place(s, [2, 0, 3], news=[2, 0, 3])
    run(s, 5)
    assert bound(calls)[:2] == (5, 3)
    for T in (4, 6, 200):
        with pytest.raises(ValueError, match="new tokens"):
            run(s, T)
    place(s)                                                  # counts of an earlier step are forgotten
    run(s, 6)
    assert bound(calls)[:2] == (6, 6)


@pytest.mark.parametrize("news", [[1, 2], [1, 2, 3, 4], [-1, 2, 3], [9, 0, 0], [8, 8, 8], []])
def test_counts_that_the_step_has_no_room_for(calls, news):
    s = step(max_tokens=20, max_new=8)
    with pytest.raises(ValueError, match="new tokens"):
        place(s, news=news)
    assert not calls


def test_decode_of_counted_tokens(calls):
    s = step(max_tokens=20)
    place(s, [1, 1, 1], news=[1, 1, 1])
    run(s, 3, decode=True)
    assert len(calls["tpla_decode_heads"]) == 1
    place(s, [2, 0, 1], news=[2, 0, 1])
    with pytest.raises(ValueError, match="new tokens"):
        run(s, 3, decode=True)
    assert len(calls["tpla_decode_heads"]) == 1 and len(calls["tpla_append_heads"]) == 1


def test_rows_that_no_token_owns_are_no_numbers_of_an_earlier_step(calls):
    s = step(max_tokens=20)
    s.o.fill_(3.0)
    s.lse.fill_(3.0)
    place(s)
    assert (s.o == 3.0).all() and (s.lse == 3.0).all()       # the last layer's output stays until the next one's
    assert torch.isnan(run(s, 20)).all() and torch.isnan(s.lse).all()          # (nothing was computed here)


@pytest.mark.parametrize("kw", [dict(max_tokens=0), dict(max_tokens=-3), dict(max_new=0), dict(max_new=-1), dict(max_tokens=9, max_new=0)])
def test_steps_without_room(kw):
    with pytest.raises(ValueError, match="room"):
        step(**kw)
