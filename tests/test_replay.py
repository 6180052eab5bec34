"""What ``replay`` decides on the host, without a GPU: a worker on the CPU whose operators
are plain stand-ins (places in a cache, no arithmetic)."""
import pytest
import torch

import paper_2608_02244_amd as fs
from paper_2608_02244_amd import replay


@pytest.fixture
def plain(monkeypatch):
    """kv_layout as the operator does it, one token after the other; the queries go
    through the other two unchanged."""
    def kv_layout(old, new, table, free, *, page_size, n_tok):
        slots, pos, start, taken = [], [], [0], 0
        for r, (o, m) in enumerate(zip(old.tolist(), new.tolist())):
            for c in range(-(-o // page_size), -(-(o + m) // page_size)):
                table[r, c] = free[taken]
                taken += 1
            for i in range(o, o + m):
                slots.append(int(table[r, i // page_size]) * page_size + i % page_size)
                pos.append(i)
            start.append(start[-1] + m)
        assert start[-1] == n_tok
        return tuple(torch.tensor(x, dtype=torch.int32)
                     for x in (slots, pos, start, (old + new).tolist(), [taken, n_tok]))

    def qk_norm_rope(qkv, *args, **kw):
        return qkv[:, :2]

    def attend(q, *args, **kw):
        return q
    for f in (kv_layout, qk_norm_rope, attend):
        monkeypatch.setattr(fs, f.__name__, f, raising=False)


def worker(**kw):
    v = dict(n_pages=8, page_size=4, q_heads=2, kv_heads=1, head_dim=64, max_len=10, device="cpu")
    v.update(kw)
    return replay.Worker(**v)


def projection(tokens):
    return torch.zeros(tokens, 4, 64, dtype=torch.bfloat16)


def pages(w):
    """Ids of the free pages and of those that the requests hold."""
    held = [int(x) for r, row in zip(w.requests, w.table)
            for x in row[:-(-w.held[r] // w.page_size)]]
    return sorted(w.free.tolist()), sorted(held)


def test_a_request_stays_within_max_len(plain):
    """10 tokens end inside the third page: the eleventh has a slot, but no row of the
    rotation table."""
    w = worker()
    w.admit([7])
    w.step([10], lambda layer: projection(10))
    before = pages(w), dict(w.held), w.table.clone()
    with pytest.raises(ValueError, match="max_len"):
        w.step([1], lambda layer: projection(1))
    assert (pages(w), w.held) == before[:2] and torch.equal(w.table, before[2])
    w = worker()
    w.admit([0])
    with pytest.raises(ValueError, match="max_len"):
        w.step([11], lambda layer: projection(11))


def test_a_step_that_fails_can_be_run_again(plain):
    """An error between the placement and the last layer loses no page."""
    w = worker(layers=2)
    w.admit([0, 1])
    w.step([3, 1], lambda layer: projection(4))

    def broken(layer):
        if layer == 1:
            raise RuntimeError("no projection")
        return projection(6)
    before = pages(w)
    with pytest.raises(RuntimeError, match="no projection"):
        w.step([2, 4], broken)
    assert pages(w) == before and w.held == {0: 3, 1: 1}
    w.step([2, 4], lambda layer: projection(6))
    free, held = pages(w)
    assert len(held) == 4 and sorted(free + held) == list(range(8))
    w.release([0, 1])
    assert pages(w) == (list(range(8)), [])


def test_release_and_admit_refuse_ids_before_they_change_anything(plain):
    w = worker()
    w.admit([3, 5])
    w.step([5, 2], lambda layer: projection(7))
    before = pages(w), list(w.requests), dict(w.held), w.table.clone()
    for call in (lambda: w.release([3, 4]), lambda: w.admit([6, 5]), lambda: w.admit([6, 6])):
        with pytest.raises(ValueError):
            call()
        assert (pages(w), w.requests, w.held) == before[:3] and torch.equal(w.table, before[3])
    w.release([5])
    w.admit([5])
    assert w.held == {3: 5, 5: 0} and w.requests == [3, 5]


def test_release_and_admit_of_nobody_leave_the_table_alone(plain):
    """No copy of the table and no index from the host at the steps (nearly all of a
    schedule's) at which no request starts or finishes."""
    w = worker()
    w.admit([0])
    w.step([5], lambda layer: projection(5))
    table, free = w.table, w.free
    w.release([])
    w.admit([])
    assert w.table is table and w.free is free


def test_play_refuses_a_schedule_whose_steps_are_not_the_tokens(plain):
    """Two requests of 3 + 2 and 1 + 4 tokens: prefilled they run 2 and 4 steps."""
    w, tokens = worker(), []
    with pytest.raises(ValueError, match="prefill"):
        replay.play(w, [0, 1], [2, 5], lambda layer, now, at: projection(len(now)),
                    lengths=[5, 5])
    assert not w.requests
    assert replay.play(w, [0, 1], [5, 6], lambda layer, now, at: projection(len(now)),
                       lambda t, now, out: tokens.append(len(out[0])), lengths=[5, 5]) == 6
    assert sum(tokens) == 10 and pages(w) == (list(range(8)), [])
