"""What a worker with a cache of 4 bits or a budget of tokens decides on the host, without a
GPU: its operators are plain stand-ins (places in a cache and pages by weight, no
arithmetic)."""
import random

import pytest
import torch

import paper_2608_02244_amd as fs
from paper_2608_02244_amd import replay


@pytest.fixture
def plain(monkeypatch):
    calls = []

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

    def store(qkv, pos, slots, cos_sin, *cache_and_weights):
        calls.append(("store", pos.tolist(), len(cache_and_weights)))
        return qkv[:, :2]

    def attend(q, *args, return_lse=False, **kw):
        return (q, torch.zeros(q.shape[:2])) if return_lse else q

    def attend_weight(q, lse, cache, table, q_start, kv_len, weight, **kw):
        calls.append(("weight", kv_len.tolist()))
        for r, m in enumerate(kv_len.tolist()):  # every token as much as its place says
            weight[r, :m] += torch.arange(m) % 7 + 1.0

    def kv_evict(weight, kv_len, table, budget, *, page_size, n_sink, n_recent, n_freed):
        width, rows, out, lens, freed = table.shape[1], [], torch.zeros_like(weight), [], []
        for r, m in enumerate(kv_len.tolist()):
            pages = -(-m // page_size)
            may = [c for c in range(-(-n_sink // page_size), pages)
                   if (c + 1) * page_size <= m - n_recent]
            drop = min(-(-max(0, m - int(budget[r])) // page_size), len(may))
            score = sorted((float(weight[r, c * page_size:(c + 1) * page_size].sum()), c)
                           for c in may)
            gone = sorted(c for _, c in score[:drop])
            stay = [c for c in range(pages) if c not in gone]
            freed += [int(table[r, c]) for c in gone]
            rows.append([int(table[r, c]) for c in stay] + [-1] * (width - len(stay)))
            lens.append(m - drop * page_size)
            for i, c in enumerate(stay):
                out[r, i * page_size:(i + 1) * page_size] = \
                    weight[r, c * page_size:(c + 1) * page_size]
        assert len(freed) == n_freed  # the host counts as the operator does
        calls.append(("evict", gone))
        return (torch.tensor(rows, dtype=torch.int32).view(-1, width), out,
                torch.tensor(lens, dtype=torch.int32), torch.tensor(freed, dtype=torch.int32),
                torch.tensor([len(freed)], dtype=torch.int32))
    for name, f in dict(kv_layout=kv_layout, qk_norm_rope=store, qk_norm_rope4=store,
                        attend=attend, attend4=attend, attend_weight=attend_weight,
                        attend4_weight=attend_weight, kv_evict=kv_evict).items():
        monkeypatch.setattr(fs, name, f, raising=False)
    return calls


def worker(**kw):
    v = dict(n_pages=40, page_size=4, q_heads=2, kv_heads=1, head_dim=64, max_len=200,
             device="cpu", budget=12)
    v.update(kw)
    return replay.Worker(**v)


def projection(tokens):
    return torch.zeros(tokens, 4, 64, dtype=torch.bfloat16)


def whole(w, n_pages):
    """Every page is free or held, once."""
    held = [int(x) for r, row in zip(w.requests, w.table)
            for x in row[:-(-w.held[r] // w.page_size)]]
    return sorted(w.free.tolist() + held) == list(range(n_pages))


def test_requests_keep_within_their_budget_and_lose_no_page(plain):
    rng = random.Random(2)
    w = worker(n_sink=4, n_recent=5, layers=2)
    brought = {}
    for step in range(60):
        if step % 7 == 0 and len(w.requests) < 4:
            w.admit([step])
            brought[step] = 0
        if step % 20 == 19:
            gone = w.requests[0]
            w.release([gone])
            del brought[gone]
        new = [rng.choice((0, 1, 1, 3)) for _ in w.requests]
        if sum(new) == 0:
            continue
        w.step(new, lambda layer: projection(sum(new)))
        for r, n in zip(w.requests, new):
            brought[r] += n
            assert w.held[r] + w.gone[r] == brought[r] == w.position(r)
            # never more than the budget, but for the last page and what has to stay
            assert w.held[r] <= max(12, -(-4 // 4) * 4 + 5 + 3)
        assert whole(w, 40) and w.attention.shape == (len(w.requests), w.width * 4)
    assert any(w.gone.values())


def test_positions_go_on_where_tokens_were_given_up(plain):
    w = worker(budget=4)
    w.admit([1, 2])
    w.step([9, 2], lambda layer: projection(11))
    assert w.gone == {1: 8, 2: 0} and w.held == {1: 1, 2: 2}
    plain.clear()
    w.step([2, 1], lambda layer: projection(3))
    assert plain[0] == ("store", [9, 10, 2], 4)
    assert w.position(1) == 11 and w.position(2) == 3


def test_a_step_that_fails_counts_no_weight_twice(plain):
    w = worker(layers=2)
    w.admit([0])
    w.step([5], lambda layer: projection(5))
    before = w.attention.clone(), w.free.clone(), dict(w.held)

    def broken(layer):
        if layer == 1:
            raise RuntimeError("no projection")
        return projection(2)
    with pytest.raises(RuntimeError):
        w.step([2], broken)
    assert torch.equal(w.attention, before[0]) and torch.equal(w.free, before[1])
    assert w.held == before[2]


def test_rows_of_weights_go_with_their_requests(plain):
    w = worker(budget=100)
    w.admit([3, 5, 9])
    w.step([2, 4, 6], lambda layer: projection(12))
    kept = w.attention[2].clone()
    w.release([3, 5])
    w.admit([4])
    assert torch.equal(w.attention[0], kept) and not w.attention[1].any()
    assert w.gone == {9: 0, 4: 0}


def test_positions_stay_within_max_len(plain):
    w = worker(max_len=12, budget=4)
    w.admit([0])
    w.step([10], lambda layer: projection(10))
    assert w.held[0] < 5
    with pytest.raises(ValueError, match="max_len"):
        w.step([3], lambda layer: projection(3))


def test_four_bits_take_the_other_operators_and_one_tensor(plain):
    w = worker(kv_bits=4, page_size=16, layers=2, budget=None)
    assert [tuple(x.shape for x in c) for c in w.caches] == [((40, 1, 1, 17 * 64),)] * 2
    w.admit([0])
    w.step([3], lambda layer: projection(3))
    assert plain == [("store", [0, 1, 2], 3)] * 2 and w.attention is None
    w = worker(kv_bits=4, page_size=16, budget=16)
    w.admit([0])
    w.step([40], lambda layer: projection(40))
    assert w.held[0] == 8 and w.gone[0] == 32


def test_refusals():
    for kw in (dict(kv_bits=8), dict(budget=0), dict(kv_bits=4, page_size=8)):
        with pytest.raises(ValueError):
            worker(**kw)


def test_a_schedule_plays_within_a_budget(plain):
    seen = []
    w = worker(budget=4)
    steps = replay.play(w, [0, 2], [30, 9], lambda layer, now, at: projection(len(now)),
                        lambda t, now, out: seen.append(list(now)), lengths=[30, 7])
    assert steps == 30 and sum(map(len, seen)) == 37
    assert not w.requests and sorted(w.free.tolist()) == list(range(40))


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_attention_weights_are_float32_under_any_default_type(plain, default):
    """attend_weight adds to 32-bit numbers only, whatever a program makes torch's default."""
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        w = worker(budget=4)
        w.admit([0, 1])
        w.step([9, 2], lambda layer: projection(11))
        w.release([1])
        w.admit([2])
        assert w.attention.dtype == torch.float32 and w.cos_sin.dtype == torch.float32
    finally:
        torch.set_default_dtype(before)
