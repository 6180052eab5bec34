"""A schedule played on the step's operators: the attention side of the serving run that
``fsched_simulate`` priced.

``simulate(..., schedule=True)`` says at which step each request starts and finishes; in
between it holds a row of the block table and brings one token per step (the chunked
reading: prompt tokens and output tokens alike).  ``Worker`` keeps what a serving process
keeps between steps (the paged cache of every layer, the block table, the free pages, the
lengths) and runs a step: ``kv_layout`` once, then ``qk_norm_rope`` and ``attend`` per
layer.  ``play`` drives it through a schedule.

A worker whose memory is the limit holds its cache in 4 bits (``kv_bits=4``), or keeps each
request within a budget of tokens: the attention weight of held tokens is added up over
steps and layers, and pages of least weight are given back (``budget``).
"""
from __future__ import annotations

from typing import Callable, Sequence

import torch

import paper_2608_02244_amd as fs


class Worker:
    """A paged KV cache of ``layers`` layers and the requests that hold parts of it.

    Lengths are known on the host (they follow from the schedule), so which pages are free
    is too; the page ids themselves stay on the GPU.

    ``kv_bits`` 4: the cache holds 4 bits an element (pages of 16 tokens and more).
    ``budget``: tokens that a request may keep behind a step.  One that holds more gives up
    whole pages, those of least attention weight first, but for its first ``n_sink`` and
    last ``n_recent`` tokens (``kv_evict``); what it keeps stays at its positions, and a
    window counts kept tokens."""

    def __init__(self, *, n_pages: int, page_size: int, q_heads: int, kv_heads: int,
                 head_dim: int, max_len: int, layers: int = 1, rope_base: float = 10000.0,
                 window: int = 0, n_sink: int = 0, dtype=torch.bfloat16, device="cuda",
                 kv_bits: int = 16, budget=None, n_recent: int = 0):
        if kv_bits not in (4, 16):
            raise ValueError("a cache holds 4 or 16 bits an element")
        if budget is not None and budget < 1:
            raise ValueError("a budget is at least one token")
        self.page_size, self.q_heads, self.window, self.n_sink = (page_size, q_heads, window,
                                                                  n_sink)
        self.max_len = max_len  # rows of the rotation table; the block table's are whole pages
        self.width = -(-max_len // page_size)
        self.kv_bits, self.budget, self.n_recent = kv_bits, budget, n_recent
        if kv_bits == 4:  # one tensor for keys and values
            self.caches = [(fs.kv4_cache(n_pages, kv_heads, page_size, head_dim,
                                         device=device).zero_(),) for _ in range(layers)]
        else:
            self.caches = [tuple(torch.zeros(n_pages, kv_heads, page_size, head_dim, dtype=dtype,
                                             device=device) for _ in range(2))
                           for _ in range(layers)]
        half = head_dim // 2
        angle = torch.arange(max_len, device=device, dtype=torch.float64)[:, None] * \
            rope_base ** (-torch.arange(half, device=device, dtype=torch.float64) / half)
        self.cos_sin = torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()
        self.weight = torch.ones(head_dim, dtype=dtype, device=device)
        self.free = torch.arange(n_pages, dtype=torch.int32, device=device)
        self.requests: list = []                      # ids, one per row of the table
        self.held: dict = {}                          # tokens of each
        self.gone: dict = {}                          # tokens of each given up
        self.table = torch.empty(0, self.width, dtype=torch.int32, device=device)
        # attention weight of held tokens, one row per row of the table
        self.attention = None if budget is None else \
            torch.empty(0, self.width * page_size, dtype=torch.float32, device=device)

    def _pages(self, tokens: int) -> int:
        return -(-tokens // self.page_size)

    def release(self, ids) -> None:
        """Finished requests give their pages back."""
        gone = set(ids)
        if not gone <= self.held.keys():
            raise ValueError(f"not among the requests: {sorted(gone - self.held.keys())}")
        if not gone:
            return
        back = [self.table[i, :self._pages(self.held[r])]
                for i, r in enumerate(self.requests) if r in gone]
        keep = [i for i, r in enumerate(self.requests) if r not in gone]
        self.free = torch.cat([self.free] + back)
        rows = torch.tensor(keep, dtype=torch.long, device=self.table.device)
        self.table = self.table[rows]
        if self.attention is not None:
            self.attention = self.attention[rows]
        self.requests = [self.requests[i] for i in keep]
        for r in gone:
            del self.held[r], self.gone[r]

    def admit(self, ids) -> None:
        """Requests that hold nothing yet get a row."""
        ids = list(ids)
        if not ids:
            return
        if len({*self.requests, *ids}) < len(self.requests) + len(ids):
            raise ValueError("a request has one row only")
        fresh = self.table.new_full((len(ids), self.width), -1)
        self.table = torch.cat((self.table, fresh))
        if self.attention is not None:
            zeros = self.attention.new_zeros(len(ids), self.attention.shape[1])
            self.attention = torch.cat((self.attention, zeros))
        self.requests += ids
        self.held.update((r, 0) for r in ids)
        self.gone.update((r, 0) for r in ids)

    def position(self, r) -> int:
        """Where the next token of request ``r`` sits."""
        return self.held[r] + self.gone[r]

    def _given_up(self, held: int) -> int:
        """Pages that a request of so many tokens gives up, as ``kv_evict`` counts them."""
        over = self._pages(max(0, held - self.budget))
        first = min(self._pages(self.n_sink), self._pages(held))
        last = max(0, held - self.n_recent) // self.page_size
        return min(over, max(0, last - first))

    def step(self, new: Sequence[int], qkv: Callable):
        """One step: ``new[i]`` tokens of request ``self.requests[i]``.  ``qkv(layer)`` gives
        the fused projection [sum(new), q_heads + 2 kv_heads, head_dim] of a layer.  Returns
        every layer's attention output."""
        old = [self.held[r] for r in self.requests]
        gone = [self.gone[r] for r in self.requests]
        if any(o + g + n > self.max_len for o, g, n in zip(old, gone, new)):
            raise ValueError("a request outgrows max_len")
        need = sum(self._pages(o + n) - self._pages(o) for o, n in zip(old, new))
        if need > len(self.free):
            raise RuntimeError(f"the step needs {need} pages, {len(self.free)} are free")
        dev = self.table.device
        lengths = torch.tensor([old, list(new)], dtype=torch.int32, device=dev)
        slots, pos, q_start, kv_len, _ = fs.kv_layout(
            lengths[0], lengths[1], self.table, self.free, page_size=self.page_size,
            n_tok=sum(new))
        if any(gone):  # a token's position counts those before it that were given up
            pos = pos + torch.tensor([g for g, n in zip(gone, new) for _ in range(n)],
                                     dtype=torch.int32, device=dev)
        four = self.kv_bits == 4
        store, attend = (fs.qk_norm_rope4, fs.attend4) if four else (fs.qk_norm_rope, fs.attend)
        kw = dict(window=self.window, n_sink=self.n_sink, max_q=max([1, *new]))
        weight = None if self.attention is None else self.attention.clone()
        out = []
        for layer, cache in enumerate(self.caches):
            q = store(qkv(layer), pos, slots, self.cos_sin, *cache, self.weight, self.weight)
            if weight is None:
                out.append(attend(q, *cache, self.table, q_start, kv_len, **kw))
                continue
            y, lse = attend(q, *cache, self.table, q_start, kv_len, return_lse=True, **kw)
            (fs.attend4_weight if four else fs.attend_weight)(
                q, lse, cache[0], self.table, q_start, kv_len, weight, **kw)
            out.append(y)
        held = [o + n for o, n in zip(old, new)]
        table, freed, up = self.table, self.free[:0], [0] * len(held)
        if weight is not None:
            up = [self._given_up(m) for m in held]
            if any(up):
                table, weight, _, freed, _ = fs.kv_evict(
                    weight, kv_len, table, torch.full_like(kv_len, self.budget),
                    page_size=self.page_size, n_sink=self.n_sink, n_recent=self.n_recent,
                    n_freed=sum(up))
        # only now: a step that ends with an error (in ``qkv``, say) can be run again
        self.free = torch.cat((self.free[need:], freed))
        self.table, self.attention = table, weight
        for r, m, u in zip(self.requests, held, up):
            self.held[r] = m - u * self.page_size
            self.gone[r] += u * self.page_size
        return out


def play(worker: Worker, start, finish, qkv: Callable, on_step: Callable = None, *,
         lengths=None) -> int:
    """Runs a schedule of one instance (``start`` and ``finish`` as ``simulate`` returns
    them: a request's first step, and the step after its last) and returns the number of
    steps with tokens.

    ``qkv(layer, requests, positions)`` gives a step's projection (one token per request
    at its position); ``on_step(step, requests, outputs)`` sees what came out.
    ``lengths``: prompt + output tokens of every request.  With them a schedule in which
    some request runs another number of steps is refused: one made with ``prefill=True``,
    whose prompts take no steps of their own, is not what this plays."""
    start, finish = [int(x) for x in start], [int(x) for x in finish]
    if lengths is not None:
        lengths = [int(x) for x in lengths]
        if [f - s for s, f in zip(start, finish)] != lengths:
            raise ValueError("the schedule's requests do not run one step per token (was it "
                             "made with prefill=True?)")
    steps = 0
    for t in range(min(start, default=0), max(finish, default=0)):
        worker.release([r for r in worker.requests if finish[r] <= t])
        worker.admit([r for r in range(len(start)) if start[r] == t])
        if not worker.requests:
            continue
        now = list(worker.requests)
        at = [worker.position(r) for r in now]
        out = worker.step([1] * len(now), lambda layer: qkv(layer, now, at))
        steps += 1
        if on_step:
            on_step(t, now, out)
    worker.release(worker.requests)
    return steps
