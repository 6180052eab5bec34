"""The model-side operators of a serving step whose speed is measured.

A schedule says which requests share a step and how many tokens of each the KV
cache holds.  These are the operators that the step itself runs on the worker:

  layout  the step's new tokens get their places in a paged KV cache: block tables
          extended from a list of free pages, slot maps, positions
  rope    queries and keys normed per head and rotated to their positions, keys and
          values put into their slots, in one pass over the fused projection
  attend  attention of the step's new tokens over the paged cache: one token per
          request (decode), a few (drafts), whole prompts, or a mix; optionally with
          a sliding window and a few first tokens that stay visible (sinks)
  shared  the same for a batch whose requests all begin with one long prefix, which
          is held and read once

A case is a dict of plain values:
  op        layout | rope | attend | shared
  shape     distribution of the request lengths (the named workloads' ones)
  n_req     requests in the batch (B); n_tok: tokens of a rope case
  mode      decode | draft | prefill | mixed: how many new tokens each request has
  Hq, Hkv, D, dtype, page  heads, head size, element type and tokens per page
  window, sinks, prefix    attention span (0: all), first visible tokens, prefix tokens

Request lengths are quantiles of the distribution, put in an order by the seed: the
work of a case does not depend on the seed.
"""
import math
import random
import statistics

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_DRAFT = 4      # most tokens of one request in a draft step
_CHUNK = 512    # most prompt tokens that one request brings into a mixed step
_EPS = 1e-6


def _case(name, op, shape="lognormal", n_req=0, n_tok=0, mode="decode", Hq=0, Hkv=0, D=0,
          dtype="bf16", page=16, window=0, sinks=0, prefix=0, interleaved=False, rot=0):
    c = dict(op=op, shape=shape, n_req=n_req, n_tok=n_tok, mode=mode, Hq=Hq, Hkv=Hkv, D=D,
             dtype=dtype, page=page, window=window, sinks=sinks, prefix=prefix,
             interleaved=interleaved, rot=rot)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of the throughput headline's batch (B = 512): one new token each
        _case("layout_decode", "layout", "pareto", 512),
        # admission of a large queue at once: every prompt gets all its pages and slots
        _case("layout_prefill", "layout", "pareto", 1024, mode="prefill"),
        # the projection of a decode step of 64 requests: launch-bound
        _case("rope_decode", "rope", n_tok=64, Hq=32, Hkv=8, D=128, rot=128),
        # prompts of a long admission, an odd number of tokens, half of each head rotated
        # in pairs of neighbours
        _case("rope_prefill", "rope", n_tok=32771, Hq=32, Hkv=8, D=128, dtype="f16", page=32,
              interleaved=True, rot=64),
        # the smallest batch of the benchmark: 8 requests of a few tokens
        _case("attend_decode_few", "attend", "uniform", 8, Hq=32, Hkv=8, D=128),
        # a decode step under the KV budget of 65,536 tokens
        _case("attend_decode", "attend", "lognormal", 64, Hq=32, Hkv=8, D=128),
        # a decode step of the headline's batch: heavy-tailed, about 0.7 M tokens held
        _case("attend_decode_heavy", "attend", "pareto", 512, Hq=32, Hkv=4, D=128, page=32),
        # window and sinks, one key head per query head, ragged bimodal lengths
        _case("attend_window", "attend", "bimodal", 128, Hq=16, Hkv=16, D=64, dtype="f16",
              window=1000, sinks=4),
        # whole prompts: the products of a long prefill
        _case("attend_prefill", "attend", "prompts", 5, mode="prefill", Hq=16, Hkv=4, D=128,
              page=64),
        # chunks of prompts beside decoding requests, with a window over long contexts
        _case("attend_mixed", "attend", "bimodal", 50, mode="mixed", Hq=40, Hkv=8, D=128,
              window=2048, sinks=16),
        # a batch behind one long instruction: a prefix of 8,192 tokens and short own parts
        _case("shared_decode", "shared", "short", 128, Hq=32, Hkv=8, D=128, prefix=8192),
        # a few requests with drafts behind a prefix that ends inside a page
        _case("shared_draft", "shared", "short", 33, mode="draft", Hq=64, Hkv=8, D=64,
              dtype="f16", prefix=1001),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("layout", "rope", "attend", "attend", "attend", "shared", "shared"))
    page = rng.choice((8, 16, 16, 32, 64, 128))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "layout":
        return _case(None, op, rng.choice(("uniform", "lognormal", "bimodal", "pareto")),
                     _log(rng, 1, 1000), mode=rng.choice(("decode", "draft", "prefill", "mixed")),
                     page=page)
    Hq, Hkv = rng.choice(((32, 8), (32, 4), (16, 16), (8, 1), (40, 8), (64, 8), (12, 4), (28, 4)))
    D = rng.choice((64, 128, 128, 256))
    if op == "rope":
        most = 32000 * 48 * 128 // ((Hq + 2 * Hkv) * D)
        return _case(None, op, n_tok=_log(rng, 1, min(most, 32000)), Hq=Hq, Hkv=Hkv, D=D,
                     dtype=dtype, page=page, interleaved=rng.random() < 0.4,
                     rot=rng.choice((D, D, D // 2)))
    window, sinks = rng.choice(((0, 0), (0, 0), (256, 4), (1000, 1), (1024, 0), (2048, 16),
                                (4096, 33)))
    if op == "shared":
        shape, mode = "short", rng.choice(("decode", "decode", "draft"))
        prefix = _log(rng, 100, 8192)
        window, sinks = rng.choice(((0, 0), (0, 0), (0, 0), (window, sinks)))
        n = _log(rng, 1, 128)
    else:
        prefix = 0
        mode = rng.choice(("decode", "decode", "decode", "draft", "mixed", "prefill"))
        shape = rng.choice(("lognormal", "bimodal", "pareto", "uniform"))
        n = _log(rng, 1, {"prefill": 6, "mixed": 50}.get(mode, 400))
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:  # no dearer than the dearest listed case, padded forms included
        c = _case(None, op, shape, n, mode=mode, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=page,
                  window=window, sinks=sinks, prefix=prefix)
        new, kv = _lengths(c)
        keys, w = n * max(kv), work(c)
        if n == 1 or (keys * Hkv * D < 5e9 and (keys + n * prefix) * Hq * max(new) < 4e9
                      and all(w[k] <= most[k] for k in most)):
            return c
        n = n * 2 // 3


def _lengths(case):
    """(new tokens, tokens held after the step) of every request, in a fixed order."""
    n, shape, mode = case["n_req"], case["shape"], case["mode"]
    u = [(i + 0.5) / n for i in range(n)]
    z = statistics.NormalDist().inv_cdf

    def uniform(lo, hi):
        return lambda x: lo + int(x * (hi + 1 - lo))

    def lognormal(median, sigma, lo, hi):
        return lambda x: min(hi, max(lo, round(median * math.exp(sigma * z(x)))))

    prompt, output = {
        "uniform": (uniform(1, 16), uniform(1, 32)),
        "lognormal": (lognormal(512, 1.0, 1, 8192), lognormal(200, 1.1, 1, 4096)),
        "bimodal": (uniform(32, 2048), lambda x: uniform(16, 128)(x / 0.8) if x < 0.8
                    else uniform(1024, 4096)((x - 0.8) / 0.2)),
        "pareto": (lognormal(1024, 0.8, 1, 16384),
                   lambda x: min(8192, max(8, int(8 * (1 - x) ** (-1 / 1.5))))),
        "prompts": (uniform(2048, 8192), uniform(16, 128)),
        "short": (lognormal(90, 0.82, 1, 905), uniform(16, 128)),
    }[shape]
    rng = random.Random(n)
    outs, done = [output(x) for x in u], list(u)
    rng.shuffle(outs)
    rng.shuffle(done)
    new, kv = [], []
    for i in range(n):
        p, progress = prompt(u[i]), int(done[i] * outs[i])
        if mode == "prefill":
            new.append(p)
            kv.append(p)
        elif mode == "mixed" and i % 8 == 0:  # a prompt on its way in, in chunks
            at = int(done[i] * p)
            new.append(min(_CHUNK, p - at))
            kv.append(at + new[-1])
        else:
            new.append(1 + i % _DRAFT if mode == "draft" else 1)
            kv.append(p + progress + new[-1])
    return new, kv


def _ceil(a, b):
    return -(-a // b)


def _visible(case, p):
    """Keys that a token at position p sees."""
    w = case["window"]
    return p + 1 if not w else min(p + 1, w) + min(case["sinks"], max(0, p + 1 - w))


def work(case):
    """Each input read once and each output written once: of the cache what some token
    of its request sees (the prefix once for all), of a block table the entries in use;
    two products per visible key, query head and token."""
    op, page, D, Hq, Hkv = (case[k] for k in ("op", "page", "D", "Hq", "Hkv"))
    if op == "rope":
        n, rot = case["n_tok"], case["rot"]
        row = (Hq + 2 * Hkv) * D * 2
        return {"bytes": n * (2 * row + 4 * rot + 8), "flops": n * (Hq + Hkv) * (4 * D + 3 * rot)}
    new, kv = _lengths(case)
    n, tokens = len(new), sum(new)
    if op == "layout":
        pages = sum(_ceil(b, page) - _ceil(b - a, page) for a, b in zip(new, kv))
        return {"bytes": 8 * n + 8 * pages + 8 * tokens + 4 * (2 * n + 1) + 8,
                "flops": 4 * tokens}
    keys = rows = 0
    pre, w, sinks = case["prefix"], case["window"], case["sinks"]
    pre_keys, lowest = (pre, pre) if not w else (0, pre)
    for a, b in zip(new, kv):
        first, last = pre + b - a, pre + b - 1
        lo = max(0, first - w + 1) if w else 0  # the first key of the window
        keys += b - max(0, max(0, lo - pre) - max(0, sinks - pre))
        lowest = min(lowest, lo)
        rows += sum(_visible(case, p) for p in range(first, last + 1))
    if w:
        pre_keys = pre - max(0, lowest - sinks)
    size = 4 * (_ceil(pre_keys, page) + sum(_ceil(b, page) for b in kv) + 2 * n + 1)
    return {"bytes": tokens * Hq * (4 * D + 4) + (keys + pre_keys) * Hkv * D * 4 + size,
            "flops": 4 * D * Hq * rows}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, page = case["op"], case["page"]
    Hq, Hkv, D, rot = case["Hq"], case["Hkv"], case["D"], case["rot"]
    dt = _DTYPES[case["dtype"]]

    def normal(*size, dtype=dt):
        return torch.randn(size, device="cuda", dtype=dtype, generator=g)

    s = dict(case)
    if op == "rope":
        n = case["n_tok"]
        n_pages = _ceil(n + n // 4 + page, page)
        angle = torch.arange(16384, device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) / (rot // 2))
        slots = torch.randperm(n_pages * page, device="cuda", generator=g)[:n].to(torch.int32)
        pad = torch.rand(n, device="cuda", generator=g) < 0.01  # rows that no request uses
        s.update(
            qkv=normal(n, Hq + 2 * Hkv, D) * (0.2 + 2 * torch.rand(n, 1, 1, device="cuda",
                                                                   generator=g)).to(dt),
            positions=torch.randint(0, 16384, (n,), device="cuda", dtype=torch.int32, generator=g),
            slots=torch.where(pad, -1, slots),
            cos_sin=torch.cat((angle.cos(), angle.sin()), 1).float().contiguous(),
            k_cache=normal(n_pages, Hkv, page, D), v_cache=normal(n_pages, Hkv, page, D),
            q_weight=1 + 0.1 * normal(D), k_weight=1 + 0.1 * normal(D))
        return s

    new, kv = _lengths(case)
    order = list(range(len(new)))
    random.Random(int(seed)).shuffle(order)
    new, kv = [new[i] for i in order], [kv[i] for i in order]
    n, tokens, pre = len(new), sum(new), case["prefix"]
    need = [_ceil(b, page) for b in kv]
    width = max(need) + 1
    total = sum(need) + _ceil(pre, page)
    n_pages = total + total // 8 + 1
    ids = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    new_t, kv_t, need_t = _i32(new), _i32(kv), _i32(need)
    col = torch.arange(width, device="cuda", dtype=torch.int32)
    start = torch.cumsum(need_t, 0, dtype=torch.int32) - need_t
    used = col[None, :] < need_t[:, None]
    table = torch.where(used, ids[(start[:, None] + col[None, :]).clamp(max=total - 1).long()], -1)
    if op == "layout":
        old = kv_t - new_t
        have = (old + page - 1) // page
        table = torch.where(col[None, :] < have[:, None], table, -1)
        left = torch.ones(n_pages, dtype=torch.bool, device="cuda")
        left[table[table >= 0].long()] = False
        free = ids[left[ids.long()]]
        s.update(old=old, new=new_t, table=table.contiguous(), free=free.contiguous(),
                 tokens=tokens)
        return s
    prefix_pages = ids[sum(need):total].contiguous()
    if case["window"]:  # pages that no token sees any more have gone back to the free list
        lo = pre + kv_t - new_t - case["window"] + 1
        gone = (pre + (col[None, :] + 1) * page <= lo[:, None]) & \
            (pre + col[None, :] * page >= case["sinks"])
        table = torch.where(gone, -1, table)
    k, v = (normal(n_pages, Hkv, page, D) for _ in range(2))
    # what no request has written is undefined: NaN here
    held = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    slot = torch.arange(page, device="cuda", dtype=torch.int32)
    fill = col[None, :, None] * page + slot < kv_t[:, None, None]
    live = table >= 0
    held[table[live].long()] = fill[live]
    if pre:
        held[prefix_pages.long()] = \
            (torch.arange(len(prefix_pages) * page, device="cuda") < pre).view(-1, page)
    for x in (k, v):
        x.masked_fill_(~held[:, None, :, None], math.nan)
    s.update(q=2 * normal(tokens, Hq, D), k_cache=k, v_cache=v, table=table.contiguous(),
             prefix_pages=prefix_pages,
             q_start=torch.cat((_i32([0]), torch.cumsum(new_t, 0, dtype=torch.int32))),
             kv_len=kv_t, max_q=max(new), scale=D ** -0.5)
    return s


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2608_02244_amd as fs
    if s["op"] == "layout":
        got = fs.kv_layout(s["old"], s["new"], s["table"], s["free"], page_size=s["page"],
                           n_tok=s["tokens"])
        return [s["table"], *got]
    if s["op"] == "rope":
        q = fs.qk_norm_rope(s["qkv"], s["positions"], s["slots"], s["cos_sin"], s["k_cache"],
                            s["v_cache"], s["q_weight"], s["k_weight"], eps=_EPS,
                            interleaved=s["interleaved"])
        return [q, s["k_cache"], s["v_cache"]]
    kw = dict(scale=s["scale"], window=s["window"], n_sink=s["sinks"], max_q=s["max_q"],
              return_lse=True)
    if s["op"] == "attend":
        return fs.attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["q_start"],
                         s["kv_len"], **kw)
    return fs.attend_shared(s["q"], s["k_cache"], s["v_cache"], s["prefix_pages"], s["prefix"],
                            s["table"], s["q_start"], s["kv_len"], **kw)


def _run_plain(s):
    return {"layout": _plain_layout, "rope": _plain_rope, "attend": _plain_attend,
            "shared": _plain_attend}[s["op"]](s)


def _plain_layout(s):
    page, table, free, old, new = s["page"], s["table"], s["free"], s["old"], s["new"]
    kv = old + new
    have, need = (old + page - 1) // page, (kv + page - 1) // page
    more = need - have
    start = torch.cumsum(more, 0) - more
    col = torch.arange(table.shape[1], device="cuda", dtype=torch.int32)[None, :]
    at = (start[:, None] + col - have[:, None]).clamp(0, max(0, len(free) - 1))
    fresh = (col >= have[:, None]) & (col < need[:, None])
    table.copy_(torch.where(fresh, free[at], table))
    q_start = torch.nn.functional.pad(torch.cumsum(new, 0, dtype=torch.int32), (1, 0))
    token = torch.arange(s["tokens"], device="cuda", dtype=torch.int32)
    req = torch.searchsorted(q_start[1:].contiguous(), token, right=True)
    pos = old[req] + token - q_start[:-1][req]
    slots = table[req, pos // page] * page + pos % page
    used = torch.stack((more.sum(), new.sum())).to(torch.int32)
    return [table, slots, pos, q_start, kv, used]


def _norm_rotate(x, weight, cos, sin, interleaved):
    half = cos.shape[-1]
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * weight
    y, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :half], y[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((y, rest), -1)


def _plain_rope(s):
    Hq, Hkv, half, page = s["Hq"], s["Hkv"], s["rot"] // 2, s["page"]
    dt = s["qkv"].dtype
    q, k, v = s["qkv"].split((Hq, Hkv, Hkv), 1)
    cs = s["cos_sin"][s["positions"].long()][:, None, :]
    cos, sin = cs[..., :half], cs[..., half:]
    q = _norm_rotate(q.float(), s["q_weight"].float(), cos, sin, s["interleaved"]).to(dt)
    k = _norm_rotate(k.float(), s["k_weight"].float(), cos, sin, s["interleaved"]).to(dt)
    used = s["slots"] >= 0
    at = s["slots"][used].long()
    s["k_cache"][at // page, :, at % page] = k[used]
    s["v_cache"][at // page, :, at % page] = v[used]
    return [q, s["k_cache"], s["v_cache"]]


def _plain_attend(s):
    q, table, kv, q_start = s["q"], s["table"], s["kv_len"], s["q_start"]
    Hq, Hkv, D, pre, w = s["Hq"], s["Hkv"], s["D"], s["prefix"], s["window"]
    n, tokens, m, grp = len(kv), q.shape[0], s["max_q"], Hq // Hkv
    new = q_start[1:] - q_start[:-1]
    i = torch.arange(m, device="cuda")
    row = (q_start[:-1, None] + i).clamp(max=tokens - 1).long()  # [n, m]
    real = i < new[:, None]
    # rows of one request and key head: its tokens times the heads that share the keys
    qp = q[row].float().view(n, m, Hkv, grp, D).permute(0, 2, 1, 3, 4).reshape(n * Hkv, m * grp, D)

    def pages(cache, at, seen):
        x = cache[at.clamp(min=0).long()]  # [..., pages, Hkv, page, D]
        x = x.movedim(-3, -4).flatten(-3, -2).float()
        return torch.where(seen[..., None, :, None], x, 0.0)

    p = pre + (kv - new)[:, None] + i  # position of every row's token
    length = table.shape[1] * s["page"]
    j = torch.arange(length, device="cuda")
    held = (j < kv[:, None]) & (table >= 0).repeat_interleave(s["page"], 1)
    keys, values = pages(s["k_cache"], table, held), pages(s["v_cache"], table, held)
    scores = torch.bmm(qp, keys.view(n * Hkv, length, D).transpose(1, 2).contiguous())
    del keys
    at, seen = pre + j, held
    if pre:
        count = len(s["prefix_pages"]) * s["page"]
        jp = torch.arange(count, device="cuda")
        pk, pv = (pages(s[c], s["prefix_pages"], jp < pre) for c in ("k_cache", "v_cache"))
        flat = qp.view(n, Hkv, m * grp, D).transpose(0, 1).reshape(Hkv, n * m * grp, D)
        first = torch.bmm(flat, pk.transpose(1, 2).contiguous())
        first = first.view(Hkv, n, m * grp, count).transpose(0, 1)
        scores = torch.cat((first.reshape(n * Hkv, m * grp, count), scores), 2)
        at = torch.cat((jp, at))
        seen = torch.cat(((jp < pre).expand(n, count), held), 1)
    see = seen[:, None, :] & (at <= p[:, :, None])
    if w:
        see = see & ((at > p[:, :, None] - w) | (at < s["sinks"]))
    scores = (scores * s["scale"]).view(n, Hkv, m, grp, -1)
    scores = torch.where(see[:, None, :, None, :], scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(scores - top)
    del scores
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    e = e.view(n * Hkv, m * grp, -1)
    if pre:
        ep = e[..., :count].reshape(n, Hkv, m * grp, count).transpose(0, 1)
        out = torch.bmm(ep.reshape(Hkv, n * m * grp, count), pv)
        out = out.view(Hkv, n, m * grp, D).transpose(0, 1).reshape(n * Hkv, m * grp, D)
        out = out + torch.bmm(e[..., count:].contiguous(), values.view(n * Hkv, length, D))
    else:
        out = torch.bmm(e, values.view(n * Hkv, length, D))
    out = out.view(n, Hkv, m, grp, D) / torch.where(total > 0, total, 1.0)
    out = out.permute(0, 2, 1, 3, 4).reshape(n * m, Hq, D)
    lse = lse.permute(0, 2, 1, 3).reshape(n * m, Hq)
    # back to the tokens' order: token t is row t - q_start of its request
    token = torch.arange(tokens, device="cuda", dtype=torch.int32)
    req = torch.searchsorted(q_start[1:].contiguous(), token, right=True)
    at = req * m + (token - q_start[:-1][req])
    return out[at].to(q.dtype), lse[at]


def exact(case, seed):
    if case["op"] == "layout":
        return None  # whole numbers, held to equality
    s = prepare(case, seed)
    return _exact_rope(s) if case["op"] == "rope" else _exact_attend(s)


def _exact_rope(s):
    """Each head as complex numbers (pairs of its rotated part) times exp(i angle)."""
    Hq, Hkv, rot, half, page = s["Hq"], s["Hkv"], s["rot"], s["rot"] // 2, s["page"]
    x = s["qkv"].double()
    cs = s["cos_sin"].double()[s["positions"].long()]
    turn = torch.complex(cs[:, :half], cs[:, half:])[:, None, :]

    def side(y, weight):
        y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / s["D"] + _EPS) * weight.double()
        if s["interleaved"]:
            z = torch.view_as_complex(y[..., :rot].unflatten(-1, (half, 2)).contiguous()) * turn
            r = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(y[..., :half].contiguous(), y[..., half:rot].contiguous()) * turn
            r = torch.cat((z.real, z.imag), -1)
        return torch.cat((r, y[..., rot:]), -1)

    caches = []
    used = (s["slots"] >= 0).nonzero()[:, 0]
    at = s["slots"][used].long()
    k = side(x[:, Hq:Hq + Hkv], s["k_weight"])
    for cache, rows in ((s["k_cache"], k), (s["v_cache"], x[:, Hq + Hkv:])):
        flat = cache.double().transpose(1, 2).reshape(-1, Hkv, s["D"])
        flat[at] = rows[used]
        caches.append(flat.view(-1, page, Hkv, s["D"]).transpose(1, 2).contiguous())
    return [side(x[:, :Hq], s["q_weight"]), *caches]


def _exact_attend(s):
    """Request by request, over the keys that it holds."""
    Hq, Hkv, D, page, pre, w = (s[k] for k in ("Hq", "Hkv", "D", "page", "prefix", "window"))
    start, kv = s["q_start"].tolist(), s["kv_len"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device="cuda")

    def rows(cache, ids, count):
        x = cache[ids.clamp(min=0).long()].transpose(1, 2).reshape(-1, Hkv, D)[:count]
        return x.double().nan_to_num(0.0).transpose(0, 1)

    pk, pv = (rows(s[c], s["prefix_pages"], pre) for c in ("k_cache", "v_cache"))
    for r in range(len(kv)):
        a, b = start[r], start[r + 1]
        ids = s["table"][r, :_ceil(kv[r], page)]
        gone = (ids < 0).repeat_interleave(page)[:kv[r]]
        k = torch.cat((pk, rows(s["k_cache"], ids, kv[r])), 1)
        v = torch.cat((pv, rows(s["v_cache"], ids, kv[r])), 1)
        j = torch.arange(pre + kv[r], device="cuda")
        p = (pre + kv[r] - (b - a) + torch.arange(b - a, device="cuda"))[:, None]
        hide = (j > p) | ((j <= p - w) & (j >= s["sinks"]) if w else torch.zeros_like(j > p))
        hide[:, pre:] |= gone
        for h in range(Hq):  # one head at a time: a long prompt's scores are large
            c = h // (Hq // Hkv)
            t = (s["q"][a:b, h].double() @ k[c].t()) * s["scale"]
            t = t.masked_fill(hide, -math.inf)
            lse[a:b, h] = torch.logsumexp(t, -1)
            out[a:b, h] = torch.softmax(t, -1) @ v[c]
    return out, lse
