"""The operators of a KV cache within a budget whose speed is measured.

The budget of tokens that a schedule is priced under is bytes on the worker.  These
operators hold more tokens in them, and give up those that matter least:

  store   queries and keys normed and rotated, keys and values into a cache of 4 bits an
          element (qk_norm_rope4), and what was stored read back (kv4_read)
  attend  attention of a step's new tokens over that cache (attend4): decode, drafts,
          prompts, mixes; a window with sinks, a shared prefix
  weight  the attention weight that every held token gets from the step's new tokens,
          summed over tokens and heads and added to what it had (attend_weight over a
          16-bit cache, attend4_weight over a 4-bit one)
  evict   pages of least weight given up until every request is within its budget, table
          and weights closed up (kv_evict)

A case is a dict of plain values:
  op        store | attend | weight | evict
  shape     distribution of the request lengths
  n_req     requests in the batch; n_tok: tokens of a store case
  mode      decode | draft | prefill | mixed: how many new tokens each request has
  Hq, Hkv, D, dtype, page  heads, head size, element type and tokens per page
  bits      16 | 4: what the cache of a weight case holds
  window, sinks, prefix    attention span (0: all), first visible tokens, prefix tokens
  budget, recent           tokens that a request may keep, last tokens that stay

The 4-bit cache: per head, 32 neighbouring elements x share a scale s = 2^e, the least
with max |x| <= 6 s (e within the element type's range), and each is the nearest of
+-{0, 0.5, 1, 1.5, 2, 3, 4, 6} s (of two equally near the one whose code is even).  One byte
holds elements 2i (low) and 2i + 1; a scale is the byte e + 127, 255 for what is not finite.
uint8 [n_pages, Hkv, page / 16, 17 D]: 16 tokens' key codes [16][D / 2], value codes
[4][16][4][D / 32] (4 tokens in turn for each of 16 pieces of a head), key scales
[16][D / 32] and value scales [4][D / 32][4].

Request lengths are quantiles of the distribution, put in an order by the seed: the
work of a case does not depend on the seed.
"""
import math
import random
import statistics

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
_EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}  # of a scale: all values are normal numbers
_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_DRAFT = 4      # most tokens of one request in a draft step
_CHUNK = 512    # most prompt tokens that one request brings into a mixed step
_EPS = 1e-6


def _case(name, op, shape="lognormal", n_req=0, n_tok=0, mode="decode", Hq=0, Hkv=0, D=0,
          dtype="bf16", page=16, bits=4, window=0, sinks=0, prefix=0, interleaved=False, rot=0,
          budget=0, recent=0):
    c = dict(op=op, shape=shape, n_req=n_req, n_tok=n_tok, mode=mode, Hq=Hq, Hkv=Hkv, D=D,
             dtype=dtype, page=page, bits=bits, window=window, sinks=sinks, prefix=prefix,
             interleaved=interleaved, rot=rot, budget=budget, recent=recent)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the projection of a decode step of 64 requests: launch-bound
        _case("store_decode", "store", n_tok=64, Hq=32, Hkv=8, D=128, rot=128),
        # prompts of a long admission, an odd number of tokens, half of each head rotated
        # in pairs of neighbours
        _case("store_prefill", "store", n_tok=32771, Hq=32, Hkv=8, D=128, dtype="f16", page=32,
              interleaved=True, rot=64),
        # the smallest batch of the benchmark: 8 requests of a few tokens
        _case("attend4_decode_few", "attend", "uniform", 8, Hq=32, Hkv=8, D=128),
        # a decode step of the throughput headline's batch (B = 512): heavy-tailed, about
        # 0.7 M tokens held
        _case("attend4_decode_heavy", "attend", "pareto", 512, Hq=32, Hkv=4, D=128, page=32),
        # two requests that hold a long context each: the keys of few rows over the device
        _case("attend4_decode_long", "attend", "long", 2, Hq=40, Hkv=8, D=128, dtype="f16",
              page=64),
        # whole prompts: the products of a long prefill
        _case("attend4_prefill", "attend", "prompts", 5, mode="prefill", Hq=16, Hkv=4, D=128,
              page=64),
        # chunks of prompts beside decoding requests, with a window over long contexts
        _case("attend4_mixed", "attend", "bimodal", 50, mode="mixed", Hq=32, Hkv=8, D=64,
              dtype="f16", window=2048, sinks=16),
        # a decode step under the KV budget of 65,536 tokens, cache of 16 bits
        _case("weight_decode", "weight", "lognormal", 64, Hq=32, Hkv=8, D=128, bits=16),
        # the headline's batch, cache of 4 bits
        _case("weight4_decode_heavy", "weight", "pareto", 512, Hq=32, Hkv=4, D=128, page=32),
        # whole prompts: which of their tokens were looked at
        _case("weight_prefill", "weight", "prompts", 5, mode="prefill", Hq=16, Hkv=4, D=128,
              page=64, bits=16),
        # the smallest batch: 8 requests of a few pages
        _case("evict_few", "evict", "lognormal", 8, budget=256, sinks=4, recent=64),
        # the headline's batch cut to half of what it holds
        _case("evict_heavy", "evict", "pareto", 512, page=32, budget=1024, sinks=16, recent=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("store", "attend", "attend", "attend", "weight", "weight", "evict"))
    page = rng.choice((16, 16, 32, 64, 128))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    if op == "evict":
        return _case(None, op, rng.choice(("lognormal", "bimodal", "pareto")),
                     _log(rng, 1, 500), page=page, budget=_log(rng, 16, 2000),
                     sinks=rng.choice((0, 1, 4, 33)), recent=rng.choice((0, 1, 64, 300)))
    Hq, Hkv = rng.choice(((32, 8), (32, 4), (16, 16), (8, 1), (40, 8), (64, 8), (12, 4), (28, 4)))
    D = rng.choice((64, 128, 128, 256))
    if op == "store":
        most = 32000 * 48 * 128 // ((Hq + 2 * Hkv) * D)
        return _case(None, op, n_tok=_log(rng, 1, min(most, 32000)), Hq=Hq, Hkv=Hkv, D=D,
                     dtype=dtype, page=page, interleaved=rng.random() < 0.4,
                     rot=rng.choice((D, D, D // 2)))
    window, sinks = rng.choice(((0, 0), (0, 0), (256, 4), (1000, 1), (1024, 0), (2048, 16),
                                (4096, 33)))
    prefix, bits = 0, 4
    mode = rng.choice(("decode", "decode", "decode", "draft", "mixed", "prefill"))
    shape = rng.choice(("lognormal", "bimodal", "pareto", "uniform"))
    n = _log(rng, 1, {"prefill": 6, "mixed": 50}.get(mode, 400))
    if op == "weight":
        bits = rng.choice((16, 4))
        page = page if bits == 4 else rng.choice((8, page))
    elif rng.random() < 0.3:
        shape, mode, prefix = "short", rng.choice(("decode", "decode", "draft")), \
            _log(rng, 100, 8192)
        n = min(n, 128)
    elif rng.random() < 0.2:
        shape, mode, n = "long", "decode", rng.randint(1, 2)
    most = {k: max(work(c)[k] for c in listed() if c["op"] == op) for k in ("bytes", "flops")}
    while True:  # no dearer than the dearest listed case, padded forms included
        c = _case(None, op, shape, n, mode=mode, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=page,
                  bits=bits, window=window, sinks=sinks, prefix=prefix)
        new, kv = _lengths(c)
        keys, w = n * max(kv), work(c)
        if n == 1 or (keys * Hkv * D < 4e9 and (keys + n * prefix) * Hq * max(new) < 4e9
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
        "long": (uniform(60000, 130000), uniform(16, 4096)),
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


def _dropped(case, kv):
    """Pages that each request gives up."""
    page, got = case["page"], []
    for m in kv:
        first = _ceil(case["sinks"], page)
        last = max(0, m - case["recent"]) // page
        got.append(min(_ceil(max(0, m - case["budget"]), page), max(0, last - first)))
    return got


def work(case):
    """Each input read once and each output written once: of the cache what some token
    of its request sees (the prefix once for all), of a block table the entries in use;
    two products per visible key, query head and token, one where only weights are wanted."""
    op, page, D, Hq, Hkv = (case[k] for k in ("op", "page", "D", "Hq", "Hkv"))
    if op == "store":
        n, rot = case["n_tok"], case["rot"]
        half = 2 * Hkv * D * 17 // 32  # keys and values of a token in 4 bits
        return {"bytes": n * (2 * (Hq + 2 * Hkv) * D + 2 * Hq * D + 4 * rot + 12 + 2 * half
                              + 4 * Hkv * D),
                "flops": n * (Hq + Hkv) * (4 * D + 3 * rot)}
    new, kv = _lengths(case)
    n, tokens = len(new), sum(new)
    width = max(_ceil(b, page) for b in kv) + 1
    if op == "evict":
        pages, gone = sum(_ceil(b, page) for b in kv), sum(_dropped(case, kv))
        return {"bytes": 4 * (sum(kv) + n * width * page + pages + n * width + 3 * n + gone + 1),
                "flops": sum(kv)}
    keys = own_rows = rows = 0
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
    elem = 2 * D if case["bits"] == 16 else D * 17 // 32  # bytes of a key of one head
    if op == "weight":
        return {"bytes": tokens * Hq * (2 * D + 4) + keys * (Hkv * elem + 8) + size,
                "flops": 2 * D * Hq * rows}
    return {"bytes": tokens * Hq * (4 * D + 4) + (keys + pre_keys) * Hkv * 2 * elem + size,
            "flops": 4 * D * Hq * rows}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _quantise(x, dtype):
    """Codes (uint8, one an element) and scale bytes of the last dimension's blocks of 32."""
    lo, hi = _EXPONENTS[dtype]
    b = x.unflatten(-1, (x.shape[-1] // 32, 32))
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)  # top = m 2^e with m in [0.5, 1): at most 6 2^(e - 3) or 6 2^(e - 2)
    e = torch.where(m <= 0.75, e - 3, e - 2)
    e = torch.where(top > 0, e, lo).clamp(lo, hi)
    y = torch.ldexp(b.abs().double(), -e)
    code = torch.zeros_like(y, dtype=torch.uint8)
    # past the middle of two levels; at the middle itself where the upper code is even
    code += (y > 0.25).byte() + (y >= 0.75).byte() + (y > 1.25).byte() + (y >= 1.75).byte()
    code += (y > 2.5).byte() + (y >= 3.5).byte() + (y > 5.0).byte()
    code += torch.signbit(b).byte() * 8
    return code.flatten(-2), (e + 127).squeeze(-1).byte()


def _parts(cache, D):
    """Views of a cache's key codes, value codes, key scales and value scales, the last
    three dimensions those of the format."""
    kc, vc, ks, vs = cache.split((8 * D, 8 * D, D // 2, D // 2), -1)
    return (kc.unflatten(-1, (16, D // 2)), vc.unflatten(-1, (4, 16, 4, D // 32)),
            ks.unflatten(-1, (16, D // 32)), vs.unflatten(-1, (4, D // 32, 4)))


def _bytes(code):
    """Two codes a byte."""
    return code[..., 0::2] + code[..., 1::2] * 16


def _fill(cache, k, v, dtype):
    """Keys and values [pages, heads, page, D] to a cache's bytes."""
    D = k.shape[-1]
    kc, vc, ks, vs = _parts(cache, D)
    code, scale = _quantise(k, dtype)
    kc.copy_(_bytes(code).unflatten(2, (-1, 16)))
    ks.copy_(scale.unflatten(2, (-1, 16)))
    code, scale = _quantise(v, dtype)
    vc.copy_(_bytes(code).unflatten(2, (-1, 4, 4)).unflatten(-1, (16, D // 32)).transpose(4, 5))
    vs.copy_(scale.unflatten(2, (-1, 4, 4)).transpose(4, 5))


def _values(cache, D, value):
    """The keys (or values) [pages, heads, page, D] that a cache's bytes stand for, in 32 bits."""
    kc, vc, ks, vs = _parts(cache, D)
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device="cuda")
    i = torch.arange(256, device="cuda")
    pair = torch.stack((level[i % 16], level[i // 16]), -1)

    def side(code, scale):  # [pages, heads, groups, 16, D / 2], [.., D / 32]
        x = pair.index_select(0, code.reshape(-1).int()).view(*code.shape[:-1], -1, 32)
        s = torch.exp2(scale.float() - 127)
        s = torch.where(scale == 255, math.nan, s)
        return (x * s[..., None]).flatten(-2).flatten(2, 3)
    if value:
        return side(vc.transpose(4, 5).flatten(-2).flatten(3, 4), vs.transpose(4, 5).flatten(3, 4))
    return side(kc, ks)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, page = case["op"], case["page"]
    Hq, Hkv, D, rot = case["Hq"], case["Hkv"], case["D"], case["rot"]
    dt = _DTYPES[case["dtype"]]

    def normal(*size, dtype=dt):
        return torch.randn(size, device="cuda", dtype=dtype, generator=g)

    def weights(kv, length):
        """What earlier steps added: heavy-tailed, nothing behind a request's last token."""
        x = normal(len(kv), length, dtype=torch.float32).mul_(2).exp_().mul_(0.1)
        return x.masked_fill_(torch.arange(length, device="cuda") >= kv[:, None], 0.0)

    s = dict(case)
    if op == "store":
        n = case["n_tok"]
        n_pages = _ceil(n + n // 4 + page, page)
        angle = torch.arange(16384, device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) / (rot // 2))
        # requests' tokens in pages of their own, pages anywhere in the cache
        at = torch.arange(n, device="cuda")
        slots = torch.randperm(n_pages, device="cuda", generator=g)[at // page] * page + at % page
        pad = torch.rand(n, device="cuda", generator=g) < 0.01  # rows that no request uses
        s.update(
            qkv=normal(n, Hq + 2 * Hkv, D) * (0.2 + 2 * torch.rand(n, 1, 1, device="cuda",
                                                                   generator=g)).to(dt),
            positions=torch.randint(0, 16384, (n,), device="cuda", dtype=torch.int32, generator=g),
            slots=torch.where(pad, -1, slots).to(torch.int32),
            cos_sin=torch.cat((angle.cos(), angle.sin()), 1).float().contiguous(),
            cache=torch.zeros(n_pages, Hkv, page // 16, 17 * D, dtype=torch.uint8, device="cuda"),
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
    if op == "evict":
        s.update(table=table.contiguous(), kv_len=kv_t, weight=weights(kv_t, width * page),
                 budgets=_i32([case["budget"]] * n), n_freed=sum(_dropped(case, kv)))
        return s
    prefix_pages = ids[sum(need):total].contiguous()
    if case["window"]:  # pages that no token sees any more have gone back to the free list
        lo = pre + kv_t - new_t - case["window"] + 1
        gone = (pre + (col[None, :] + 1) * page <= lo[:, None]) & \
            (pre + col[None, :] * page >= case["sinks"])
        table = torch.where(gone, -1, table)
    # what no request has written is undefined: NaN here
    held = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
    slot = torch.arange(page, device="cuda", dtype=torch.int32)
    fill = col[None, :, None] * page + slot < kv_t[:, None, None]
    live = table >= 0
    held[table[live].long()] = fill[live]
    if pre:
        held[prefix_pages.long()] = \
            (torch.arange(len(prefix_pages) * page, device="cuda") < pre).view(-1, page)
    k, v = (normal(n_pages, Hkv, page, D) for _ in range(2))
    if case["bits"] == 4:
        cache = torch.empty(n_pages, Hkv, page // 16, 17 * D, dtype=torch.uint8, device="cuda")
        for a in range(0, n_pages, 4096):  # some pages at a time: the steps in between are large
            b = slice(a, a + 4096)
            _fill(cache[b], k[b].float(), v[b].float(), case["dtype"])
        ks, vs = _parts(cache, D)[2:]
        ks.masked_fill_(~held.view(n_pages, 1, -1, 16, 1), 255)
        vs.masked_fill_(~held.view(n_pages, 1, -1, 4, 1, 4), 255)
        s.update(cache=cache)
    else:
        s.update(k_cache=k.masked_fill_(~held[:, None, :, None], math.nan))
    del k, v
    s.update(q=2 * normal(tokens, Hq, D), table=table.contiguous(), prefix_pages=prefix_pages,
             q_start=torch.cat((_i32([0]), torch.cumsum(new_t, 0, dtype=torch.int32))),
             kv_len=kv_t, max_q=max(new), scale=D ** -0.5)
    if op == "weight":
        scores, _, back = _scores(s)
        lse = torch.logsumexp(scores, -1).permute(0, 2, 1, 3).reshape(n * s["max_q"], Hq)
        s.update(lse=lse[back].contiguous(), weight=weights(kv_t, width * page))
    return s


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_2608_02244_amd as fs
    if s["op"] == "store":
        q = fs.qk_norm_rope4(s["qkv"], s["positions"], s["slots"], s["cos_sin"], s["cache"],
                             s["q_weight"], s["k_weight"], eps=_EPS,
                             interleaved=s["interleaved"])
        return [q, *fs.kv4_read(s["cache"], s["slots"], dtype=q.dtype)]
    if s["op"] == "evict":
        got = fs.kv_evict(s["weight"], s["kv_len"], s["table"], s["budgets"],
                          page_size=s["page"], n_sink=s["sinks"], n_recent=s["recent"],
                          n_freed=s["n_freed"])
        return list(got)
    kw = dict(scale=s["scale"], window=s["window"], n_sink=s["sinks"], max_q=s["max_q"])
    step = s["table"], s["q_start"], s["kv_len"]
    if s["op"] == "weight":
        if s["bits"] == 4:
            return fs.attend4_weight(s["q"], s["lse"], s["cache"], *step, s["weight"], **kw)
        return fs.attend_weight(s["q"], s["lse"], s["k_cache"], *step, s["weight"], **kw)
    if s["prefix"]:
        kw.update(prefix_pages=s["prefix_pages"], prefix_len=s["prefix"])
    return fs.attend4(s["q"], s["cache"], *step, return_lse=True, **kw)


def _run_plain(s):
    return {"store": _plain_store, "attend": _plain_attend, "weight": _plain_weight,
            "evict": _plain_evict}[s["op"]](s)


def _norm_rotate(x, weight, cos, sin, interleaved):
    half = cos.shape[-1]
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * weight
    y, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :half], y[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((y, rest), -1)


def _plain_store(s):
    Hq, Hkv, D, half, page = s["Hq"], s["Hkv"], s["D"], s["rot"] // 2, s["page"]
    dt = s["qkv"].dtype
    q, k, v = s["qkv"].split((Hq, Hkv, Hkv), 1)
    cs = s["cos_sin"][s["positions"].long()][:, None, :]
    cos, sin = cs[..., :half], cs[..., half:]
    q = _norm_rotate(q.float(), s["q_weight"].float(), cos, sin, s["interleaved"]).to(dt)
    # 64 bits: what is next to the border of two codes falls to one side
    k = _norm_rotate(k.double(), s["k_weight"].double(), cos.double(), sin.double(),
                     s["interleaved"])
    used = s["slots"] >= 0
    at = s["slots"][used].long()
    p, grp, t = at // page, at % page // 16, at % 16
    kc, vc, ks, vs = _parts(s["cache"], D)
    code, scale = _quantise(k[used], s["dtype"])
    kc[p, :, grp, t], ks[p, :, grp, t] = _bytes(code), scale
    code, scale = _quantise(v[used].float(), s["dtype"])
    vc[p, :, grp, t // 4, :, t % 4] = _bytes(code).unflatten(-1, (16, D // 32))
    vs[p, :, grp, t // 4, :, t % 4] = scale
    # and back: the slots' tokens as the cache holds them, zeros without a slot
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device="cuda")

    def read(code, scale):
        x = torch.stack((level[(code % 16).int()], level[(code // 16).int()]), -1)
        x = x.flatten(-2).unflatten(-1, (D // 32, 32)) * torch.exp2(scale.float() - 127)[..., None]
        out = torch.zeros(len(used), Hkv, D, device="cuda", dtype=dt)
        out[used] = x.flatten(-2).to(dt)
        return out
    return [q, read(kc[p, :, grp, t], ks[p, :, grp, t]),
            read(vc[p, :, grp, t // 4, :, t % 4].flatten(-2), vs[p, :, grp, t // 4, :, t % 4])]


def _keys(s):
    return s["k_cache"].float() if s["bits"] == 16 else _values(s["cache"], s["D"], False)


def _paged(cache, at, seen):
    x = cache[at.clamp(min=0).long()]  # [..., pages, Hkv, page, D]
    return torch.where(seen[..., None, :, None], x.movedim(-3, -4).flatten(-3, -2), 0.0)


def _scores(s):
    """Scores [n, Hkv, max_q, group, keys] with -inf where a row does not see a key, those
    of the prefix first; which own keys are held; the row of every token."""
    q, table, kv, q_start = s["q"], s["table"], s["kv_len"], s["q_start"]
    k = _keys(s)
    Hq, Hkv, D, pre, w = s["Hq"], s["Hkv"], s["D"], s["prefix"], s["window"]
    n, tokens, m, grp = len(kv), q.shape[0], s["max_q"], Hq // Hkv
    new = q_start[1:] - q_start[:-1]
    i = torch.arange(m, device="cuda")
    row = (q_start[:-1, None] + i).clamp(max=tokens - 1).long()  # [n, m]
    # rows of one request and key head: its tokens times the heads that share the keys
    qp = q[row].float().view(n, m, Hkv, grp, D).permute(0, 2, 1, 3, 4).reshape(n * Hkv, m * grp, D)
    p = pre + (kv - new)[:, None] + i  # position of every row's token
    length = table.shape[1] * s["page"]
    j = torch.arange(length, device="cuda")
    held = (j < kv[:, None]) & (table >= 0).repeat_interleave(s["page"], 1)
    keys = _paged(k, table, held)
    scores = torch.bmm(qp, keys.view(n * Hkv, length, D).transpose(1, 2).contiguous())
    del keys
    at, seen = pre + j, held
    if pre:
        count = len(s["prefix_pages"]) * s["page"]
        jp = torch.arange(count, device="cuda")
        pk = _paged(k, s["prefix_pages"], jp < pre)
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
    # back to the tokens' order: token t is row t - q_start of its request
    token = torch.arange(tokens, device="cuda", dtype=torch.int32)
    req = torch.searchsorted(q_start[1:].contiguous(), token, right=True)
    return scores, held, req * m + (token - q_start[:-1][req])


def _plain_attend(s):
    Hq, Hkv, D, pre, m = s["Hq"], s["Hkv"], s["D"], s["prefix"], s["max_q"]
    n, grp = len(s["kv_len"]), Hq // Hkv
    scores, held, back = _scores(s)
    v = _values(s["cache"], D, True)
    values = _paged(v, s["table"], held).view(n * Hkv, -1, D)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(scores - top)
    del scores
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    e = e.view(n * Hkv, m * grp, -1)
    if pre:
        count = len(s["prefix_pages"]) * s["page"]
        pv = _paged(v, s["prefix_pages"], torch.arange(count, device="cuda") < pre)
        ep = e[..., :count].reshape(n, Hkv, m * grp, count).transpose(0, 1)
        out = torch.bmm(ep.reshape(Hkv, n * m * grp, count), pv)
        out = out.view(Hkv, n, m * grp, D).transpose(0, 1).reshape(n * Hkv, m * grp, D)
        out = out + torch.bmm(e[..., count:].contiguous(), values)
    else:
        out = torch.bmm(e, values)
    out = out.view(n, Hkv, m, grp, D) / torch.where(total > 0, total, 1.0)
    out = out.permute(0, 2, 1, 3, 4).reshape(n * m, Hq, D)
    lse = lse.permute(0, 2, 1, 3).reshape(n * m, Hq)
    return out[back].to(s["q"].dtype), lse[back]


def _plain_weight(s):
    Hq, Hkv, m = s["Hq"], s["Hkv"], s["max_q"]
    n, grp = len(s["kv_len"]), Hq // Hkv
    scores, _, back = _scores(s)
    lse = torch.full((n * m, Hq), math.inf, device="cuda")  # rows past a request's last token
    lse[back] = s["lse"]
    lse = torch.where(lse == -math.inf, math.inf, lse)  # rows that see nothing
    lse = lse.view(n, m, Hkv, grp).permute(0, 2, 1, 3)
    s["weight"] += torch.exp(scores - lse[..., None]).sum((1, 2, 3))
    return s["weight"]


def _plain_evict(s):
    page, w, kv, table = s["page"], s["weight"], s["kv_len"], s["table"]
    n, width = table.shape
    score = w.double().view(n, width, page).sum(-1)
    c = torch.arange(width, device="cuda", dtype=torch.int32)
    may = ((c * page >= s["sinks"]) & ((c + 1) * page <= (kv - s["recent"])[:, None])
           & ((c + 1) * page <= kv[:, None]))
    need = ((kv - s["budgets"]).clamp(min=0) + page - 1) // page
    need = torch.minimum(need, may.sum(1, dtype=torch.int32))
    order = torch.argsort(torch.where(may, score, math.inf), dim=1, stable=True)
    rank = torch.empty_like(order).scatter_(1, order, c.long().expand(n, width))
    drop = may & (rank < need[:, None])
    kept = (c * page < kv[:, None]) & ~drop
    # kept pages first, in their order
    order = torch.argsort((~kept).byte(), dim=1, stable=True)
    stays = c < kept.sum(1, keepdim=True)
    new_table = torch.where(stays, table.gather(1, order), -1)
    pages = w.view(n, width, page).gather(1, order[..., None].expand(n, width, page))
    new_weight = torch.where(stays[..., None], pages, 0.0).view(n, width * page)
    gone = table[drop]
    freed = torch.full((s["n_freed"],), -1, dtype=torch.int32, device="cuda")
    freed[:] = gone[:s["n_freed"]]
    count = drop.sum(dtype=torch.int32).view(1)
    return [new_table, new_weight, kv - need * page, freed, count]


def exact(case, seed):
    if case["op"] == "evict":
        s = prepare(case, seed)
        return [None, _exact_evict(s), None, None, None]
    s = prepare(case, seed)
    return {"store": _exact_store, "attend": _exact_attend, "weight": _exact_weight}[s["op"]](s)


def _exact_store(s):
    """Each head as complex numbers (pairs of its rotated part) times exp(i angle); codes by
    the distance to every level."""
    Hq, Hkv, rot, half = s["Hq"], s["Hkv"], s["rot"], s["rot"] // 2
    lo, hi = _EXPONENTS[s["dtype"]]
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

    def coarse(y):
        # levels in the order in which min() is to take the first of equally near ones
        level = torch.tensor((0.0, 1.0, 2.0, 4.0, 0.5, 1.5, 3.0, 6.0), dtype=torch.float64,
                             device="cuda")
        z = y.unflatten(-1, (-1, 32))
        e = torch.ceil(torch.log2(z.abs().amax(-1, keepdim=True) / 6)).clamp(lo, hi)
        near, far = None, None
        for v in level:
            d = (z.abs() * 2.0 ** -e - v).abs()
            near = torch.where(d < far, v, near) if far is not None else v.expand_as(d)
            far = torch.minimum(d, far) if far is not None else d
        return (torch.copysign(near, z) * 2.0 ** e).flatten(-2) * (s["slots"] >= 0)[:, None, None]

    return [side(x[:, :Hq], s["q_weight"]), coarse(side(x[:, Hq:Hq + Hkv], s["k_weight"])),
            coarse(x[:, Hq + Hkv:])]


def _decoded(s, ids, count, value):
    """One request's first `count` keys (or values) [Hkv, count, D] in 64 bits, by the
    format's arithmetic."""
    Hkv, D = s["Hkv"], s["D"]
    if s["bits"] == 16:
        x = s["k_cache"][ids.clamp(min=0).long()].transpose(1, 2).reshape(-1, Hkv, D)[:count]
        return x.double().nan_to_num(0.0).transpose(0, 1)
    raw = s["cache"][ids.clamp(min=0).long()].transpose(1, 2).flatten(0, 1)  # [groups, Hkv, 17 D]
    if value:
        code = raw[..., 8 * D:16 * D].reshape(-1, Hkv, 4, 16, 4, D // 32).permute(0, 2, 4, 1, 3, 5)
        scale = raw[..., 33 * D // 2:].reshape(-1, Hkv, 4, D // 32, 4).permute(0, 2, 4, 1, 3)
    else:
        code = raw[..., :8 * D].reshape(-1, Hkv, 16, D // 2).permute(0, 2, 1, 3)
        scale = raw[..., 16 * D:33 * D // 2].reshape(-1, Hkv, 16, D // 32).permute(0, 2, 1, 3)
    code = code.reshape(-1, Hkv, D // 2)[:count].long()
    scale = scale.reshape(-1, Hkv, D // 32)[:count]
    c = torch.stack((code & 15, code >> 4), -1).flatten(-2)
    e, m = c >> 1 & 3, c & 1
    x = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e.double() - 1))
    x = torch.where(c > 7, -x, x) * 2.0 ** (scale.double() - 127).repeat_interleave(32, -1)
    return x.masked_fill((scale == 255).repeat_interleave(32, -1), 0.0).transpose(0, 1)


def _requests(s):
    """Request by request: its number, its rows, its keys and values, and what is hidden."""
    page, pre, w = s["page"], s["prefix"], s["window"]
    start, kv = s["q_start"].tolist(), s["kv_len"].tolist()
    need = s["op"] == "attend"
    if pre:
        pk, pv = (_decoded(s, s["prefix_pages"], pre, x) for x in (False, True))
    for r in range(len(kv)):
        a, b = start[r], start[r + 1]
        ids = s["table"][r, :_ceil(kv[r], page)]
        gone = (ids < 0).repeat_interleave(page)[:kv[r]]
        k = _decoded(s, ids, kv[r], False)
        v = _decoded(s, ids, kv[r], True) if need else None
        if pre:
            k, v = torch.cat((pk, k), 1), torch.cat((pv, v), 1) if need else None
        j = torch.arange(pre + kv[r], device="cuda")
        p = (pre + kv[r] - (b - a) + torch.arange(b - a, device="cuda"))[:, None]
        hide = (j > p) | ((j <= p - w) & (j >= s["sinks"]) if w else torch.zeros_like(j > p))
        hide[:, pre:] |= gone
        yield r, a, b, k, v, hide


def _exact_attend(s):
    Hq, grp = s["Hq"], s["Hq"] // s["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for r, a, b, k, v, hide in _requests(s):
        for h in range(Hq):  # one head at a time: a long prompt's scores are large
            t = (s["q"][a:b, h].double() @ k[h // grp].t()) * s["scale"]
            t = t.masked_fill(hide, -math.inf)
            lse[a:b, h] = torch.logsumexp(t, -1)
            out[a:b, h] = torch.softmax(t, -1) @ v[h // grp]
    return out, lse


def _exact_weight(s):
    Hq, grp = s["Hq"], s["Hq"] // s["Hkv"]
    weight = s["weight"].double()
    for r, a, b, k, v, hide in _requests(s):
        for h in range(Hq):
            t = (s["q"][a:b, h].double() @ k[h // grp].t()) * s["scale"]
            t = t.masked_fill(hide, -math.inf) - s["lse"][a:b, h, None].double()
            weight[r, :k.shape[1]] += t.exp().sum(0)
    return weight


def _exact_evict(s):
    """Request by request: the weights of the tokens that stay, on the host."""
    page, w = s["page"], s["weight"].double().cpu()
    out = torch.zeros_like(w)
    for r, m in enumerate(s["kv_len"].tolist()):
        first, last = _ceil(s["sinks"], page), max(0, m - s["recent"]) // page
        score = sorted((float(w[r, c * page:(c + 1) * page].sum()), c)
                       for c in range(first, last))
        drop = {c for _, c in score[:_ceil(max(0, m - s["budget"]), page)]}
        stay = [w[r, c * page:min(m, (c + 1) * page)] for c in range(_ceil(m, page))
                if c not in drop]
        stay = torch.cat(stay)
        out[r, :len(stay)] = stay
    return out.cuda()
