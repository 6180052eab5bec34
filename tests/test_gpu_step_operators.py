"""The step operators on the GPU against plain implementations in 64 bits.

Tolerances follow from the number formats and are fixed here before any run: with
u the unit roundoff of the 16-bit type (2^-8 for bf16, 2^-11 for f16),
  attention   |err| <= 1.1 u (A + |o|) + small, A = sum_j w_j |v_j| (the weights are
              rounded once for the products, the result once), small = 2^-19 (1 + A) for
              the 32-bit sums, scores and exponentials;
  lse         the 32-bit scores' rounding, (D + 8) 2^-24 scale sum_d |q_d k_jd| at most,
              plus that of the sum, the logarithm and the result;
  rotation    u |y| + 2^-20 times the pair's size.
Layouts are whole numbers and have to be equal."""
import math
import random
import sys

import pytest

import paper_2608_02244_amd as fs

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def dev():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def dtype_of(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


def log(msg):
    print(msg, flush=True)
    sys.stdout.flush()


# ---------------------------------------------------------------- kv_layout

def plain_layout(old, new, table, free, page, n_tok, first_pos=0):
    """One request and token after the other (lists)."""
    width = len(table[0]) if table else 0
    table = [list(r) for r in table]
    slots, pos, q_start, kv_len, taken = [], [], [0], [], 0
    for r, (o, m) in enumerate(zip(old, new)):
        o, m = max(0, o), max(0, m)
        have, need = min(-(-o // page), width), min(-(-(o + m) // page), width)
        for c in range(have, need):
            table[r][c] = free[taken] if taken < len(free) else -1
            taken += 1
        for i in range(o, o + m):
            c = i // page
            ok = c < width and table[r][c] >= 0 and table[r][c] * page + i % page < 2 ** 31
            slots.append(table[r][c] * page + i % page if ok else -1)
            pos.append(first_pos + i)
        q_start.append(q_start[-1] + m)
        kv_len.append(o + m)
    used = [taken, q_start[-1]]
    pad = max(0, n_tok - len(slots))
    return (table, slots[:n_tok] + [-1] * pad, pos[:n_tok] + [-1] * pad,
            [min(x, n_tok) for x in q_start], kv_len, used)


def check_layout(dev, old, new, width, page, n_free=None, n_tok=None, first_pos=0, seed=0):
    import torch
    rng = random.Random(seed)
    n = len(old)
    pages = sum(-(-max(0, o) // page) for o in old)
    total = pages + sum(-(-max(0, m) // page) + 1 for m in new)
    ids = list(range(total))
    rng.shuffle(ids)
    table, at = [], 0
    for o in old:
        k = min(width, -(-max(0, o) // page))
        table.append(ids[at:at + k] + [-1] * (width - k))
        at += k
    free = ids[at:] if n_free is None else ids[at:at + n_free]
    n_tok = sum(max(0, m) for m in new) if n_tok is None else n_tok

    def t(x, shape):
        return torch.tensor(x, dtype=torch.int32, device=dev).reshape(shape)
    gt = t(table, (n, width))
    log(f"kv_layout n={n} width={width} page={page} n_tok={n_tok} free={len(free)}")
    got = fs.kv_layout(t(old, (n,)), t(new, (n,)), gt, t(free, (len(free),)), page_size=page,
                       n_tok=n_tok, first_pos=first_pos)
    ref = plain_layout(old, new, table, free, page, n_tok, first_pos)
    names = ("table", "slots", "positions", "q_start", "kv_len", "used")
    for name, g, r in zip(names, (gt,) + got, ref):
        assert g.cpu().reshape(-1).tolist() == [y for x in r for y in
                                                (x if isinstance(x, list) else [x])], name


@pytest.mark.parametrize("page", [1, 2, 16, 64, 1024])
@pytest.mark.parametrize("n", [1, 2, 63, 257, 700])
def test_layout_mixed_requests(dev, n, page):
    rng = random.Random(n * 1000 + page)
    old = [rng.choice((0, 1, page - 1, page, page + 1, rng.randint(0, 300))) for _ in range(n)]
    new = [rng.choice((0, 1, 1, 1, 2, page, rng.randint(0, 90))) for _ in range(n)]
    check_layout(dev, old, new, max(-(-(o + m) // page) for o, m in zip(old, new)) + 2, page,
                 first_pos=rng.choice((0, 37)), seed=n)


def test_layout_largest_request_count(dev):
    rng = random.Random(1)
    n = 4096
    check_layout(dev, [rng.randint(0, 70) for _ in range(n)], [rng.randint(0, 3) for _ in range(n)],
                 8, 16)


def test_layout_one_long_prompt_and_silent_requests(dev):
    check_layout(dev, [0, 5, 0, 0, 9], [0, 0, 70001, 0, 0], 4400, 16)
    check_layout(dev, [0], [1], 1, 16)
    check_layout(dev, [0, 0, 0], [0, 0, 0], 2, 16)
    check_layout(dev, [17], [0], 2, 16, n_free=0)


def test_layout_what_does_not_fit(dev):
    check_layout(dev, [3, 16, 40], [40, 1, 30], 6, 16, n_free=2)          # too few free pages
    check_layout(dev, [3, 16, 40], [40, 1, 30], 6, 16, n_free=0)
    check_layout(dev, [3, 16, 40], [40, 1, 30], 3, 16)                    # rows too short
    check_layout(dev, [3, 16, 40], [40, 1, 30], 6, 16, n_tok=50)          # more tokens than room
    check_layout(dev, [3, 16, 40], [40, 1, 30], 6, 16, n_tok=100)         # fewer
    check_layout(dev, [-5, 16, 40], [40, -1, 30], 6, 16)                  # negative lengths
    check_layout(dev, [5, 6], [4, 5], 0, 16)                              # no table at all


def test_layout_slots_beyond_31_bits_and_lengths_near_the_type_s_end(dev):
    import torch

    def t(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)
    top = 2 ** 31 - 1
    table = t([[2 ** 27 - 1, -1], [2 ** 27, -1], [top, -1]])
    got = fs.kv_layout(t([4, 4, 4]), t([2, 2, 2]), table, t([1]), page_size=16, n_tok=6)
    assert got[0].tolist() == [top - 15 + 4, top - 15 + 5, -1, -1, -1, -1]
    # a request that can never fit: nothing overflows, the others keep their places
    table = t([[-1, -1], [-1, -1]])
    got = fs.kv_layout(t([top, 0]), t([top, 3]), table, t([7, 8]), page_size=16, n_tok=8)
    assert got[3].tolist() == [top, 3] and got[2].tolist() == [0, 8, 8]
    assert got[0].tolist() == [-1] * 8 and got[4].tolist() == [1, top]
    assert table.tolist() == [[-1, -1], [7, -1]]


def test_layout_repeated_call_and_unaligned_outputs(dev):
    import ctypes

    import torch
    from paper_2608_02244_amd import step
    old, new = [10, 0, 33], [9, 40, 2]
    t = [torch.tensor(x, dtype=torch.int32, device=dev) for x in (old, new)]
    free = torch.arange(50, 60, dtype=torch.int32, device=dev)
    table = torch.full((3, 5), -1, dtype=torch.int32, device=dev)
    table[0, 0], table[2, :3] = 1, torch.tensor([2, 3, 4], device=dev)
    first = fs.kv_layout(*t, table, free, page_size=16, n_tok=51)
    kept = table.clone()
    again = fs.kv_layout(*t, table, free, page_size=16, n_tok=51)
    assert torch.equal(kept, table) and all(torch.equal(a, b) for a, b in zip(first, again))
    room = torch.full((200,), -7, dtype=torch.int32, device=dev)
    slots, pos = room[1:52], room[101:152]  # 4 bytes off a 16-byte boundary
    p = step.LayoutParams(n_req=3, n_tok=51, page_size=16, table_width=5, n_free=10,
                          flags=fs.F_DEVICE_PTRS | fs.F_SYNC)
    q = torch.empty(4, dtype=torch.int32, device=dev)
    k, u = torch.empty(3, dtype=torch.int32, device=dev), torch.empty(2, dtype=torch.int32,
                                                                      device=dev)
    torch.cuda.synchronize()
    assert fs.lib().fsched_kv_layout(ctypes.byref(p), *[x.data_ptr() for x in (
        t[0], t[1], free, table, slots, pos, q, k, u)], None) == 0
    assert torch.equal(slots, first[0]) and torch.equal(pos, first[1])
    assert room[0] == -7 and room[52] == -7 and room[100] == -7 and room[152] == -7


# ------------------------------------------------------------- qk_norm_rope

def plain_rope(x, w, cos_sin, positions, interleaved, eps):
    """x [n, heads, D] float64 -> normed and rotated."""
    import torch
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    if cos_sin is None:
        return x
    rot = cos_sin.shape[1]
    half = rot // 2
    ok = (positions >= 0) & (positions < cos_sin.shape[0])
    row = cos_sin[positions.clamp(0, cos_sin.shape[0] - 1).long()][:, None, :]
    out = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = row[..., i], row[..., half + i]
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    out[~ok] = 0.0
    return out


ROPE = [  # n_tok, Hq, Hkv, D, rot, interleaved, page, dtype, norm
    (1, 1, 1, 64, 64, False, 16, "bf16", True),
    (3, 32, 8, 128, 128, False, 16, "bf16", True),
    (70, 40, 8, 128, 64, True, 8, "f16", True),
    (129, 12, 4, 256, 256, False, 32, "bf16", True),
    (17, 28, 4, 256, 128, True, 1, "f16", True),
    (501, 64, 8, 64, 32, False, 64, "f16", True),
    (33, 5, 1, 64, 16, False, 16, "bf16", True),
    (33, 7, 3, 128, 16, True, 16, "f16", False),
    (1031, 3, 1, 128, 0, False, 16, "bf16", True),
    (5000, 16, 16, 64, 64, True, 128, "bf16", False),
]


@pytest.mark.parametrize("c", ROPE, ids=lambda c: "-".join(map(str, c)))
def test_rope_against_64_bits(dev, c):
    import torch
    n, Hq, Hkv, D, rot, inter, page, dt, norm = c
    t = dtype_of(dt)
    g = torch.Generator().manual_seed(n)
    n_pages, n_pos, eps = (2 * n) // page + 3, 300, 1e-5
    qkv = (torch.randn(n, Hq + 2 * Hkv, D, generator=g) *
           torch.logspace(-2, 1, n)[:, None, None]).to(t)
    qkv[0, 0] = 0  # a head of zeros: its norm is that of eps alone
    pos = torch.randint(0, n_pos, (n,), generator=g, dtype=torch.int32)
    slots = torch.randperm(n_pages * page, generator=g)[:n].to(torch.int32)
    if n > 2:
        pos[1] = n_pos          # no row of the table: queries zero, nothing stored
        pos[2] = -1
        slots[0] = -1           # padding rows store nothing
    if n > 4:
        slots[3], slots[4] = n_pages * page, 2 ** 31 - 1
    angle = torch.rand(n_pos, rot // 2, generator=g) * 6.3
    cs = torch.cat((angle.cos(), angle.sin()), 1).contiguous() if rot else None
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(t) if norm else None for _ in range(2)]
    kc, vc = (torch.randn(n_pages, Hkv, page, D, generator=g).to(t) for _ in range(2))
    d = [x.to(dev) if x is not None else None for x in (qkv, pos, slots, cs, kc, vc, *w)]
    log(f"qk_norm_rope {c}")
    q = fs.qk_norm_rope(*d, eps=eps, interleaved=inter)
    x = qkv.double()
    known = (pos >= 0) & (pos < n_pos) if rot else torch.ones(n, dtype=torch.bool)
    csd = cs.double() if rot else None
    refq = plain_rope(x[:, :Hq], w[0].double() if norm else None, csd, pos, inter, eps)
    refk = plain_rope(x[:, Hq:Hq + Hkv], w[1].double() if norm else None, csd, pos, inter, eps)

    def near(got, ref):
        size = ref.abs()
        if rot:  # a pair's size
            p = ref[..., :rot]
            p = p.unflatten(-1, (rot // 2, 2)) if inter else p.unflatten(-1, (2, rot // 2))
            m = p.abs().amax(-1 if inter else -2, keepdim=True).expand(p.shape).flatten(-2)
            size = torch.cat((m, size[..., rot:]), -1)
        tiny = 2.0 ** -25 if dt == "f16" else 0.0  # half the spacing of f16's smallest values
        tol = U[dt] * ref.abs() + 2.0 ** -20 * size + tiny
        assert ((got.double().cpu() - ref).abs() <= tol).all()
    near(q, refq)
    ok = known & (slots >= 0) & (slots < n_pages * page)
    at = slots[ok].long()
    for cache, dev_cache, rows, exact in ((kc, d[4], refk, False), (vc, d[5], x[:, Hq + Hkv:], True)):
        got = dev_cache.cpu()
        flat = got.transpose(1, 2).reshape(-1, Hkv, D)
        if exact or not (norm or rot):
            assert torch.equal(flat[at].double(), rows[ok])
        else:
            near(flat[at], rows[ok])
        rest = torch.ones(n_pages * page, dtype=torch.bool)
        rest[at] = False
        assert torch.equal(flat[rest], cache.transpose(1, 2).reshape(-1, Hkv, D)[rest])


def test_rope_strided_permuted_and_in_place(dev):
    """The projection inside wider rows, a cache with slots before heads, queries
    written over themselves, and no slots at all: the same bits."""
    import torch
    g = torch.Generator(device=dev).manual_seed(5)
    n, Hq, Hkv, D, page = 77, 8, 2, 128, 16
    wide = torch.randn(n, Hq + 2 * Hkv + 3, D, device=dev, generator=g).bfloat16()
    qkv = wide[:, :Hq + 2 * Hkv]
    pos = torch.randint(0, 500, (n,), device=dev, generator=g, dtype=torch.int32)
    slots = torch.randperm(160, device=dev, generator=g)[:n].to(torch.int32)
    ang = torch.rand(500, D // 2, device=dev, generator=g)
    cs = torch.cat((ang.cos(), ang.sin()), 1).contiguous()
    w = torch.ones(D, device=dev).bfloat16()
    a = [torch.zeros(10, Hkv, page, D, device=dev).bfloat16() for _ in range(2)]
    b = [torch.zeros(10, page, Hkv, D, device=dev).bfloat16().transpose(1, 2) for _ in range(2)]
    q0 = fs.qk_norm_rope(qkv.contiguous(), pos, slots, cs, *a, w, w)
    q1 = fs.qk_norm_rope(qkv, pos, slots, cs, *b, w, w)
    assert torch.equal(q0, q1) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c = [torch.zeros_like(x) for x in a]
    assert torch.equal(fs.qk_norm_rope(qkv, pos, None, cs, *c, w, w), q0)
    assert not c[0].any() and not c[1].any()
    keep = wide.clone()
    fs.qk_norm_rope(qkv, pos, None, cs, *c, w, w, out=qkv[:, :Hq])
    assert torch.equal(wide[:, :Hq], q0) and torch.equal(wide[:, Hq:], keep[:, Hq:])


# ------------------------------------------------------------------ attention

class Batch:
    """A ragged batch with its own pages in a shuffled cache; NaN wherever no token
    of a request has been written or can be seen."""

    def __init__(self, dev, new, own, Hq, Hkv, D, dt="bf16", page=16, window=0, sinks=0, prefix=0,
                 seed=0, order="hs", evict=True, spread=2.0):
        import torch
        self.__dict__.update(new=new, own=own, Hq=Hq, Hkv=Hkv, D=D, dt=dt, page=page,
                             window=window, sinks=sinks, prefix=prefix)
        g = torch.Generator().manual_seed(seed)
        t = dtype_of(dt)
        need = [-(-k // page) for k in own]
        width = max(need + [0]) + 1
        total = sum(need) + -(-prefix // page)
        n_pages = total + 3
        ids = torch.randperm(n_pages, generator=g).to(torch.int32)
        shape = (n_pages, Hkv, page, D)
        k, v = (torch.randn(shape, generator=g).to(t) for _ in range(2))
        held = torch.zeros(n_pages, page, dtype=torch.bool)
        table = torch.full((len(own), width), -1, dtype=torch.int32)
        at = 0
        for r, m in enumerate(need):
            lo = prefix + own[r] - new[r] - window + 1 if window else 0
            for c in range(m):
                page_id = ids[at]
                at += 1
                first, last = prefix + c * page, prefix + (c + 1) * page - 1
                if evict and window and last < lo and first >= sinks:
                    continue  # given back
                table[r, c] = page_id
                for i in range(page):
                    p = first + i
                    seen = c * page + i < own[r] and (p >= lo or p < sinks)
                    held[page_id, i] = seen
        self.prefix_pages = ids[at:total].clone()
        for j in range(prefix):
            held[self.prefix_pages[j // page], j % page] = True
        for x in (k, v):
            x.masked_fill_(~held[:, None, :, None], math.nan)
        self.q = (spread * torch.randn(max(1, sum(new)), Hq, D, generator=g)).to(t)[:sum(new)]
        starts = [0]
        for m in new:
            starts.append(starts[-1] + m)
        self.k, self.v, self.table = k, v, table
        self.q_start = torch.tensor(starts, dtype=torch.int32)
        self.kv_len = torch.tensor(own, dtype=torch.int32)
        self.scale = D ** -0.5
        self.dev = dev

        def put(x):
            x = x.to(dev)
            return x.transpose(1, 2).contiguous().transpose(1, 2) if order == "sh" else x
        self.args = [self.q.to(dev), put(k), put(v), table.to(dev), self.q_start.to(dev),
                     self.kv_len.to(dev)]
        self.kw = dict(scale=self.scale, window=window, n_sink=sinks, return_lse=True,
                       max_q=max(new + [1]))

    def call(self, **kw):
        kw = {**self.kw, **kw}
        if self.prefix:
            return fs.attend_shared(*self.args[:3], self.prefix_pages.to(self.dev), self.prefix,
                                    *self.args[3:], **kw)
        return fs.attend(*self.args, **kw)

    def reference(self):
        """(out, lse, tolerance of out, tolerance of lse), float64, row by row."""
        import torch
        n, Hq, D, grp, page = len(self.q), self.Hq, self.D, self.Hq // self.Hkv, self.page
        out = torch.zeros(n, Hq, D, dtype=torch.float64)
        lse = torch.full((n, Hq), -math.inf, dtype=torch.float64)
        tol, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
        n_pages = self.k.shape[0]
        for r, own in enumerate(self.own):
            a, b = int(self.q_start[r]), int(self.q_start[r + 1])
            if a == b:
                continue
            places = [(int(self.prefix_pages[j // page]), j % page) for j in range(self.prefix)]
            places += [(int(self.table[r, j // page]), j % page) for j in range(own)]
            pos = [j for j, (pg, _) in enumerate(places) if 0 <= pg < n_pages]
            pgs = torch.tensor([places[j][0] for j in pos], dtype=torch.long)
            offs = torch.tensor([places[j][1] for j in pos], dtype=torch.long)
            K = self.k.double()[pgs, :, offs].transpose(0, 1) if pos else None  # [Hkv, keys, D]
            V = self.v.double()[pgs, :, offs].transpose(0, 1) if pos else None
            j = torch.tensor(pos, dtype=torch.long)
            for i in range(b - a):
                p = self.prefix + own - (b - a) + i
                see = (j <= p)
                if self.window:
                    see = see & ((j > p - self.window) | (j < self.sinks))
                if not pos or not see.any():
                    continue
                for h in range(Hq):
                    x = self.q[a + i, h].double()
                    kk, vv = K[h // grp][see], V[h // grp][see]
                    s = kk @ x * self.scale
                    lse[a + i, h] = torch.logsumexp(s, 0)
                    w = torch.softmax(s, 0)
                    out[a + i, h] = w @ vv
                    A = w @ vv.abs()
                    tol[a + i, h] = 1.1 * U[self.dt] * (A + out[a + i, h].abs()) + \
                        2.0 ** -19 * (1 + A)
                    err = (D + 8) * 2.0 ** -24 * float((kk.abs() @ x.abs()).max()) * self.scale
                    tol_l[a + i, h] = err + 2.0 ** -20 + 2.0 ** -22 * abs(float(lse[a + i, h]))
        return out, lse, tol, tol_l

    def check(self, **kw):
        import torch
        log(f"attend new={self.new[:6]} own={self.own[:6]} n={len(self.own)} heads={self.Hq}/"
            f"{self.Hkv} D={self.D} {self.dt} page={self.page} window={self.window}/{self.sinks} "
            f"prefix={self.prefix}")
        out, lse = self.call(**kw)
        out, lse = out.double().cpu(), lse.double().cpu()
        ro, rl, to, tl = self.reference()
        empty = rl == -math.inf
        assert (out[empty] == 0).all() and (lse[empty] == -math.inf).all()
        assert torch.isfinite(out).all()
        assert ((out - ro).abs() <= to).all(), ((out - ro).abs() - to).max()
        fine = ~empty
        assert ((lse - rl).abs()[fine] <= tl[fine]).all()


HEADS = [(1, 1), (8, 1), (32, 8), (5, 5), (40, 8), (28, 4), (12, 4), (64, 8), (64, 1), (33, 3)]


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}")
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_attend_decode_heads(dev, heads, dt):
    Batch(dev, [1] * 5, [1, 17, 64, 200, 3], *heads, 64, dt).check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("page", [1, 2, 8, 16, 32, 128])
def test_attend_decode_pages(dev, D, page):
    own = [1, 2, page, page + 1, 31, 32, 33, 127, 128, 129, 0, 450]
    Batch(dev, [1] * 10 + [0, 1], own, 8, 2, D, page=page, seed=page).check()


def test_attend_decode_rows_that_see_nothing(dev):
    import torch
    b = Batch(dev, [1, 1, 2, 0, 3], [0, 5, 1, 0, 0], 8, 2, 64)
    b.check()  # requests that hold nothing, or fewer tokens than they bring
    b = Batch(dev, [1, 1, 1], [40, 40, 40], 8, 2, 64)
    b.table[0, :] = -1                       # every page gone
    b.table[1, 1] = 2 ** 31 - 1              # an id outside the cache
    b.table[2, 0] = b.k.shape[0]
    b.args[3] = b.table.to(dev)
    b.check()
    b = Batch(dev, [1, 1], [20, 30], 8, 2, 64)
    b.own = [20, 48]                         # longer than the row of the block table
    b.args[5] = torch.tensor([20, 10 ** 9], dtype=torch.int32, device=dev)
    b.table[1, 2] = -1
    b.args[3] = b.table.to(dev)
    b.v[b.table[1, 1], :, 14:] = 0.5
    b.k[b.table[1, 1], :, 14:] = 0.5
    b.args[1], b.args[2] = b.k.to(dev), b.v.to(dev)
    b.check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (16, 4), (33, 40), (64, 0),
                                          (100, 1), (1000, 8), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_attend_window(dev, window, sinks):
    own = [1, 5, 16, 17, 40, 64, 99, 100, 101, 300, 0, 700]
    new = [1] * 10 + [0, 1]
    Batch(dev, new, own, 8, 2, 64, page=8, window=window, sinks=sinks, seed=window % 97).check()
    new = [1, 4, 3, 17, 2, 30, 1, 1, 50, 7, 0, 80]
    Batch(dev, new, own, 8, 2, 64, page=8, window=window, sinks=sinks, seed=window % 89).check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("heads", [(4, 4), (8, 1), (10, 2)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_attend_few_and_many_new_tokens(dev, D, heads):
    """Drafts, whole prompts, chunks behind a held part, decoding requests among them."""
    for new, own in (([2, 3, 4, 1], [2, 50, 4, 9]), ([70, 1, 33], [70, 300, 65]),
                     ([128, 1, 2, 0, 65], [128, 9, 40, 3, 200]), ([1, 190], [1, 255])):
        Batch(dev, new, own, *heads, D, page=16, seed=sum(new)).check()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_attend_long_prompt(dev, dt):
    Batch(dev, [520], [520], 2, 1, 128, dt, page=64).check()
    Batch(dev, [300], [900], 2, 2, 64, dt, page=4, window=70, sinks=3).check()


@pytest.mark.parametrize("D,page,own", [(128, 16, [20000]), (64, 8, [9001, 1]),
                                        (256, 64, [12000])])
def test_attend_decode_one_long_request(dev, D, page, own):
    """One request's keys spread over the device, in hundreds of parts."""
    Batch(dev, [1] * len(own), own, 4, 1, D, page=page).check()


@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 100, 640])
@pytest.mark.parametrize("mode", ["decode", "draft", "chunk"])
def test_shared_prefix(dev, prefix, mode):
    own = [1, 16, 17, 40, 90, 6, 0, 129]
    new = {"decode": [1] * 6 + [0, 1], "draft": [1, 2, 3, 4, 1, 2, 0, 4],
           "chunk": [1, 16, 5, 33, 60, 6, 0, 70]}[mode]
    Batch(dev, new, own, 8, 2, 64, prefix=prefix, seed=prefix).check()
    Batch(dev, new, own, 12, 4, 128, "f16", page=8, prefix=prefix, seed=prefix).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (8, 3), (50, 0), (90, 200), (400, 20)])
def test_shared_prefix_behind_a_window(dev, window, sinks):
    for new in ([1, 1, 1, 1], [1, 40, 2, 70]):
        Batch(dev, new, [1, 60, 30, 100], 8, 2, 64, prefix=130, window=window, sinks=sinks,
              seed=window).check()


def test_shared_prefix_many_rows_and_one_request(dev):
    Batch(dev, [1] * 75, [1 + 3 * i % 50 for i in range(75)], 16, 2, 64, prefix=300).check()
    Batch(dev, [1], [5], 8, 1, 256, prefix=1000).check()
    Batch(dev, [1, 3], [0, 2], 8, 2, 128, prefix=40).check()  # fewer own tokens than new ones


@pytest.mark.parametrize("n,heads,D", [(300, (8, 8), 64), (170, (16, 16), 128)])
def test_shared_prefix_more_requests_than_waves(dev, n, heads, D):
    """Own parts so short and many that a wave works on several requests in a row."""
    Batch(dev, [1] * n, [1 + 7 * i % 39 for i in range(n)], *heads, D, prefix=33, seed=n).check()
    Batch(dev, [1 + i % 2 for i in range(n)], [2 + 11 * i % 71 for i in range(n)], *heads, D,
          prefix=18, seed=n).check()


def test_attend_peaked_and_flat_scores(dev):
    """Scores whose weights span the type's range, both ways."""
    for spread in (0.0, 0.01, 30.0):
        Batch(dev, [1, 1, 40], [600, 31, 100], 4, 2, 128, spread=spread).check()
        Batch(dev, [1, 1, 40], [600, 31, 100], 4, 2, 128, "f16", spread=spread).check()


def test_attend_cache_order_strides_and_given_outputs(dev):
    """Slots before heads in memory, queries and outputs inside wider rows: the same bits."""
    import torch
    for new, own in (([1, 1, 1], [70, 5, 33]), ([40, 1, 20], [70, 5, 33])):
        a = Batch(dev, new, own, 8, 2, 128)
        b = Batch(dev, new, own, 8, 2, 128, order="sh")
        out, lse = a.call()
        n = len(a.q)
        wide = torch.zeros(n, 8, 384, device=dev, dtype=out.dtype)
        wide[:, :, 128:256] = a.args[0]
        b.args[0] = wide[:, :, 128:256]
        room = torch.full((n, 11, 256), 7.0, device=dev, dtype=out.dtype)
        got = room[:, 1:9, 64:192]
        out2, lse2 = b.call(out=got)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        room[:, 1:9, 64:192] = 7.0
        assert (room == 7.0).all()


def test_attend_rows_past_max_q_stay(dev):
    import torch
    b = Batch(dev, [1, 3, 1], [20, 30, 5], 8, 2, 64)
    out, lse = b.call()
    mark = torch.full_like(out, 5.0)
    got, _ = b.call(out=mark, max_q=1)
    keep = torch.tensor([0, 1, 4], device=dev)
    assert (got[2:4] == 5.0).all()
    del lse, keep
    # the request's tokens keep their positions: its first token is the same row
    assert torch.allclose(got[1].float(), out[1].float(), atol=0.05)


def test_attend_tokens_of_no_request_stay(dev):
    import torch
    b = Batch(dev, [2, 3], [20, 30], 8, 2, 64)
    out, _ = b.call()
    q = torch.cat((b.args[0], b.args[0]))
    b.args[0] = q
    mark = torch.full_like(q, 5.0)
    got, _ = b.call(out=mark)
    assert torch.equal(got[:5], out) and (got[5:] == 5.0).all()
    # starts that are not in order stay within q
    b.args[4] = torch.tensor([7, 2, 10 ** 6], dtype=torch.int32, device=dev)
    b.call()
    torch.cuda.synchronize()


def test_attend_other_stream_workspace_and_equal_bits(dev):
    import torch
    b = Batch(dev, [1] * 20 + [50, 1], [37 * i % 900 + 1 for i in range(20)] + [800, 3], 16, 2, 128)
    out, lse = b.call()
    ws = fs.attend_workspace(len(b.q), len(b.own), 16, 2, 128, page_size=16,
                             table_width=b.table.shape[1], max_q=50)
    ws.fill_(255)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            o2, l2 = b.call(workspace=ws)
            assert torch.equal(out, o2) and torch.equal(lse, l2)
    torch.cuda.current_stream().wait_stream(s)
    with pytest.raises(fs.FschedError) as e:
        if ws.numel() > 256:
            b.call(workspace=ws[:256])
        else:
            raise fs.FschedError(fs.ESCRATCH, "no workspace is needed")
    assert e.value.code == fs.ESCRATCH


def test_attend_offsets_past_32_bits(dev):
    """A page whose elements lie beyond 2^32: pages 2^31 elements apart."""
    import torch
    free, _ = torch.cuda.mem_get_info()
    step = 1 << 31
    if free < (3 * step) * 2 + (1 << 30):
        pytest.skip("not enough free memory")
    b = Batch(dev, [1, 1, 40], [16, 12, 44], 4, 2, 64, page=16)
    n = b.k.shape[0]
    assert n >= 6
    room = torch.empty(2 * step + (1 << 20), dtype=torch.bfloat16, device=dev)
    half = n // 2

    def far(x, shift):  # page p at p * (2 * step // (n - 1)) elements
        gap = (2 * step // (n - 1)) // 8 * 8
        view = room.as_strided(x.shape, (gap, 16 * 64, 64, 1), shift)
        view.copy_(x)
        return view
    b.args[1] = far(b.k.to(dev), 0)
    b.args[2] = far(b.v.to(dev), 8192)
    assert half and b.args[1].stride(0) * (n - 1) > 2 ** 31
    b.check()
    slots = torch.tensor([(n - 1) * 16 + 3], dtype=torch.int32, device=dev)
    qkv = torch.randn(1, 8, 64, device=dev).bfloat16()
    fs.qk_norm_rope(qkv, None, slots, None, b.args[1], b.args[2])
    assert torch.equal(b.args[1][n - 1, :, 3], qkv[0, 4:6])
    assert torch.equal(b.args[2][n - 1, :, 3], qkv[0, 6:8])


def test_step_in_a_captured_graph(dev):
    """Placement, store and attention in one graph with a workspace, replayed with other
    inputs between eager work: every replay equals the eager calls."""
    import torch
    n, Hq, Hkv, D, page, width = 9, 8, 2, 64, 16, 12
    g = torch.Generator(device=dev).manual_seed(3)
    kc, vc = (torch.randn(n * width, Hkv, page, D, device=dev, generator=g).bfloat16()
              for _ in range(2))
    table = torch.arange(n * width, device=dev, dtype=torch.int32).view(n, width).contiguous()
    free = torch.arange(4, device=dev, dtype=torch.int32)
    old = torch.zeros(n, device=dev, dtype=torch.int32)
    new = torch.ones(n, device=dev, dtype=torch.int32)
    qkv = torch.randn(n, Hq + 2 * Hkv, D, device=dev, generator=g).bfloat16()
    ang = torch.rand(200, D // 2, device=dev, generator=g)
    cs = torch.cat((ang.cos(), ang.sin()), 1).contiguous()
    w = torch.ones(D, device=dev).bfloat16()
    ws = fs.attend_workspace(n, n, Hq, Hkv, D, page_size=page, table_width=width, max_q=1)

    def one():
        slots, pos, q_start, kv_len, _ = fs.kv_layout(old, new, table, free, page_size=page,
                                                      n_tok=n)
        q = fs.qk_norm_rope(qkv, pos, slots, cs, kc, vc, w, w)
        return fs.attend(q, kc, vc, table, q_start, kv_len, max_q=1, workspace=ws,
                         return_lse=True)
    old.fill_(31)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        one()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = one()
    for turn, at in enumerate((33, 100, 17, 150)):
        old.fill_(at)
        old[turn] = 3
        qkv.copy_(torch.randn(qkv.shape, device=dev, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        a = [x.clone() for x in got]
        b = one()
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_given_stream_runs_there_and_owns_its_outputs(dev):
    import torch
    b = Batch(dev, [1, 40, 1], [70, 90, 33], 8, 2, 64)
    out, lse = b.call()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, got_lse = b.call(stream=s)
    s.synchronize()
    assert torch.equal(out, got) and torch.equal(lse, got_lse)
    at = got.data_ptr()
    del got
    with torch.cuda.stream(s):  # its memory went back to the stream that it was made for
        assert torch.empty_like(out).data_ptr() == at
    lens = torch.tensor([1, 2], dtype=torch.int32, device=dev)
    table = torch.full((2, 3), -1, dtype=torch.int32, device=dev)
    free = torch.arange(6, dtype=torch.int32, device=dev)
    s.wait_stream(torch.cuda.current_stream())
    got = fs.kv_layout(lens * 0, lens, table, free, page_size=16, n_tok=3, stream=s)
    s.synchronize()
    assert got[0].tolist() == [0, 16, 17] and got[3].tolist() == [1, 2]


@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 2)])
def test_replay_of_a_schedule(dev, window, sinks):
    """An ISJL schedule played on the operators: every request's every token attends over
    exactly the request's own tokens, whatever pages they went to.  The reference keeps
    queries and keys in 64 bits; their rounding to f16 moves a score by at most
    d = (2 u + u^2) scale sum |q k|, and the output by (exp(2 d) - 1) A beside its own
    rounding."""
    import numpy as np
    import torch
    from paper_2608_02244_amd import replay
    rng = np.random.default_rng(5)
    n, Hq, Hkv, D, page, layers, u = 12, 4, 2, 64, 4, 2, U["f16"]
    a, p, o = (rng.integers(lo, hi, (1, n)).astype(np.int32)
               for lo, hi in ((0, 20), (1, 20), (1, 30)))
    _, start, finish = fs.simulate(a, p, o, policy="isjl", B=4, alpha=8, M_kv=160, cost_c=0,
                                   cost_tau=0, schedule=True)
    length = (p + o)[0].tolist()
    g = torch.Generator().manual_seed(9)
    x = torch.randn(layers, n, max(length), Hq + 2 * Hkv, D, generator=g).half()
    xd = x.to(dev)
    w = replay.Worker(n_pages=160 // page + n, page_size=page, q_heads=Hq, kv_heads=Hkv,
                      head_dim=D, max_len=max(length), layers=layers, window=window,
                      n_sink=sinks, dtype=torch.float16, device=dev)
    pages = len(w.free)
    got = torch.zeros(layers, n, max(length), Hq, D, dtype=torch.float64)
    seen = [0] * n

    def on_step(t, now, outs):
        for i, r in enumerate(now):
            for layer, y in enumerate(outs):
                got[layer, r, seen[r]] = y[i].double().cpu()
            seen[r] += 1
    replay.play(w, start[0], finish[0],
                lambda layer, now, at: torch.stack([xd[layer, r, i] for r, i in zip(now, at)]),
                on_step)
    assert seen == length
    assert sorted(w.free.tolist()) == list(range(pages))  # every page came back, once
    y = x.double()
    y[..., :Hq + Hkv, :] /= (y[..., :Hq + Hkv, :].square().mean(-1, keepdim=True) + 1e-6).sqrt()
    cs = w.cos_sin.double().cpu()[:max(length), None, :]
    c, s = cs[..., :D // 2], cs[..., D // 2:]
    f, e = y[..., :Hq + Hkv, :D // 2].clone(), y[..., :Hq + Hkv, D // 2:].clone()
    y[..., :Hq + Hkv, :D // 2], y[..., :Hq + Hkv, D // 2:] = f * c - e * s, e * c + f * s
    for layer in range(layers):
        for r in range(n):
            for h in range(Hq):
                z = y[layer, r, :length[r]]
                q, k, v = z[:, h], z[:, Hq + h // 2], z[:, Hq + Hkv + h // 2]
                i = torch.arange(length[r])
                hide = i[None, :] > i[:, None]
                if window:
                    hide |= (i[None, :] <= i[:, None] - window) & (i[None, :] >= sinks)
                wt = torch.softmax((q @ k.t() * D ** -0.5).masked_fill(hide, -math.inf), 1)
                ref, A = wt @ v, wt @ v.abs()
                d = (2 * u + u * u) * D ** -0.5 * (q.abs() @ k.abs().t()).amax(1, keepdim=True)
                tol = (torch.exp(2 * d) - 1) * A + 1.1 * u * (A + ref.abs()) + 2.0 ** -18 * (1 + A)
                assert ((got[layer, r, :length[r], h] - ref).abs() <= tol).all()
