"""The operators of a KV cache within a budget on the GPU against plain implementations in
64 bits: the cache of 4 bits (store, read, attention), the attention weight of held tokens,
and pages given up by it.

What is stored in 4 bits has to be equal byte for byte (keys are computed in 64 bits before
they are rounded, values are rounded as they are).  Tolerances are fixed before any run:
  attention   as over a 16-bit cache, the held values being elements of the type;
  weights     of a sum of n terms exp(s - lse):  w (e + 2^-22 (|s| + |lse|) + (n + 8) 2^-24)
              + 2^-23 |weight|, with e = (D + 8) 2^-24 scale sum_d |q_d k_d| for the 32-bit
              scores, the second term for the exponential's argument and itself, the third
              for the sum, the last for the addition to what was there;
  evictions   whole numbers and moved numbers have to be equal."""
import math
import random

import pytest

import paper_2608_02244_amd as fs
from test_gpu_step_operators import Batch, HEADS, ROPE, U, dev, dtype_of, log, plain_rope  # noqa: F401

pytestmark = pytest.mark.gpu

EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ the format

def quantise(x, dt):
    """x [..., D] float64 -> codes and scale bytes, by the distance to every level."""
    import torch
    lo, hi = EXPONENTS[dt]
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(b).all(-1, keepdim=True)
    top = torch.where(bad, 1.0, top)
    m, e = torch.frexp(top)
    e = torch.where(m <= 0.75, e - 3, e - 2)  # top <= 6 * 2^e
    e = torch.where(top > 0, e, lo).clamp(lo, hi)
    y = torch.ldexp(torch.where(bad, 0.0, b.abs()), -e)
    d = torch.stack([(y - v).abs() for v in LEVELS], -1)
    least = d.amin(-1, keepdim=True)
    # of two equally near levels the one of even place
    odd = torch.arange(8) % 2
    code = torch.where(d == least, odd.double(), 9.0).argmin(-1)
    code = torch.where(torch.signbit(b) & ~bad, code + 8, code)
    return code.flatten(-2), torch.where(bad, 255, e + 127).squeeze(-1).long()


def values(code, scale):
    """float64 that codes [..., D] and scale bytes [..., D / 32] stand for."""
    import torch
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64)
    s = torch.where(scale == 255, math.nan, torch.ldexp(torch.ones(()).double(), scale - 127))
    return (level[code].unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def packed(kcode, kscale, vcode, vscale):
    """Bytes [pages, heads, page / 16, 17 D] of codes [pages, heads, page, D] and scales,
    token by token."""
    import torch
    P, H, page, D = kcode.shape
    out = torch.zeros(P, H, page // 16, 17 * D, dtype=torch.uint8)
    for t in range(page):
        g, i = t // 16, t % 16
        for code, first in ((kcode, 0), (vcode, 8 * D)):
            b = (code[:, :, t, 0::2] + 16 * code[:, :, t, 1::2]).to(torch.uint8)
            if first == 0:
                out[:, :, g, i * D // 2:(i + 1) * D // 2] = b
            else:
                w = D // 32
                for n in range(16):
                    at = first + ((i // 4 * 16 + n) * 4 + i % 4) * w
                    out[:, :, g, at:at + w] = b[..., n * w:(n + 1) * w]
        for j in range(D // 32):
            out[:, :, g, 16 * D + i * (D // 32) + j] = kscale[:, :, t, j].to(torch.uint8)
            out[:, :, g, 16 * D + D // 2 + (i // 4 * (D // 32) + j) * 4 + i % 4] = \
                vscale[:, :, t, j].to(torch.uint8)
    return out


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_read_every_code_and_scale(dev, D, dt):
    """Codes and scales at random, all scales of the type and the one of NaN."""
    import torch
    g = torch.Generator().manual_seed(D)
    lo, hi = EXPONENTS[dt]
    P, H, page = 9, 3, 32
    code = [torch.randint(0, 16, (P, H, page, D), generator=g) for _ in range(2)]
    scale = [torch.randint(lo + 127, hi + 128, (P, H, page, D // 32), generator=g)
             for _ in range(2)]
    for s in scale:
        s[0, 0, 0, 0] = 255
        s[0, 0, 1, 0], s[0, 0, 2, 0] = lo + 127, hi + 127
    cache = packed(code[0], scale[0], code[1], scale[1]).to(dev)
    slots = torch.randperm(P * page, generator=g).to(torch.int32)
    slots[5], slots[6], slots[7] = -1, P * page, 2 ** 31 - 1
    log(f"kv4_read D={D} {dt}")
    got = fs.kv4_read(cache, slots.to(dev), dtype=dtype_of(dt))
    ok = (slots >= 0) & (slots < P * page)
    at = slots.clamp(0, P * page - 1).long()
    for x, c, s in zip(got, code, scale):
        ref = values(c, s)[at // page, :, at % page]
        ref[~ok] = 0.0
        x = x.double().cpu()
        assert torch.equal(torch.isnan(x), torch.isnan(ref))
        assert torch.equal(x.nan_to_num(7.0), ref.nan_to_num(7.0))


# ------------------------------------------------------------------- the store

STORE = [(*c[:6], max(16, c[6]), *c[7:]) for c in ROPE]


def store_case(dev, c, seed=None):
    import torch
    n, Hq, Hkv, D, rot, inter, page, dt, norm = c
    t = dtype_of(dt)
    g = torch.Generator().manual_seed(n if seed is None else seed)
    n_pages, n_pos = (2 * n) // page + 3, 300
    qkv = (torch.randn(n, Hq + 2 * Hkv, D, generator=g) *
           torch.logspace(-2, 1, n)[:, None, None]).to(t)
    pos = torch.randint(0, n_pos, (n,), generator=g, dtype=torch.int32)
    slots = torch.randperm(n_pages * page, generator=g)[:n].to(torch.int32)
    if n > 2:
        pos[1], pos[2], slots[0] = n_pos, -1, -1
    if n > 4:
        slots[3], slots[4] = n_pages * page, 2 ** 31 - 1
    angle = torch.rand(n_pos, rot // 2, generator=g) * 6.3
    cs = torch.cat((angle.cos(), angle.sin()), 1).contiguous() if rot else None
    w = [(1 + 0.3 * torch.randn(D, generator=g)).to(t) if norm else None for _ in range(2)]
    cache = torch.randint(0, 256, (n_pages, Hkv, page // 16, 17 * D), generator=g).to(torch.uint8)
    return qkv, pos, slots, cs, cache, w


@pytest.mark.parametrize("c", STORE, ids=lambda c: "-".join(map(str, c)))
def test_store_byte_for_byte(dev, c):
    import torch
    n, Hq, Hkv, D, rot, inter, page, dt, norm = c
    eps = 2.0 ** -17  # a 32-bit number: the oracle has the same
    qkv, pos, slots, cs, cache, w = store_case(dev, c)
    d = [x.to(dev) if x is not None else None for x in (qkv, pos, slots, cs, cache, *w)]
    log(f"qk_norm_rope4 {c}")
    q = fs.qk_norm_rope4(*d, eps=eps, interleaved=inter)
    # queries as with a 16-bit cache, bit for bit
    kv = [torch.zeros(cache.shape[0], Hkv, page, D, device=dev, dtype=qkv.dtype) for _ in range(2)]
    assert torch.equal(q, fs.qk_norm_rope(*d[:4], *kv, *d[5:], eps=eps, interleaved=inter))
    x = qkv.double()
    known = (pos >= 0) & (pos < 300) if rot else torch.ones(n, dtype=torch.bool)
    k = plain_rope(x[:, Hq:Hq + Hkv], w[1].double() if norm else None,
                   cs.double() if rot else None, pos, inter, eps)
    ok = known & (slots >= 0) & (slots < cache.shape[0] * page)
    at = slots[ok].long()
    code, scale = ([torch.zeros(cache.shape[0], Hkv, page, m, dtype=torch.long) for _ in range(2)]
                   for m in (D, D // 32))
    for i, y in enumerate((k, x[:, Hq + Hkv:])):
        a, b = quantise(y[ok], dt)
        code[i][at // page, :, at % page], scale[i][at // page, :, at % page] = a, b
    ref = packed(code[0], scale[0], code[1], scale[1])
    # bytes that hold no stored token stay as they were
    mine = torch.zeros_like(scale[0][..., :1])
    mine[at // page, :, at % page] = 255
    mask = packed(*[(mine // 17).expand(-1, -1, -1, D), mine.expand(-1, -1, -1, D // 32)] * 2)
    ref = torch.where(mask == 255, ref, cache)
    assert torch.equal(d[4].cpu(), ref)
    got = fs.kv4_read(d[4], d[2], dtype=qkv.dtype)
    for i in range(2):
        assert torch.equal(got[i][ok.to(dev)].double().cpu(),
                           values(code[i], scale[i])[at // page, :, at % page])


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_store_extreme_values(dev, dt):
    """Zeros, the type's least and largest numbers, ties, NaN and infinities."""
    import torch
    t, D = dtype_of(dt), 64
    info = torch.finfo(t)
    rows = [[0.0] * 32, [-0.0] * 32, [info.max] * 32, [info.max, -info.max] + [1.0] * 30,
            [info.smallest_normal] * 32, [2.0 ** -24 if dt == "f16" else 2.0 ** -133] * 32,
            [6.0, 0.25, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0, 0.26, 0.74] + [0.0] * 20,
            [1.0, math.nan] + [0.0] * 30, [math.inf] + [1.0] * 31, [-math.inf] + [1.0] * 31,
            [12.0] + [12 * 2.0 ** -i for i in range(31)], [3.0] * 32, [6.03125] * 32, [49152.0] * 32,
            [50000.0] * 32]
    x = torch.tensor(rows, dtype=torch.float64).to(t)
    n = len(rows)
    other = x.flip(0)
    qkv = torch.stack((torch.cat((x, x), 1), torch.cat((x, other), 1), torch.cat((other, x), 1)), 1)
    cache = torch.zeros(2, 1, 1, 17 * D, dtype=torch.uint8, device=dev)
    slots = torch.arange(n, dtype=torch.int32, device=dev)
    log(f"qk_norm_rope4 extremes {dt}")
    fs.qk_norm_rope4(qkv.to(dev), None, slots, None, cache)
    got = fs.kv4_read(cache, slots, dtype=t)
    for i in range(2):
        ref = values(*quantise(qkv[:, 1 + i].double(), dt))
        y = got[i][:, 0].double().cpu()
        assert torch.equal(torch.isnan(y), torch.isnan(ref))
        assert torch.equal(y.nan_to_num(7.0), ref.nan_to_num(7.0))


@pytest.mark.parametrize("page", [16, 64])
def test_store_strided_in_place_and_without_slots(dev, page):
    import torch
    c = (77, 8, 2, 128, 128, False, page, "bf16", True)
    qkv, pos, slots, cs, cache, w = store_case(dev, c)
    d = [x.to(dev) for x in (qkv, pos, slots, cs, cache, *w)]
    a, b = d[4].clone(), d[4].clone().transpose(1, 2).contiguous().transpose(1, 2)
    q = fs.qk_norm_rope4(*d[:4], a, *d[5:])
    wide = torch.zeros(77, 15, 128, device=dev, dtype=qkv.dtype)
    wide[:, :12] = d[0]
    q2 = fs.qk_norm_rope4(wide[:, :12], *d[1:4], b, *d[5:])
    assert torch.equal(q, q2) and torch.equal(a, b) and not torch.equal(a, d[4])
    e = d[4].clone()
    fs.qk_norm_rope4(wide[:, :12], d[1], None, d[3], e, *d[5:], out=wide[:, :8])
    assert torch.equal(wide[:, :8], q) and torch.equal(e, d[4])
    assert torch.equal(fs.kv4_read(a, d[2])[0], fs.kv4_read(b, d[2])[0])


# --------------------------------------------------------------- the attention

class Batch4(Batch):
    """The batch's keys and values in 4 bits; where nothing was written codes at random
    with the scale of NaN."""

    def __init__(self, dev, *args, order="hs", page=16, **kw):
        import torch
        super().__init__(dev, *args, page=page, **kw)
        g = torch.Generator().manual_seed(7)
        parts = []
        for name in ("k", "v"):
            x = getattr(self, name).double()
            code, scale = quantise(x, self.dt)
            setattr(self, name, values(code, scale))
            code = torch.where((scale == 255).repeat_interleave(32, -1),
                               torch.randint(0, 16, code.shape, generator=g), code)
            parts += [code, scale]
        cache = packed(*parts).to(dev)
        self.cache = cache.transpose(1, 2).contiguous().transpose(1, 2) if order == "sh" else cache
        self.lse_kw = {k: v for k, v in self.kw.items() if k != "return_lse"}

    def call(self, **kw):
        kw = {**self.kw, **kw}
        if self.prefix:
            kw.update(prefix_pages=self.prefix_pages.to(self.dev), prefix_len=self.prefix)
        return fs.attend4(self.args[0], self.cache, *self.args[3:], **kw)


@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}")
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_attend4_decode_heads(dev, heads, dt):
    Batch4(dev, [1] * 5, [1, 17, 64, 200, 3], *heads, 64, dt).check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_attend4_decode_pages(dev, D, dt, page):
    own = [1, 2, page, page + 1, 15, 31, 32, 33, 127, 128, 129, 0, 450]
    Batch4(dev, [1] * 11 + [0, 1], own, 8, 2, D, dt, page=page, seed=page).check()
    Batch4(dev, [1, 3, 1], [40, 70, 9], 40, 2, D, dt, page=page, seed=page).check()


def test_attend4_rows_that_see_nothing(dev):
    import torch
    b = Batch4(dev, [1, 1, 2, 0, 3], [0, 5, 1, 0, 0], 8, 2, 64)
    b.check()  # requests that hold nothing, or fewer tokens than they bring
    b = Batch4(dev, [1, 1, 1, 50], [40, 40, 40, 60], 8, 2, 64)
    b.table[0, :] = -1                       # every page gone
    b.table[1, 1] = 2 ** 31 - 1              # an id outside the cache
    b.table[2, 0] = b.k.shape[0]
    b.table[3, 1] = -5
    b.args[3] = b.table.to(dev)
    b.check()
    b = Batch4(dev, [1, 1], [20, 48], 8, 2, 64)
    b.args[5] = torch.tensor([20, 10 ** 9], dtype=torch.int32, device=dev)
    b.table = b.table[:, :3].contiguous()    # lengths past the row count as the row's end
    b.args[3] = b.table.to(dev)
    b.check()
    none = torch.empty(0, 2, 1, 17 * 64, dtype=torch.uint8, device=dev)  # no cache at all
    for new in (1, 40):
        q = torch.ones(new, 8, 64, device=dev, dtype=torch.bfloat16)
        out, lse = fs.attend4(q, none, torch.zeros(1, 4, dtype=torch.int32, device=dev),
                              torch.tensor([0, new], dtype=torch.int32, device=dev),
                              torch.tensor([60], dtype=torch.int32, device=dev), max_q=new,
                              return_lse=True)
        assert not out.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (16, 4), (33, 40), (64, 0),
                                          (100, 1), (1000, 8), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_attend4_window(dev, window, sinks):
    own = [1, 5, 16, 17, 40, 64, 99, 100, 101, 300, 0, 700]
    new = [1] * 10 + [0, 1]
    Batch4(dev, new, own, 8, 2, 64, window=window, sinks=sinks, seed=window % 97).check()
    new = [1, 4, 3, 17, 2, 30, 1, 1, 50, 7, 0, 80]
    Batch4(dev, new, own, 8, 2, 128, window=window, sinks=sinks, seed=window % 89).check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 64])
def test_attend4_short_tables(dev, D, page):
    """Tables of at most 128 keys, and of the next size: few requests and many, drafts."""
    import torch
    own = [1, 0, 16, 17, 33, 64, 48, 2, 31, 50, 60, 5]
    for most in (1, 33, 64, 112, 113, 128):
        Batch4(dev, [1] * 11 + [0], [min(m, most) for m in own] if most <= 64 else own[:-1] + [most],
               8, 2, D, page=page, seed=most).check()
    Batch4(dev, [1, 3, 2], [40, 3, 60], 10, 2, D, page=page).check()
    Batch4(dev, [1] * 12, own, 8, 2, D, page=page, window=20, sinks=3).check()
    b = Batch4(dev, [1] * 900, [i % 60 for i in range(900)], 16, 8, D, page=page)
    b.table[5::7, 0] = -1
    b.args[3] = b.table.to(dev)
    b.check()
    w = fs.attend4_workspace(900, 900, 16, 8, D, page_size=page, table_width=b.table.shape[1],
                             max_q=1)
    assert all(torch.equal(x, y) for x, y in zip(b.call(workspace=w), b.call()))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("heads", [(4, 4), (8, 1), (10, 2)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_attend4_few_and_many_new_tokens(dev, D, heads):
    """Drafts, whole prompts, chunks behind a held part, decoding requests among them."""
    for new, own in (([2, 3, 4, 1], [2, 50, 4, 9]), ([70, 1, 33], [70, 300, 65]),
                     ([128, 1, 2, 0, 65], [128, 9, 40, 3, 200]), ([1, 190], [1, 255])):
        Batch4(dev, new, own, *heads, D, seed=sum(new)).check()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_attend4_long_prompt(dev, dt):
    Batch4(dev, [520], [520], 2, 1, 128, dt, page=64).check()
    Batch4(dev, [300], [900], 2, 2, 64, dt, window=70, sinks=3).check()
    Batch4(dev, [150], [330], 2, 1, 256, dt, page=32).check()


@pytest.mark.parametrize("D,page,own", [(128, 16, [20000]), (64, 32, [9001, 1]),
                                        (256, 64, [12000])])
def test_attend4_decode_one_long_request(dev, D, page, own):
    """One request's keys spread over the device, in hundreds of parts."""
    Batch4(dev, [1] * len(own), own, 4, 1, D, page=page).check()


@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 100, 640])
@pytest.mark.parametrize("mode", ["decode", "draft", "chunk"])
def test_attend4_behind_a_prefix(dev, prefix, mode):
    own = [1, 16, 17, 40, 90, 6, 0, 129]
    new = {"decode": [1] * 6 + [0, 1], "draft": [1, 2, 3, 4, 1, 2, 0, 4],
           "chunk": [1, 16, 5, 33, 60, 6, 0, 70]}[mode]
    Batch4(dev, new, own, 8, 2, 64, prefix=prefix, seed=prefix).check()
    Batch4(dev, new, own, 12, 4, 128, "f16", page=32, prefix=prefix, seed=prefix).check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (50, 0), (90, 200), (400, 20)])
def test_attend4_behind_a_prefix_and_a_window(dev, window, sinks):
    for new in ([1, 1, 1, 1], [1, 40, 2, 70]):
        Batch4(dev, new, [1, 60, 30, 100], 8, 2, 64, prefix=130, window=window, sinks=sinks,
               seed=window).check()
    Batch4(dev, [1, 3], [0, 2], 8, 2, 128, prefix=40).check()  # fewer own tokens than new ones
    Batch4(dev, [1] * 200, [1 + 7 * i % 39 for i in range(200)], 8, 8, 64, prefix=33).check()


def test_attend4_peaked_and_flat_scores(dev):
    for spread in (0.0, 0.01, 30.0):
        for dt in ("bf16", "f16"):
            Batch4(dev, [1, 1, 40], [600, 31, 100], 4, 2, 128, dt, spread=spread).check()


def test_attend4_order_strides_workspace_and_equal_bits(dev):
    import torch
    for new, own in (([1, 1, 1], [70, 5, 33]), ([40, 1, 20], [70, 5, 33])):
        a = Batch4(dev, new, own, 8, 2, 128, page=64)
        b = Batch4(dev, new, own, 8, 2, 128, page=64, order="sh")
        out, lse = a.call()
        n = len(a.q)
        wide = torch.zeros(n, 8, 384, device=dev, dtype=out.dtype)
        wide[:, :, 128:256] = a.args[0]
        b.args[0] = wide[:, :, 128:256]
        room = torch.full((n, 11, 256), 7.0, device=dev, dtype=out.dtype)
        out2, lse2 = b.call(out=room[:, 1:9, 64:192])
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        room[:, 1:9, 64:192] = 7.0
        assert (room == 7.0).all()
        ws = fs.attend4_workspace(n, 3, 8, 2, 128, page_size=64, table_width=a.table.shape[1],
                                  max_q=max(new))
        ws.fill_(255)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            out2, lse2 = a.call(workspace=ws, stream=s)
            s.synchronize()
            assert torch.equal(out, out2) and torch.equal(lse, lse2)
        with pytest.raises(fs.FschedError) as e:
            a.call(workspace=torch.empty(0, dtype=torch.uint8, device=dev))
        assert e.value.code == fs.ESCRATCH


def test_attend4_rows_of_no_request_and_past_max_q_stay(dev):
    import torch
    b = Batch4(dev, [2, 3], [20, 30], 8, 2, 64)
    out, _ = b.call()
    b.args[0] = torch.cat((b.args[0], b.args[0]))
    got, _ = b.call(out=torch.full_like(b.args[0], 5.0))
    assert torch.equal(got[:5], out) and (got[5:] == 5.0).all()
    got, _ = b.call(out=torch.full_like(b.args[0], 5.0), max_q=1)
    assert (got[[1, 3, 4]] == 5.0).all() and (got[[0, 2]] != 5.0).any()
    b.args[4] = torch.tensor([7, 2, 10 ** 6], dtype=torch.int32, device=dev)  # out of order
    b.call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [[1, 1], [3, 60]], ids=["few", "many"])
def test_attend4_not_finite_where_seen(dev, new):
    """A block that stands for NaN makes NaN what it enters: a key's the rows that see it, a
    value's its own elements of their outputs (and, as 0 * NaN, maybe those of other rows of
    the request)."""
    import torch
    b = Batch4(dev, new, [50, 90], 8, 2, 128)
    ref, ref_lse = (x.double().cpu() for x in b.call())
    page, at = b.table[1, 3], 13  # token 61 of request 1
    for side in ("key", "value"):
        cache = b.cache.clone()
        scales = (16 * 128 + at * 4 if side == "key" else 16 * 128 + 64 + at // 4 * 16 + at % 4)
        cache[page, 1, 0, scales + (2 if side == "key" else 8)] = 255  # elements 64 .. 95
        kw = {**b.kw}
        out, lse = (x.double().cpu() for x in fs.attend4(b.args[0], cache, *b.args[3:], **kw))
        bad = torch.zeros_like(ref, dtype=torch.bool)
        sees = [new[0] + i for i in range(new[1]) if 90 - new[1] + i >= 48 + at]
        bad[sees, 4:, (slice(None) if side == "key" else slice(64, 96))] = True
        may = bad.clone()
        if side == "value":
            may[new[0]:, 4:, 64:96] = True
        assert (out.isnan() | ~bad).all() and not (out.isnan() & ~may).any()
        assert torch.equal(out[~may], ref[~may])
        lost = bad.all(-1)
        assert torch.equal(lse.isnan(), lost) and torch.equal(lse[~lost], ref_lse[~lost])


def test_heads_requests_and_pages_at_their_most(dev):
    """1,024 query heads on one and on as many; 4,096 requests; pages behind 2^32 bytes."""
    import torch
    Batch4(dev, [1, 2], [20, 37], 1024, 1, 64).check()
    Batch4(dev, [1, 2], [20, 37], 1024, 1024, 64).check()
    new = [1] * 4094 + [40, 20]
    Batch4(dev, new, [m + i % 5 for i, m in enumerate(new)], 2, 1, 64).check()
    H, page, D, n = 8, 64, 128, 300
    few = fs.kv4_cache(6, H, page, D, device=dev).zero_()
    many = fs.kv4_cache(80000, H, page, D, device=dev)  # 5.6 GB
    g = torch.Generator(device=dev).manual_seed(1)
    qkv = torch.randn(n, 32 + 2 * H, D, device=dev, generator=g).bfloat16()
    pos = torch.arange(n, dtype=torch.int32, device=dev)
    cs = torch.rand(n, D, device=dev, generator=g)
    got = []
    for cache, first in ((few, 0), (many, 80000 - 6)):
        table = torch.arange(first, first + 6, dtype=torch.int32, device=dev).view(1, 6)
        slots = pos + first * page
        q = fs.qk_norm_rope4(qkv, pos, slots, cs, cache)
        out = [q, *fs.kv4_read(cache, slots)]
        for m in (1, n):
            step = (torch.tensor([0, m], dtype=torch.int32, device=dev),
                    torch.tensor([n], dtype=torch.int32, device=dev))
            out += fs.attend4(q[:m], cache, table, *step, return_lse=True)
            weight = torch.zeros(1, 6 * page, device=dev)
            out.append(fs.attend4_weight(q[:m], out[-1], cache, table, *step, weight))
        got.append(out)
    assert all(torch.equal(x, y) for x, y in zip(*got))


# ------------------------------------------------------------------ the weight

def check_weight(b, rows_apart=0, seed=0, change=None):
    """Weights of a batch (of either kind) against 64 bits, and nothing else written.
    `change`: what a caller does with q and lse before the call."""
    import torch
    dev, page, n, Hq, grp = b.dev, b.page, len(b.own), b.Hq, b.Hq // b.Hkv
    log(f"attend_weight {type(b).__name__} new={b.new[:6]} own={b.own[:6]} n={n} heads={Hq}/"
        f"{b.Hkv} D={b.D} {b.dt} page={page} window={b.window}/{b.sinks} prefix={b.prefix}")
    lse = b.reference()[1].float()
    if change:
        change(b.q, lse)
        b.args[0] = b.q.to(dev)
    row = b.table.shape[1] * page
    g = torch.Generator().manual_seed(seed)
    start = torch.rand(n, row + rows_apart, generator=g)
    got = start.to(dev)
    kw = {k: v for k, v in b.kw.items() if k != "return_lse"}
    step = (*b.args[3:], got[:, :row])
    if isinstance(b, Batch4):
        back = fs.attend4_weight(b.args[0], lse.to(dev), b.cache, *step, prefix_len=b.prefix, **kw)
    else:
        back = fs.attend_weight(b.args[0], lse.to(dev), b.args[1], *step, prefix_len=b.prefix, **kw)
    assert back.data_ptr() == got.data_ptr()
    ref, tol = start.double(), 2.0 ** -23 * start.double()
    n_pages = b.k.shape[0]
    for r, own in enumerate(b.own):
        a, e = int(b.q_start[r]), int(b.q_start[r + 1])
        pages = b.table[r, torch.arange(own) // page].long()
        held = (pages >= 0) & (pages < n_pages)
        K = b.k[pages.clamp(0, n_pages - 1), :, torch.arange(own) % page].double().nan_to_num(0.0)
        j = b.prefix + torch.arange(own)
        for i in range(e - a):
            p = b.prefix + own - (e - a) + i
            see = (j <= p) & held
            if b.window:
                see = see & ((j > p - b.window) | (j < b.sinks))
            if not see.any():
                continue
            for h in range(Hq):
                x, kk = b.q[a + i, h].double(), K[:, h // grp]
                s = kk @ x * b.scale
                at = lse[a + i, h].double()
                if at == -math.inf:
                    continue
                if at.isnan():
                    ref[r, :own] = torch.where(see, at, ref[r, :own])
                    continue
                w = torch.where(see, torch.exp(s - at), 0.0)
                ref[r, :own] += w
                size = (kk.abs() @ x.abs()) * b.scale
                tol[r, :own] += w * ((b.D + 8) * 2.0 ** -24 * size +
                                     2.0 ** -22 * (s.abs() + at.abs()) +
                                     ((e - a) * Hq + 8) * 2.0 ** -24) + 2.0 ** -126
    tol += 2.0 ** -23 * ref
    untouched = ref == start.double()
    got = got.double().cpu()
    assert torch.equal(got[untouched], start.double()[untouched])
    assert torch.equal(got.isnan(), ref.isnan())
    got, ref, tol = (x.nan_to_num(0.0) for x in (got, ref, tol))
    assert ((got - ref).abs() <= tol).all(), ((got - ref).abs() - tol).max()


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16bit", "4bit"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: f"{h[0]}x{h[1]}")
def test_weight_decode_heads(dev, kind, heads):
    check_weight(kind(dev, [1] * 6, [1, 17, 64, 200, 3, 700], *heads, 64), rows_apart=5)


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16bit", "4bit"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_weight_new_tokens(dev, kind, D, dt):
    for new, own in (([2, 3, 4, 1, 0], [2, 50, 4, 9, 30]), ([70, 1, 33], [70, 300, 65]),
                     ([1, 190], [1, 255])):
        check_weight(kind(dev, new, own, 10, 2, D, dt, seed=sum(new)))


@pytest.mark.parametrize("page", [1, 2, 8, 64])
def test_weight_pages(dev, page):
    check_weight(Batch(dev, [1, 20, 1], [37, 90, 300], 8, 2, 128, page=page))
    if page >= 16:
        check_weight(Batch4(dev, [1, 20, 1], [37, 90, 300], 8, 2, 128, page=page))


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16bit", "4bit"])
@pytest.mark.parametrize("window,sinks,prefix", [(1, 0, 0), (5, 2, 0), (33, 40, 0), (64, 0, 30),
                                                 (100, 200, 130), (0, 0, 100), (1000, 8, 17),
                                                 (2 ** 31 - 1, 2 ** 31 - 1, 0)])
def test_weight_masks(dev, kind, window, sinks, prefix):
    own = [1, 17, 64, 99, 101, 300, 0, 500]
    for new in ([1] * 6 + [0, 1], [1, 4, 30, 2, 50, 7, 0, 80]):
        check_weight(kind(dev, new, own, 8, 2, 64, window=window, sinks=sinks, prefix=prefix,
                          seed=window % 97))


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16bit", "4bit"])
def test_weight_of_what_is_not_there(dev, kind):
    import torch
    check_weight(kind(dev, [1, 1, 2, 0, 3], [0, 5, 1, 0, 0], 8, 2, 64))
    b = kind(dev, [1, 1, 1, 50], [40, 40, 40, 60], 8, 2, 64)
    b.table[0, :] = -1
    b.table[1, 1], b.table[2, 0], b.table[3, 1] = 2 ** 31 - 1, b.k.shape[0], -5
    b.args[3] = b.table.to(dev)
    check_weight(b)
    b = kind(dev, [2, 3], [20, 30], 8, 2, 64)
    b.args[4] = torch.tensor([7, 2, 10 ** 6], dtype=torch.int32, device=dev)  # out of order
    w = torch.zeros(2, b.table.shape[1] * 16, device=dev)
    lse = torch.zeros(5, 8, device=dev)
    call = (fs.attend4_weight, b.cache) if kind is Batch4 else (fs.attend_weight, b.args[1])
    call[0](b.args[0], lse, call[1], *b.args[3:], w)
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16bit", "4bit"])
def test_weight_many_requests_long_rows_and_equal_bits(dev, kind):
    import torch
    check_weight(kind(dev, [1] * 150, [1 + 37 * i % 400 for i in range(150)], 4, 2, 64))
    check_weight(kind(dev, [1], [9000], 4, 1, 128))
    b = kind(dev, [300, 1, 40], [600, 90, 40], 4, 2, 128)
    lse = b.call()[1]
    call = (fs.attend4_weight, b.cache) if kind is Batch4 else (fs.attend_weight, b.args[1])
    kw = {k: v for k, v in b.kw.items() if k != "return_lse"}
    got = [torch.zeros(3, b.table.shape[1] * 16, device=dev) for _ in range(3)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for i, w in enumerate(got):
        call[0](b.args[0], lse, call[1], *b.args[3:], w, stream=s if i else None, **kw)
        torch.cuda.synchronize()
        assert torch.equal(w, got[0])
    # every row's weights sum to one
    assert abs(float(got[0].sum()) / (341 * 4) - 1) < 2.0 ** -16


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16bit", "4bit"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_weight_rows_left_out_and_not_finite(dev, kind, window, sinks):
    """A row whose lse is -infinity gives nothing, whatever it holds; one whose lse is NaN
    gives NaN to the keys that it sees, and to no others."""
    def change(q, lse):
        q[0, 1], lse[0, 1] = math.nan, -math.inf
        q[2], lse[2] = math.inf, -math.inf          # a token of the few
        lse[3, 5] = math.nan
        q[14, 3], lse[14, 3] = math.nan, -math.inf  # and of the many
        lse[20], lse[70, 0] = -math.inf, math.nan
        q[83], lse[83] = math.nan, -math.inf        # the last of a tile's rows
    check_weight(kind(dev, [1, 3, 80], [40, 50, 200], 8, 2, 64, window=window, sinks=sinks),
                 change=change)


@pytest.mark.parametrize("kind", [Batch, Batch4], ids=["16bit", "4bit"])
def test_weight_many_heads_and_most_requests(dev, kind):
    check_weight(kind(dev, [1, 2], [20, 37], 1024, 1, 64))
    check_weight(kind(dev, [1, 2], [20, 37], 1024, 1024, 64))
    new = [1] * 4094 + [40, 20]
    check_weight(kind(dev, new, [m + i % 5 for i, m in enumerate(new)], 2, 1, 64))


# ---------------------------------------------------------------- the eviction

def plain_evict(weight, kv, table, budget, page, sinks, recent):
    """Request after request, page after page (lists)."""
    width = len(table[0]) if table else 0
    out = [[], [], [], []]
    for w, m, row, b in zip(weight, kv, table, budget):
        m = min(max(0, m), width * page)
        pages = -(-m // page)
        first = min(-(-sinks // page), pages)
        may = [c for c in range(first, pages) if (c + 1) * page <= m - recent]
        may = [c for c in may if (c + 1) * page <= m]
        drop = min(-(-max(0, m - max(0, b)) // page), len(may))
        score = sorted((math.fsum(w[c * page:(c + 1) * page]), c) for c in may)
        gone = sorted(c for _, c in score[:drop])
        stay = [c for c in range(pages) if c not in gone]
        out[0].append([row[c] for c in stay] + [-1] * (width - len(stay)))
        kept = [x for c in stay for x in w[c * page:min(m, (c + 1) * page)]]
        out[1].append(kept + [0.0] * (width * page - len(kept)))
        out[2].append(m - drop * page)
        out[3] += [row[c] for c in gone if row[c] >= 0]
    return out


def check_evict(dev, kv, width, page, budget, sinks=0, recent=0, n_freed=None, seed=0, levels=0,
                holes=0.0, rows_apart=0):
    """``levels``: weights of so many values only (pages of equal weight)."""
    import torch
    rng = random.Random(seed)
    n = len(kv)
    ids = list(range(n * width))
    rng.shuffle(ids)
    table = [[ids[r * width + c] if c * page < kv[r] and rng.random() >= holes else -1 - c % 3
              for c in range(width)] for r in range(n)]
    # multiples of 2^-12: sums of them are exact in 64 bits
    weight = [[(rng.randrange(levels) if levels else int(2 ** 12 * rng.expovariate(1))) / 2 ** 12
               if j < kv[r] else 0.0 for j in range(width * page)] for r in range(n)]
    budget = [budget] * n if isinstance(budget, int) else budget

    def t(x, *shape, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype, device=dev).reshape(shape)
    w = torch.full((n, width * page + rows_apart), 9.0, device=dev)
    w[:, :width * page] = t(weight, n, width * page, dtype=torch.float32)
    log(f"kv_evict n={n} kv={kv[:5]} width={width} page={page} budget={budget[:4]} {sinks}/{recent}")
    got = fs.kv_evict(w[:, :width * page], t(kv, n), t(table, n, width), t(budget, n),
                      page_size=page, n_sink=sinks, n_recent=recent, n_freed=n_freed)
    ref = plain_evict(weight, kv, table, budget, page, sinks, recent)
    room = n * width if n_freed is None else n_freed
    freed = ref[3][:room] + [-1] * (room - len(ref[3]))
    for name, g, r in zip(("table", "weight", "kv_len", "freed", "count"), got,
                          (ref[0], ref[1], ref[2], freed, [len(ref[3])])):
        flat = [y for x in r for y in (x if isinstance(x, list) else [x])]
        assert g.cpu().reshape(-1).tolist() == flat, name


@pytest.mark.parametrize("page", [1, 2, 16, 64, 256])
@pytest.mark.parametrize("sinks,recent", [(0, 0), (1, 1), (4, 70), (100, 300), (10 ** 9, 0),
                                          (0, 2 ** 31 - 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_evict_pages_sinks_and_recent(dev, page, sinks, recent):
    rng = random.Random(page)
    kv = [0, 1, page - 1, page, page + 1, 5 * page, 300, 777] + [rng.randint(0, 900)
                                                                 for _ in range(9)]
    width = max(-(-m // page) for m in kv) + 2
    check_evict(dev, kv, width, page, [rng.choice((0, 1, 50, 200, 700, 2000)) for _ in kv],
                sinks, recent, seed=page + sinks % 7, rows_apart=3)


def test_evict_equal_weights_and_budgets_at_the_borders(dev):
    for levels in (1, 2):
        check_evict(dev, [160, 161, 175, 176, 320], 24, 16, [0, 16, 80, 160, 161], levels=levels)
    check_evict(dev, [64] * 8, 4, 16, [64, 63, 49, 48, 47, 1, 0, -5], levels=1)
    check_evict(dev, [4000] * 3, 300, 16, [17, 2000, 3990], levels=3)
    check_evict(dev, [900] * 4, 100, 16, [100, 200, 300, 400], levels=2, holes=0.3)


def test_evict_negative_weights_and_wide_rows(dev):
    import torch
    check_evict(dev, [20000, 3, 12345], 2500, 8, [5000, 1, 100], sinks=9, recent=40)
    check_evict(dev, [70000], 70001, 1, [31000], sinks=3, recent=5)
    w = torch.tensor([[-1.0, 0.0, -0.0, 3.0, -2.0, 1.0]], device=dev)
    t = torch.arange(6, dtype=torch.int32, device=dev).view(1, 6)
    i = torch.tensor([6], dtype=torch.int32, device=dev)
    got = fs.kv_evict(w, i, t, i * 0 + 2, page_size=1)
    assert got[0].tolist() == [[3, 5, -1, -1, -1, -1]] and got[3].tolist()[:4] == [0, 1, 2, 4]
    got = fs.kv_evict(w, i, t, i * 0 + 3, page_size=1)  # 0 and -0 are equal: the earlier goes
    assert got[0].tolist() == [[2, 3, 5, -1, -1, -1]] and got[1].tolist()[0][:3] == [0.0, 3.0, 1.0]


def test_evict_many_requests_and_room_for_freed_pages(dev):
    rng = random.Random(3)
    kv = [rng.randint(0, 200) for _ in range(700)]
    check_evict(dev, kv, 14, 16, 60, sinks=4, recent=20)
    check_evict(dev, kv[:50], 14, 16, 60, n_freed=7)
    check_evict(dev, kv[:50], 14, 16, 60, n_freed=0)
    check_evict(dev, [rng.randint(0, 20) for _ in range(4096)], 3, 8, 5)


def test_evict_nothing_and_lengths_past_the_row(dev):
    import torch
    check_evict(dev, [], 4, 16, 10, n_freed=3)
    check_evict(dev, [0, 0], 0, 16, 10, n_freed=3)
    check_evict(dev, [50, 60], 5, 16, 1000)
    kv = torch.tensor([10 ** 9, -7], dtype=torch.int32, device=dev)
    t = torch.arange(8, dtype=torch.int32, device=dev).view(2, 4)
    w = torch.arange(32, dtype=torch.float32, device=dev).view(2, 16)
    got = fs.kv_evict(w, kv, t, kv * 0 + 9, page_size=4)
    assert got[2].tolist() == [8, 0] and got[0].tolist() == [[2, 3, -1, -1], [-1] * 4]
    assert got[4].tolist() == [2] and got[3].tolist() == [0, 1] + [-1] * 6


# --------------------------------------------------------------- all together

def test_step_within_a_budget_in_a_captured_graph(dev):
    """Placement, store in 4 bits, attention, weights and an eviction in one graph, replayed
    with other inputs between eager work: every replay equals the eager calls."""
    import torch
    n, Hq, Hkv, D, page, width = 9, 8, 2, 64, 16, 12
    g = torch.Generator(device=dev).manual_seed(3)
    cache = fs.kv4_cache(n * width, Hkv, page, D, device=dev)
    cache.copy_(torch.randint(0, 100, cache.shape, device=dev, generator=g).to(torch.uint8))
    table = torch.arange(n * width, device=dev, dtype=torch.int32).view(n, width).contiguous()
    free = torch.arange(4, device=dev, dtype=torch.int32)
    old, new = (torch.full((n,), x, device=dev, dtype=torch.int32) for x in (31, 1))
    budget = torch.full((n,), 48, device=dev, dtype=torch.int32)
    qkv = torch.randn(n, Hq + 2 * Hkv, D, device=dev, generator=g).bfloat16()
    ang = torch.rand(200, D // 2, device=dev, generator=g)
    cs = torch.cat((ang.cos(), ang.sin()), 1).contiguous()
    w = torch.ones(D, device=dev).bfloat16()
    first = torch.rand(n, width * page, device=dev, generator=g)

    def one():
        slots, pos, q_start, kv_len, _ = fs.kv_layout(old, new, table, free, page_size=page,
                                                      n_tok=n)
        q = fs.qk_norm_rope4(qkv, pos, slots, cs, cache, w, w)
        out, lse = fs.attend4(q, cache, table, q_start, kv_len, max_q=1, return_lse=True)
        weight = fs.attend4_weight(q, lse, cache, table, q_start, kv_len, first.clone(), max_q=1)
        return (out, lse, weight, *fs.kv_evict(weight, kv_len, table, budget, page_size=page,
                                               n_recent=1, n_freed=n * width))
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
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_streams_at_once(dev):
    """Calls of two streams overlap and give what each gives alone."""
    import torch
    streams = [torch.cuda.Stream() for _ in range(2)]
    batches = [Batch4(dev, [1] * 20 + [70], [300 + 7 * i for i in range(20)] + [400], 8, 2, 128,
                      seed=i) for i in range(2)]

    def calls(b, stream=None):
        out, lse = b.call(stream=stream)
        w = torch.zeros(21, b.table.shape[1] * 16, device=dev)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        kw = dict(scale=b.scale, max_q=70, stream=stream)
        fs.attend4_weight(b.args[0], lse, b.cache, *b.args[3:], w, **kw)
        return (out, lse, w, *fs.kv_evict(w, b.args[5], b.args[3], b.args[5] // 2, page_size=16,
                                          n_sink=2, n_recent=40, stream=stream))
    alone = [calls(b) for b in batches]
    torch.cuda.synchronize()
    for _ in range(5):
        both = [calls(b, s) for b, s in zip(batches, streams)]
        torch.cuda.synchronize()
        for x, y in zip(alone, both):
            assert all(torch.equal(p, q) for p, q in zip(x, y))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("budget", [None, 32])
def test_replay_of_a_schedule(dev, bits, budget):
    """An ISJL schedule played on a worker with a cache of 4 bits, a budget of tokens, or
    both.  Which pages a request gave up is read from its row of the table; every token
    attends over exactly the tokens that its request holds then, at their own positions.
    The reference has queries in 64 bits, and keys too with 16 bits; rounding them to f16
    moves a score by at most d = (2 u + u^2) scale sum |q k| (u scale sum |q k| with 4 bits,
    whose keys are the cache's), and the output by (exp(2 d) - 1) A beside its own rounding."""
    import numpy as np
    import torch
    from paper_2608_02244_amd import replay
    rng = np.random.default_rng(5)
    n, Hq, Hkv, D, page, layers, u = 8, 4, 2, 64, 16, 2, U["f16"]
    a, p, o = (rng.integers(lo, hi, (1, n)).astype(np.int32)
               for lo, hi in ((0, 20), (1, 90), (1, 60)))
    _, start, finish = fs.simulate(a, p, o, policy="isjl", B=4, alpha=8, M_kv=600, cost_c=0,
                                   cost_tau=0, schedule=True)
    length = (p + o)[0].tolist()
    g = torch.Generator().manual_seed(9)
    x = torch.randn(layers, n, max(length), Hq + 2 * Hkv, D, generator=g).half()
    xd = x.to(dev)
    w = replay.Worker(n_pages=600 // page + n, page_size=page, q_heads=Hq, kv_heads=Hkv,
                      head_dim=D, max_len=max(length), layers=layers, dtype=torch.float16,
                      device=dev, kv_bits=bits, budget=budget, n_recent=8, n_sink=3)
    pages = len(w.free)
    y = x.double()
    y[..., :Hq + Hkv, :] /= (y[..., :Hq + Hkv, :].square().mean(-1, keepdim=True) + 1e-6).sqrt()
    cs = w.cos_sin.double().cpu()[:max(length), None, :]
    c, s = cs[..., :D // 2], cs[..., D // 2:]
    f, e = y[..., :Hq + Hkv, :D // 2].clone(), y[..., :Hq + Hkv, D // 2:].clone()
    y[..., :Hq + Hkv, :D // 2], y[..., :Hq + Hkv, D // 2:] = f * c - e * s, e * c + f * s
    if bits == 4:
        y[..., Hq:, :] = values(*quantise(y[..., Hq:, :], "f16"))
    holds, rows, seen, given = {}, {}, [0] * n, 0
    at_step = []

    def on_step(t, now, outs):
        nonlocal given
        at_step.append(t)
        for i, r in enumerate(now):
            mine = holds.setdefault(r, []) + [seen[r]]  # positions held while it attended
            seen[r] += 1
            for layer, out in enumerate(outs):
                z = y[layer, r]
                for h in range(Hq):
                    q, k = z[mine[-1], h], z[mine, Hq + h // 2]
                    v = z[mine, Hq + Hkv + h // 2]
                    wt = torch.softmax(k @ q * D ** -0.5, 0)
                    A = wt @ v.abs()
                    m = u if bits == 4 else 2 * u + u * u
                    d = m * D ** -0.5 * float((k.abs() @ q.abs()).max())
                    tol = math.expm1(2 * d) * A + 1.1 * u * (A + (wt @ v).abs()) + 2.0 ** -18 * (1 + A)
                    assert ((out[i, h].double().cpu() - wt @ v).abs() <= tol).all()
            row = w.table[w.requests.index(r)].tolist()
            before = rows.get(r, [])
            have = -(-len(mine) // page)
            kept = [q for q in before[:have] if q in row] if budget else before[:have]
            if budget and len(kept) < len(before):
                gone = [j for j, q in enumerate(before) if q not in row]
                given += len(gone)
                mine = [x for j, x in enumerate(mine) if j // page not in gone]
            holds[r] = mine
            rows[r] = row[:-(-len(mine) // page)]
            assert w.held[r] == len(mine) and w.position(r) == seen[r]
        free = w.free.tolist() + [q for r in w.requests for q in rows[r]]
        assert sorted(free) == list(range(pages))
    log(f"replay bits={bits} budget={budget} {sum(length)} tokens")
    replay.play(w, start[0], finish[0],
                lambda layer, now, at: torch.stack([xd[layer, r, i] for r, i in zip(now, at)]),
                on_step)
    assert seen == length and sorted(w.free.tolist()) == list(range(pages))
    assert bool(given) == bool(budget)
