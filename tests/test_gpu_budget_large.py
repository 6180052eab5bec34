"""The operators of a KV cache within a budget where the work fills the card several times
over: attention weights whose blocks go through many units, key heads and tiles, and
evictions from rows that one block does not hold.  References are in 64 bits, request by
request; what has to be large is computed from the shapes and asserted.

Tolerance of a weight, fixed before any run: as for small batches (w (e + 2^-22 (|s| + |lse|))
+ 2^-23 |weight|, e = (D + 8) 2^-24 scale sum_d |q_d k_d|), but the sum of a key's n terms is
taken over lanes: with many rows 32, each of which adds n / 32; with few rows one or two terms
for each key head (at most 16 here).  Behind that are the exchange between lanes (5) and the
joining of a tile's parts, whose number is computed from the shapes: no term goes through more
additions than n / 16 + 16 + parts, of 2^-24 of the sum each.  (In the longest prompts with
most heads, where n is largest, 64 rows of one key head left out of the last tiles' sums are
ten times that and more, but less in the first tiles'.)"""
import math

import pytest

import paper_2608_02244_amd as fs
from test_gpu_budget_operators import check_evict
from test_gpu_step_operators import dev, dtype_of, log  # noqa: F401

pytestmark = pytest.mark.gpu


class Large:
    """A batch made on the GPU: keys at random, NaN wherever no token of a request is."""

    def __init__(self, dev, new, own, Hq, Hkv, D, dt, bits, page, window=0, sinks=0):
        import torch
        self.__dict__.update(dev=dev, new=new, own=own, Hq=Hq, Hkv=Hkv, D=D, bits=bits, page=page,
                             window=window, sinks=sinks, scale=D ** -0.5)
        t = dtype_of(dt)
        g = torch.Generator(device=dev).manual_seed(len(own) + D)
        need = [-(-m // page) for m in own]
        n_pages, width = sum(need) + 3, max(need) + 1
        ids = torch.randperm(n_pages, device=dev, generator=g).to(torch.int32)
        self.table = torch.full((len(own), width), -1, dtype=torch.int32, device=dev)
        self.slots, at = [], 0
        for r, (m, n) in enumerate(zip(own, need)):
            self.table[r, :n] = ids[at:at + n]
            at += n
            j = torch.arange(m, device=dev)
            self.slots.append((self.table[r, j // page] * page + j % page).to(torch.int32))
        held = torch.zeros(n_pages * page, dtype=torch.bool, device=dev)
        held[torch.cat(self.slots).long()] = True
        held = held.view(n_pages, page)
        if bits == 16:
            self.k = torch.randn(n_pages, Hkv, page, D, device=dev, generator=g).to(t)
            self.k.masked_fill_(~held[:, None, :, None], math.nan)
        else:
            shape = (n_pages, Hkv, page // 16, 17 * D)
            self.k = torch.randint(0, 256, shape, device=dev, generator=g, dtype=torch.uint8)
            scales = self.k[..., 16 * D:]  # of keys and values: 1/4 .. 1
            scales.copy_(torch.randint(125, 128, scales.shape, device=dev, generator=g,
                                       dtype=torch.uint8))
            keys = self.k[..., 16 * D:16 * D + D // 2].unflatten(-1, (16, D // 32))
            keys.masked_fill_(~held.view(n_pages, 1, page // 16, 16, 1), 255)
        self.q = (1.5 * torch.randn(sum(new), Hq, D, device=dev, generator=g)).to(t)
        start = [0]
        for m in new:
            start.append(start[-1] + m)
        self.start = start
        self.step = (self.table, torch.tensor(start, dtype=torch.int32, device=dev),
                     torch.tensor(own, dtype=torch.int32, device=dev))

    def keys(self, r):
        """[own, Hkv, D] float64 of request r."""
        s = self.slots[r].long()
        if self.bits == 16:
            return self.k[s // self.page, :, s % self.page].double()
        return fs.kv4_read(self.k, self.slots[r], dtype=self.q.dtype)[0].double()

    def check(self):
        import torch
        log(f"attend_weight bits={self.bits} n={len(self.own)} new={self.new[:3]} "
            f"own={self.own[:3]} heads={self.Hq}/{self.Hkv} D={self.D} page={self.page} "
            f"window={self.window}/{self.sinks}")
        g = torch.Generator(device=self.dev).manual_seed(3)
        row, grp = self.table.shape[1] * self.page, self.Hq // self.Hkv
        start = torch.rand(len(self.own), row, device=self.dev, generator=g)
        ref, tol = start.double(), 2.0 ** -23 * start.double()
        parts = self.most_parts()
        seen = torch.zeros_like(start, dtype=torch.bool)
        lse = torch.full(self.q.shape[:2], -math.inf, device=self.dev)
        for r, (m, own) in enumerate(zip(self.new, self.own)):
            K, x = self.keys(r), self.q[self.start[r]:self.start[r] + m].double()
            j = torch.arange(own, device=self.dev)
            p = (own - m + torch.arange(m, device=self.dev))[:, None]
            see = j <= p
            if self.window:
                see = see & ((j > p - self.window) | (j < self.sinks))
            seen[r, :own] = see.any(0)
            n = see.sum(0) * self.Hq
            for h in range(self.Hq):
                kk = K[:, h // grp].t().contiguous()
                s = torch.where(see, torch.mm(x[:, h], kk) * self.scale, -math.inf)
                a = torch.logsumexp(s, 1).float()
                lse[self.start[r]:self.start[r] + m, h] = a
                a = a.double()[:, None]
                w = torch.exp(s - a)
                size = torch.mm(x[:, h].abs(), kk.abs()) * self.scale
                part = (self.D + 8) * 2.0 ** -24 * size + \
                    2.0 ** -22 * (torch.where(see, s, 0.0).abs() + a.abs()) + \
                    ((n / 16 + 16 + parts) * 2.0 ** -24)[None]
                ref[r, :own] += w.sum(0)
                tol[r, :own] += (w * part).sum(0) + 2.0 ** -126
        got = start.clone()
        f = fs.attend4_weight if self.bits == 4 else fs.attend_weight
        kw = dict(scale=self.scale, window=self.window, n_sink=self.sinks, max_q=max(self.new))
        f(self.q, lse, self.k, *self.step, got, **kw)
        assert torch.equal(got[~seen], start[~seen])
        off = (got.double() - ref).abs() - tol - 2.0 ** -23 * ref
        assert (off <= 0).all(), (float(off.max()), int((off > 0).sum()))
        again = start.clone()
        f(self.q, lse, self.k, *self.step, again, **kw)
        assert torch.equal(got, again)

    # units as the kernels cut them (tokens, keys and heads to pieces), from the shapes

    def row_units(self):
        """Units of 32 keys of requests with at most 32 rows."""
        n = 0
        for m, own in zip(self.new, self.own):
            if m * self.Hq // self.Hkv <= 32:
                lo = max(0, own - m - self.window + 1) if self.window else 0
                n += -(-own // 32) - lo // 32
        return n

    def tile_units(self):
        """Units of every tile, of one key head: stages of 64 rows, and eight to begin them."""
        grp, per = self.Hq // self.Hkv, 128 if self.D == 256 else 256
        units = []
        for m, own in zip(self.new, self.own):
            if m * grp <= 32:
                continue
            for k0 in range(0, own, per):
                k1 = min(k0 + per, own)
                a, e = max(0, k0 - (own - m)), m
                if self.window and k0 >= self.sinks:
                    e = min(e, k1 - 1 + self.window - (own - m))
                if e > a:
                    units.append(-(-(e - a) * grp // 64) + 8)
        return units

    def piece(self):
        """Units of a block's piece of the tiles."""
        return sum(self.tile_units()) * self.Hkv / (2 * compute_units(self.dev))

    def most_parts(self):
        """Parts of the longest tile."""
        units = self.tile_units()
        return math.ceil(max(units) * self.Hkv / self.piece()) + 1 if units else 1


def compute_units(dev):
    import torch
    return torch.cuda.get_device_properties(dev).multi_processor_count


def check_rows(b):
    # blocks of four waves, four to a unit at most: every wave has some units of its own
    assert b.row_units() > 4 * 16 * compute_units(b.dev), b.row_units()
    b.check()


def check_tiles(b, whole=False):
    """``whole``: with tiles that lie whole in a piece."""
    assert b.piece() > 10
    if whole:
        assert min(b.tile_units()) * b.Hkv * 2 < b.piece()
    b.check()


BITS = pytest.mark.parametrize("bits", [16, 4])
DIMS = pytest.mark.parametrize("D", [64, 128, 256])


@BITS
@DIMS
@pytest.mark.parametrize("heads", [(8, 4), (20, 4), (16, 8)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_weight_rows_of_many_units(dev, bits, D, heads):
    """Decode: every wave has several units of a request, and units of two requests."""
    own = [1000 + 1237 * i % 4001 for i in range(220)]
    check_rows(Large(dev, [1] * 220, own, *heads, D, "bf16", bits, 16))


@BITS
@DIMS
def test_weight_rows_of_drafts(dev, bits, D):
    """17 to 32 rows: two row tiles."""
    own = [1500 + 1237 * i % 4001 for i in range(220)]
    check_rows(Large(dev, [1 + i % 4 for i in range(220)], own, 32, 4, D, "f16", bits, 64))


@BITS
@pytest.mark.parametrize("window,sinks", [(900, 40), (777, 0)])
def test_weight_rows_behind_a_window(dev, bits, window, sinks):
    own = [1000 + 1237 * i % 2003 for i in range(700)]
    check_rows(Large(dev, [1] * 700, own, 8, 4, 64, "bf16", bits, 32, window, sinks))
    check_rows(Large(dev, [3] * 700, own, 16, 2, 128, "f16", bits, 16, window, sinks))


@pytest.mark.parametrize("page", [1, 8])
def test_weight_rows_of_small_pages(dev, page):
    own = [1000 + 1237 * i % 4001 for i in range(220)]
    check_rows(Large(dev, [1] * 220, own, 8, 4, 64, "bf16", 16, page))


@BITS
@DIMS
@pytest.mark.parametrize("heads", [(32, 16), (30, 6), (12, 4), (16, 2)],
                         ids=lambda h: f"{h[0]}x{h[1]}")
def test_weight_tiles_of_prompts(dev, bits, D, heads):
    """Whole prompts: pieces of many stages that begin and end inside tiles and key heads."""
    new = [1900, 3311]
    check_tiles(Large(dev, new, new, *heads, D, "bf16", bits, 16))


@BITS
@pytest.mark.parametrize("D,heads", [(64, (16, 8)), (128, (30, 6)), (256, (16, 4))])
def test_weight_tiles_of_chunks_behind_a_window(dev, bits, D, heads):
    """Chunks of prompts behind what their requests hold, decoding requests beside them."""
    new, own = [1100, 1, 1900, 1, 700], [2500, 900, 2700, 33, 700]
    check_tiles(Large(dev, new, own, *heads, D, "f16", bits, 32))
    check_tiles(Large(dev, [2 * m for m in new], [2 * m for m in own], *heads, D, "f16", bits, 64,
                      window=900, sinks=21))


@BITS
@DIMS
@pytest.mark.parametrize("heads", [(4, 2), (3, 1)], ids=lambda h: f"{h[0]}x{h[1]}")
def test_weight_tiles_of_many_short_prompts(dev, bits, D, heads):
    """Pieces of several tiles: some whole in one, others at both of its ends."""
    new = [40 + 29 * i % 211 for i in range(800)]
    check_tiles(Large(dev, new, new, *heads, D, "bf16", bits, 16), whole=True)


# --------------------------------------------- evictions in more than one launch

# (page, width): rows that one block holds and the next size, by tokens (32,768) and by
# pages (4,096)
ROWS = [(8, 4096), (8, 4097), (1, 4097), (2, 4097), (4, 8193), (16, 2048), (16, 2049), (64, 513),
        (128, 257), (256, 129)]


@pytest.mark.parametrize("page,width", ROWS)
@pytest.mark.parametrize("levels,holes,apart", [(0, 0.0, 0), (2, 0.2, 3), (0, 0.1, 3), (3, 0.0, 0)])
def test_evict_rows_past_one_block(dev, page, width, levels, holes, apart):
    """Requests of uneven length, an empty one and one within its budget among them."""
    row = width * page
    kv = [row, 0, row - 3, 2 * page + 1, 2 * row // 3]
    budget = [row // 2, 5, row - 5 * page, row, 3]
    check_evict(dev, kv, width, page, budget, sinks=3, recent=page + 9, seed=page, levels=levels,
                holes=holes, rows_apart=apart)


def test_evict_rows_past_one_block_with_nothing_to_drop(dev):
    check_evict(dev, [33000, 40, 0], 2100, 16, 33000, sinks=3, recent=9, levels=2)
    check_evict(dev, [33000, 33600], 2100, 16, 10, sinks=10 ** 9, levels=2)
    check_evict(dev, [33000, 33600], 2100, 16, 10, recent=2 ** 31 - 1, n_freed=5, levels=2)
    check_evict(dev, [33000, 33600, 20000], 2100, 16, 0, n_freed=100, rows_apart=1)


def test_evict_a_page_that_two_requests_list(dev):
    """Each request gives it up for itself: its id comes once for each that does."""
    import torch
    table = torch.tensor([[5, 6, 7], [5, 8, 9], [5, 2, 3]], dtype=torch.int32, device=dev)
    weight = torch.tensor([[0.0, 2, 1], [0, 1, 2], [3, 2, 1]], device=dev)
    kv = torch.tensor([3, 3, 3], dtype=torch.int32, device=dev)
    got = fs.kv_evict(weight, kv, table, torch.full_like(kv, 2), page_size=1)
    assert got[0].tolist() == [[6, 7, -1], [8, 9, -1], [5, 2, -1]]
    assert got[3].tolist()[:3] == [5, 5, 3] and got[4].tolist() == [3]
