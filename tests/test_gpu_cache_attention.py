"""Attention of new tokens over the paged cache, against 64 bits.

How far a result may be off: with A = sum_j p_j |v_j| over a row's normalised weights and B = the largest scale * sum_d |q_d k_jd|,
* scores are binary32 sums of exact products: off by at most (D + 4) 2^-24 B, their weights by e^2 of that relatively, and exp adds 2^-22
  for itself and 2^-22 B for its argument in another base;
* weights are rounded once to the element type: half a step h, relatively; that of the sum of weights cancels at best, so 2 h at worst;
* weights below binary32's smallest normal number 2^-126 are 0 (the largest of a row is 1, so their sum is at least that): a value's part
  of the result is then lost, |v_j| 2^-126 at most;
* sums over n keys add n 2^-24, the joining of parts and the final division 2^-21;
* the output is rounded once: h |o|.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF_STEP = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}


@pytest.fixture(scope="module")
def ctx():
    from paper_2605_07330_amd import srs
    c = srs.Context(0)
    yield c
    c.close()


class Batch:
    def __init__(self, start, count, hq, hkv, d, page, dtype=torch.bfloat16, layout="plain", seed=0, spread=1.0, extra_rows=0, wide=0):
        g = torch.Generator(device=DEV).manual_seed(seed * 1000 + d)
        self.start, self.count, self.page, self.hq, self.hkv, self.d, self.dtype = list(start), list(count), page, hq, hkv, d, dtype
        keys = [s + c for s, c in zip(start, count)]
        have = [-(-k // page) for k in keys]
        self.pages = sum(have) + 5
        order = torch.randperm(self.pages, generator=g, device=DEV).tolist()
        width = max(have + [1]) + wide
        table = torch.full((len(start), width), -1, dtype=torch.int32)
        for r, h in enumerate(have):
            table[r, :h] = torch.tensor([order.pop() for _ in range(h)], dtype=torch.int32)
        self.table = table.to(DEV)
        self.begin = torch.tensor([0] + list(torch.tensor(count, dtype=torch.int64).cumsum(0)), dtype=torch.int32, device=DEV)
        self.at = torch.tensor(start, dtype=torch.int32, device=DEV)
        T = sum(count) + extra_rows
        self.q = (torch.randn(T, hq, d, generator=g, device=DEV) * spread).to(dtype)
        def pool():
            if layout == "heads first":
                return torch.randn(self.pages, hkv, page, d, generator=g, device=DEV).to(dtype).transpose(1, 2)
            if layout == "one tensor":
                return torch.randn(self.pages, page, 2, hkv, d + 8, generator=g, device=DEV).to(dtype)[:, :, 1, :, :d]
            return torch.randn(self.pages, page, hkv, d, generator=g, device=DEV).to(dtype)
        self.k, self.v = pool(), pool()

    def places(self, r):
        """Page and place of each of the request's keys."""
        j = torch.arange(self.start[r] + self.count[r], device=DEV)
        return self.table[r].long()[(j // self.page).clamp(max=self.table.shape[1] - 1)], j % self.page, j

    def expect(self, scale=None, causal=True, window=0, sinks=0):
        """out, lse, and how far they may be off (all float64)."""
        scale = self.d ** -0.5 if scale is None else scale
        h, group = HALF_STEP[self.dtype], self.hq // self.hkv
        out = torch.zeros(self.q.shape, dtype=torch.float64, device=DEV)
        lse = torch.full(self.q.shape[:2], -math.inf, dtype=torch.float64, device=DEV)
        tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
        b = self.begin.tolist()
        for r in range(len(self.start)):
            if b[r + 1] == b[r]:
                continue
            page, place, j = self.places(r)
            rows = slice(b[r], b[r + 1])
            i = self.start[r] + torch.arange(b[r + 1] - b[r], device=DEV)[:, None]
            seen = (page >= 0) & (page < self.pages) & (j < self.table.shape[1] * self.page)
            seen = seen[None].expand(i.shape[0], -1).clone()
            if causal:
                seen &= j <= i
            if window:
                seen &= (i - j < window) | (j < sinks)
            ok = page.clamp(0, self.pages - 1)
            k, v = self.k[ok, place].double().repeat_interleave(group, 1), self.v[ok, place].double().repeat_interleave(group, 1)
            q = self.q[rows].double()
            for head in range(self.hq):
                s = (q[:, head] @ k[:, head].t()) * scale
                size = (q[:, head].abs() @ k[:, head].abs().t()) * abs(scale)
                s = s.masked_fill(~seen, -math.inf)
                size = size.masked_fill(~seen, 0.0)
                some = seen.any(1)
                top = s.amax(1, keepdim=True).masked_fill(~some[:, None], 0.0)
                p = (s - top).exp()
                total = p.sum(1, keepdim=True)
                w = torch.where(seen, p / total.clamp(min=1e-300), torch.zeros_like(p))
                vv = v[:, head]
                hidden = ~seen.any(0)
                vv = vv.masked_fill(hidden[:, None], 0.0)                   # no row's, whatever it holds
                o = torch.zeros(s.shape[0], self.d, dtype=torch.float64, device=DEV)
                A = torch.zeros_like(o)
                clean = torch.isfinite(vv).all(1)
                o += w[:, clean] @ vv[clean]
                A += w[:, clean] @ vv[clean].abs()
                for key in (~clean).nonzero().flatten().tolist():            # not a number reaches those rows only that see it
                    o += torch.where(seen[:, key, None], w[:, key, None] * vv[key], torch.zeros_like(o))
                out[rows, head] = torch.where(some[:, None], o, torch.zeros_like(o))
                lse[rows, head] = torch.where(some, top[:, 0] + total[:, 0].log(), torch.full_like(top[:, 0], -math.inf))
                B, n = size.amax(1), seen.sum(1)
                score = (self.d + 4) * 2.0**-24 * B + 2.0**-22 * B + 2.0**-22
                tol[rows, head] = h * o.abs() + A * (2 * h + 2 * score + n * 2.0**-24 + 2.0**-21)[:, None] + 2.0**-126 * vv[clean].abs().sum(0)
                ltol[rows, head] = score + n * 2.0**-24 + 2.0**-21 + 2.0**-23 * lse[rows, head].abs().nan_to_num(0, 0, 0)
        return out, lse, tol, ltol

    def call(self, ctx, out=None, lse=None, **kw):
        out = torch.full_like(self.q, 9.0) if out is None else out
        lse = torch.full(self.q.shape[:2], 9.0, device=DEV) if lse is None else lse
        ctx.cache_attention(self.q, out, self.k, self.v, self.table, self.begin, self.at, lse=lse, **kw)
        return out, lse


def compare(got, want):
    (out, lse), (o, l, tol, ltol) = got, want
    n = tol.shape[0]
    for x, y, t, name in ((out, o, tol, "out"), (lse, l, ltol, "lse")):
        x = x[:n].double()
        fine = torch.isfinite(y)
        assert torch.equal(torch.isnan(x), torch.isnan(y)), name
        assert torch.equal(x[~fine & ~torch.isnan(y)], y[~fine & ~torch.isnan(y)]), name
        off = ((x - y).abs() - t)[fine]
        assert not off.numel() or off.max() <= 0, f"{name}: off by {off.max().item()} beyond the bound"


def check(ctx, batch, flags=0, hints=(True, False), **kw):
    want = batch.expect(**kw)
    for hint in hints:
        most = {"most_tokens": max(batch.count), "most_keys": max(s + c for s, c in zip(batch.start, batch.count))} if hint else {}
        compare(batch.call(ctx, **kw, **most), want)
        assert ctx.status() == flags


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (32, 4, 128), (8, 8, 64), (5, 1, 128), (6, 2, 80), (4, 2, 256), (40, 1, 64), (3, 3, 8), (10, 2, 96)])
@pytest.mark.parametrize("page", [16, 24, 64])
def test_decoding(ctx, dtype, hq, hkv, d, page):
    """One token each: lengths from a single key to several tiles, around pages and tiles."""
    starts = [0, 1, 14, 15, 16, 31, 32, 63, 64, 127, 128, 129, 255, 300, 511, 700]
    check(ctx, Batch(starts, [1] * len(starts), hq, hkv, d, page, dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d,page", [(32, 8, 128, 16), (8, 1, 128, 64), (6, 2, 80, 24), (4, 4, 64, 1), (2, 1, 256, 128), (10, 2, 96, 32), (70, 1, 64, 16), (264, 1, 32, 16)])
def test_chunks(ctx, dtype, hq, hkv, d, page):
    """Chunks of every kind beside decoding requests and requests with nothing new."""
    check(ctx, Batch([0, 5, 100, 0, 33, 64, 200, 77], [1, 1, 0, 130, 2, 64, 17, 1], hq, hkv, d, page, dtype))


@pytest.mark.parametrize("start,count", [([0], [1]), ([0], [2]), ([0], [31]), ([0], [32]), ([0], [33]), ([0], [257]), ([1000], [1]), ([4095], [130]), ([0, 0], [0, 0]),
                                         ([0, 3], [0, 1])])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 8)])
def test_lengths(ctx, start, count, hq, hkv):
    batch = Batch(start, count, hq, hkv, 128, 16)
    if sum(count):
        check(ctx, batch)
    else:
        out, lse = batch.call(ctx)
        assert out.numel() == 0 and ctx.status() == 0


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 0), (64, 4), (100, 40), (129, 200), (100000, 7), (33, 600)])
@pytest.mark.parametrize("count", [[1, 1, 1], [1, 40, 130]])
@pytest.mark.parametrize("d,page", [(128, 16), (64, 24)])
def test_windows(ctx, window, sinks, count, d, page):
    check(ctx, Batch([10, 333, 1000], count, 8, 2, d, page), window=window, sinks=sinks)


def test_a_long_window(ctx):
    check(ctx, Batch([20000, 9000], [1, 70], 8, 1, 128, 64), window=3000, sinks=130)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_long_axis(ctx, dtype):
    """Few rows over many keys: the keys are shared out and the parts joined."""
    check(ctx, Batch([40000, 17, 9000], [1, 1, 1], 8, 1, 128, 64, dtype))
    check(ctx, Batch([30000], [5], 4, 2, 64, 24, dtype))
    check(ctx, Batch([20000], [40], 8, 2, 128, 16, dtype))


def test_every_row_sees_every_key(ctx):
    check(ctx, Batch([0, 50, 200], [70, 1, 33], 8, 2, 128, 16), causal=False)
    check(ctx, Batch([5000], [3], 8, 2, 64, 24), causal=False)


@pytest.mark.parametrize("layout", ["heads first", "one tensor"])
@pytest.mark.parametrize("count", [[1, 1], [1, 150]])
def test_layouts(ctx, layout, count):
    check(ctx, Batch([500, 70], count, 8, 2, 128, 16, layout=layout))
    check(ctx, Batch([500, 70], count, 6, 2, 72, 24, layout=layout))


def test_rows_of_a_projection(ctx):
    """Queries inside wider rows, outputs inside others, heads before tokens; what lies between stays."""
    b = Batch([100, 0], [1, 50], 8, 2, 128, 16)
    want = b.expect()
    T = b.q.shape[0]
    wide = torch.randn(T, 12, 128, device=DEV).to(b.dtype)
    wide[:, 2:10] = b.q
    b.q = wide[:, 2:10]
    buffer = torch.full((8, T + 3, 136), 5.0, dtype=b.dtype, device=DEV)
    out = buffer[:, 1:T + 1, 8:].transpose(0, 1)
    compare(b.call(ctx, out=out), want)
    buffer[:, 1:T + 1, 8:] = 5.0
    assert bool((buffer == 5.0).all())


@pytest.mark.parametrize("count", [[1, 1, 1], [3, 1, 90]])
@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
def test_junk_where_no_row_looks(ctx, count, page, junk):
    """Pages that belong to nobody, places behind the last token and keys that a window hides."""
    b = Batch([37, 400, 777], count, 8, 2, 128, page)
    for kw in ({}, {"window": 50, "sinks": 3}):
        mine = torch.zeros(b.pages, b.page, dtype=torch.bool, device=DEV)
        for r in range(3):
            p, place, j = b.places(r)
            first = b.start[r] - kw.get("window", 10**9) + 1
            keep = (j >= first) | (j < kw.get("sinks", 0))
            mine[p[keep], place[keep]] = True
        b.k[~mine], b.v[~mine] = junk, -junk
        check(ctx, b, **kw)


@pytest.mark.parametrize("count", [[2, 1], [5, 1], [150, 40]])
@pytest.mark.parametrize("hq", [2, 8])
def test_junk_that_later_rows_see(ctx, count, hq):
    """A key or value that is not a number reaches the rows that see it, and no row before it."""
    b = Batch([37, 400], count, hq, 2, 128, 16)
    for r, what in ((0, "v"), (1, "k")):
        p, place, j = b.places(r)
        at = b.start[r] + (b.count[r] + 1) // 2
        if at < j.numel():
            getattr(b, what)[p[at], place[at], 0, 5] = float("nan")
    p, place, j = b.places(0)
    b.v[p[-1], place[-1], 1, 7] = float("inf")
    check(ctx, b)


def test_junk_inside_a_window(ctx):
    """Values that are not finite pass out of the window of later rows."""
    b = Batch([200], [150], 4, 2, 64, 16)
    p, place, j = b.places(0)
    for at in (150, 190, 205, 260):
        b.v[p[at], place[at], 1, 3] = float("inf")
    check(ctx, b, window=40, sinks=2)


def test_infinite_scores_and_large_ones(ctx):
    b = Batch([300, 20], [1, 60], 8, 2, 128, 16, spread=40.0)          # one key takes all the weight
    check(ctx, b)
    b.q[0] *= 0                                                         # all keys alike
    check(ctx, b)
    check(ctx, b, scale=0.0)
    check(ctx, b, scale=-0.05)
    low = torch.finfo(torch.bfloat16).min
    p, place, j = b.places(1)
    b.v[p[3], place[3]] = low                                           # the type's lowest value is a value
    check(ctx, b)


def test_pages_that_are_not_there(ctx):
    """Their keys count as hidden; a row left without any is 0."""
    from paper_2605_07330_amd import srs
    for count in ([1, 1, 1, 1], [3, 1, 70, 20]):
        b = Batch([37, 400, 100, 5], count, 8, 2, 128, 16)
        b.table[0, 1], b.table[1, 7], b.table[2, :3] = -1, b.pages, 2**31 - 1
        b.table[3] = -2**31
        check(ctx, b, flags=srs.FLAG_BAD_INDEX)
        out, lse = b.call(ctx)
        rows = slice(int(b.begin[3]), int(b.begin[4]))
        assert not bool(out[rows].any()) and bool((lse[rows] == -math.inf).all())
        assert ctx.status() == srs.FLAG_BAD_INDEX


def test_a_missing_page_that_no_row_needs(ctx):
    b = Batch([500, 800], [1, 20], 8, 2, 128, 16)
    b.table[0, 2:27], b.table[1, 2:45] = -1, 10**9                       # behind the window, before it the sinks
    check(ctx, b, window=64, sinks=20)


def test_a_table_too_narrow(ctx):
    from paper_2605_07330_amd import srs
    b = Batch([100, 30], [1, 20], 8, 2, 128, 16)
    b.table = b.table[:, :3].contiguous()
    check(ctx, b, flags=srs.FLAG_BAD_INDEX)


def test_no_page_at_all(ctx):
    from paper_2605_07330_amd import srs
    for width in (0, 4):
        b = Batch([100, 30], [1, 20], 8, 2, 128, 16)
        b.table, b.k, b.v = b.table[:, :width].contiguous(), b.k[:0] if width else b.k, b.v[:0] if width else b.v
        out, lse = b.call(ctx)
        assert not bool(out.any()) and bool((lse == -math.inf).all())
        assert ctx.status() == srs.FLAG_BAD_INDEX


def test_rows_outside_every_request(ctx):
    """A padded batch: rows behind the last request, and in front of the first, stay."""
    b = Batch([37, 400], [1, 20], 8, 2, 128, 16, extra_rows=50)
    want = b.expect()
    out, lse = b.call(ctx)
    compare((out[:21], lse[:21]), tuple(x[:21] for x in want))
    assert bool((out[21:] == 9.0).all()) and bool((lse[21:] == 9.0).all())
    b.begin += 13
    out, lse = b.call(ctx)
    assert bool((out[:13] == 9.0).all()) and bool((out[34:] == 9.0).all()) and not bool((out[13:34] == 9.0).all(2).any())
    assert ctx.status() == 0


@pytest.mark.parametrize("begin", [[-4, 5, 21], [0, 30, 21], [0, 1, 500], [25, 26, 27], [2**31 - 1, 2**31 - 1, 2**31 - 1]])
def test_requests_with_rows_that_are_not_there(ctx, begin):
    """Left out, with a flag; the others are computed."""
    from paper_2605_07330_amd import srs
    b = Batch([37, 400], [1, 20], 8, 2, 128, 16)
    b.begin = torch.tensor(begin, dtype=torch.int32, device=DEV)
    b.call(ctx)
    some = any(not 0 <= x <= y <= 21 for x, y in zip(begin, begin[1:]))
    assert ctx.status() == (srs.FLAG_BAD_INDEX if some else 0)


def test_a_negative_start(ctx):
    from paper_2605_07330_amd import srs
    b = Batch([37, 400], [1, 20], 8, 2, 128, 16)
    want = b.expect()
    b.at[0] = -1
    out, lse = b.call(ctx)
    assert ctx.status() == srs.FLAG_BAD_INDEX
    assert bool((out[0] == 9.0).all())
    compare((out[1:], lse[1:]), tuple(x[1:] for x in want))


def test_wrong_hints_cost_time_only(ctx):
    b = Batch([900, 400, 3000], [1, 200, 9], 8, 2, 128, 16)
    want = b.expect()
    for most_tokens, most_keys in ((1, 1), (1, 10**6), (10**6, 64), (2, 700), (10**9, 10**9)):
        compare(b.call(ctx, most_tokens=most_tokens, most_keys=most_keys), want)
        assert ctx.status() == 0


def test_without_lse_and_the_same_again(ctx):
    b = Batch([900, 400, 5000], [1, 200, 1], 8, 2, 128, 16)
    out, _ = b.call(ctx)
    for _ in range(3):
        again = torch.full_like(b.q, 1.0)
        ctx.cache_attention(b.q, again, b.k, b.v, b.table, b.begin, b.at)
        assert torch.equal(out, again)                                  # and bit for bit the same each time


@pytest.mark.parametrize("count", [[1, 1, 1], [3, 1, 90]])
def test_in_place(ctx, count):
    """The output over the queries."""
    b = Batch([37, 4000, 777], count, 8, 2, 128, 16)
    want = b.expect()
    compare(b.call(ctx, out=b.q), want)
    assert ctx.status() == 0


@pytest.mark.parametrize("count", [1, 40])
def test_keys_and_values_laid_out_differently(ctx, count):
    b = Batch([500, 70], [count, 1], 8, 2, 128, 16)
    b.v = b.v.transpose(1, 2).contiguous().transpose(1, 2)
    check(ctx, b)
    b.k = torch.cat([b.k, b.k], 3)[..., 128:]                           # wider rows
    check(ctx, b)


def test_many_requests(ctx):
    """More than one round of the search for a row's request; requests without rows among them."""
    g = torch.Generator().manual_seed(4)
    start, count = torch.randint(0, 60, (700,), generator=g).tolist(), torch.randint(0, 3, (700,), generator=g).tolist()
    count[5], count[350], count[699] = 40, 33, 21
    check(ctx, Batch(start, count, 2, 1, 64, 16))


def test_parts_of_many_requests(ctx):
    """Few parts each, of some only; heads that share a key head in two blocks."""
    start = [50] * 69 + [5000]
    check(ctx, Batch(start, [1] * 70, 8, 4, 64, 16))
    check(ctx, Batch([3000, 20, 900], [1, 1, 1], 40, 2, 128, 16))
    check(ctx, Batch([6000, 20, 900], [1, 2, 1], 6, 1, 256, 24))


# Workgroups a little over one or two rounds of the card: heads wide, head dimension, start and count of the requests, page.
ROUNDS = [(64, 64, 128, [1000], [1029], 16), (64, 64, 64, [200], [1539], 16), (32, 32, 256, [100], [2049], 16), (128, 16, 128, [1500], [521], 64),
          (192, 48, 72, [0, 3000, 700, 5], [200, 90, 1, 60], 24), (48, 48, 96, [1100, 1100, 2000], [128, 1300, 1], 16)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d,start,count,page", ROUNDS)
def test_a_last_round_of_few_workgroups(ctx, dtype, hq, hkv, d, start, count, page):
    """What is left after whole rounds is shared out and joined; rows behind the last sequence stay."""
    batch = Batch(start, count, hq, hkv, d, page, dtype, extra_rows=40)
    want = batch.expect()
    T = sum(count)
    want = tuple(x[:T] for x in want)
    out, lse = batch.call(ctx, most_tokens=max(count), most_keys=max(s + c for s, c in zip(start, count)))
    compare((out, lse), want)
    assert bool((out[T:] == 9.0).all() and (lse[T:] == 9.0).all()) and ctx.status() == 0
    again = batch.call(ctx, out=batch.q)                                        # the queries' own place, without hints
    compare(again, want)


@pytest.mark.parametrize("kw", [{"window": 1500, "sinks": 40}, {"causal": False}, {"scale": -0.3}])
def test_a_last_round_otherwise(ctx, kw):
    batch = Batch([2500], [521], 128, 16, 128, 16)
    check(ctx, batch, **kw)


def test_a_last_round_with_holes_and_junk(ctx):
    """Its keys miss a page; values that only some rows see are not finite."""
    from paper_2605_07330_amd import srs
    batch = Batch([1500], [521], 128, 16, 128, 16)
    first, last = batch.table[0, 1503 // 16].item(), batch.table[0, 2020 // 16].item()
    batch.v[first, 1503 % 16, 2, 7] = math.inf
    batch.v[last, 2020 % 16, 3] = math.nan
    batch.table[0, 40] = -1
    check(ctx, batch, flags=srs.FLAG_BAD_INDEX)


def test_sixty_four_requests_of_all_lengths(ctx):
    """As many as are put in order by the length of their keys; equal lengths and empty requests among them."""
    start = [(r * 37) % 300 if r % 5 else 128 for r in range(64)]
    count = [(0, 1, 3, 40, 70, 129)[r % 6] for r in range(64)]
    check(ctx, Batch(start, count, 8, 2, 64, 16))
    check(ctx, Batch(start + [9], count + [33], 8, 2, 64, 16))                  # one more


def test_a_last_round_from_a_graph(ctx):
    from paper_2605_07330_amd import srs
    batch = Batch([1500], [521], 128, 16, 128, 16)
    want = batch.expect()
    out, lse = torch.full_like(batch.q, 9.0), torch.full(batch.q.shape[:2], 9.0, device=DEV)
    need = srs.attention_workspace(1, 521, 128, 16, 128, batch.table.shape[1], 16, most_tokens=521, most_keys=2021)
    assert need
    room = torch.empty(need, dtype=torch.uint8, device=DEV)
    call = lambda: batch.call(ctx, out=out, lse=lse, most_tokens=521, most_keys=2021, workspace=room)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        out.fill_(9.0)
        lse.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        compare((out, lse), want)
    assert ctx.status() == 0


def test_offsets_beyond_32_bits(ctx):
    """A cache of more than 2^32 elements, its last pages in use."""
    pages, page, hkv, d = 2**32 // (1024 * 128) + 40, 64, 16, 128
    b = Batch([200, 90], [1, 60], 16, hkv, d, page)
    k, v = b.k, b.v
    big = torch.empty(pages, page, hkv, d, dtype=b.dtype, device=DEV)
    big_v = torch.empty(pages, page, hkv, d, dtype=b.dtype, device=DEV)
    big[-b.pages:], big_v[-b.pages:] = k, v
    want = b.expect()
    b.table = torch.where(b.table >= 0, b.table + (pages - b.pages), b.table)
    b.k, b.v = big, big_v
    compare(b.call(ctx), want)
    assert ctx.status() == 0


@pytest.mark.parametrize("start,count", [([900, 400, 5000], [1, 1, 1]), ([900, 400, 5000], [1, 200, 9])])
def test_from_a_graph(ctx, start, count):
    """Replays on new queries, lengths and tables, with the program's own work between them, two graphs taking turns."""
    one, two = Batch(start, count, 8, 2, 128, 16, seed=1), Batch(start[::-1], count, 8, 2, 128, 16, seed=2)
    outs, graphs = [], []
    for b in (one, two):
        out, lse = torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device=DEV)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            b.call(ctx, out=out, lse=lse)
        outs.append((out, lse)), graphs.append(graph)
    for step in range(4):
        for b, graph, (out, lse) in zip((one, two), graphs, outs):
            b.q.copy_(torch.randn(b.q.shape, device=DEV))
            b.at.sub_(step)
            b.start = [s - step for s in b.start]
            out.fill_(3.0)
            graph.replay()
            want = b.expect()
            eager = b.call(ctx)
            torch.cuda.synchronize()
            compare((out, lse), want)
            assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
    assert ctx.status() == 0


def test_on_another_stream(ctx):
    b = Batch([900, 400, 9000], [1, 20, 1], 8, 2, 128, 16)
    want = b.expect()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [b.call(ctx, stream=side, out=torch.zeros_like(b.q)) for _ in range(3)]
    side.synchronize()
    for g in got:
        compare(g, want)
    with torch.cuda.stream(side):
        got = b.call(ctx)
    side.synchronize()
    compare(got, want)
    assert ctx.status(side) == 0


def test_workspace_of_the_callers(ctx):
    from paper_2605_07330_amd import srs
    b = Batch([9000, 400], [1, 1], 8, 2, 128, 16)
    want = b.expect()
    hints = {"most_tokens": 1, "most_keys": 9001}
    need = srs.attention_workspace(2, 2, 8, 2, 128, b.table.shape[1], 16, **hints)
    room = torch.full((need + 512,), 0x5A, dtype=torch.uint8, device=DEV)
    compare(b.call(ctx, workspace=room[256:256 + need], **hints), want)
    assert bool((room[:256] == 0x5A).all()) and bool((room[256 + need:] == 0x5A).all())
    if need:
        for small in (room[:need - 1], room[8:8 + need + 8]):             # too small, not aligned
            with pytest.raises(srs.SrsError):
                b.call(ctx, workspace=small, **hints)
    assert ctx.status() == 0


def test_refusals(ctx):
    from paper_2605_07330_amd import srs
    b = Batch([30, 4], [1, 2], 8, 2, 64, 16)
    out = torch.full_like(b.q, 9.0)
    good = dict(q=b.q, out=out, k_cache=b.k, v_cache=b.v, table=b.table, token_begin=b.begin, start=b.at)
    for kw in ({"q": b.q.half()}, {"q": b.q[:, :, :32]}, {"q": b.q.cpu()}, {"out": out[:1]}, {"k_cache": b.k[:1]}, {"k_cache": b.k.half()}, {"table": b.table[0]},
               {"table": b.table[:1]}, {"table": b.table.long()}, {"start": b.at.float()}, {"token_begin": b.begin[:2]}, {"lse": torch.zeros(2, device=DEV)},
               {"lse": torch.zeros(3, 8, dtype=torch.float64, device=DEV)}, {"q": b.q.transpose(1, 2)}):
        with pytest.raises((TypeError, ValueError)):
            ctx.cache_attention(**{**good, **kw})
    odd = torch.randn(3, 8, 65, device=DEV).bfloat16()[..., :64]
    for kw in ({"window": -1}, {"sinks": 3}, {"window": 4, "causal": False}, {"scale": float("nan")}, {"most_keys": -1}, {"q": odd}, {"out": odd},
               {"q": b.q[:, :7], "out": out[:, :7]}, {"out": out[:, :4]}):
        with pytest.raises(srs.SrsError):
            ctx.cache_attention(**{**good, **kw})
    single = {"q": b.q.float(), "out": out.float(), "k_cache": b.k.float(), "v_cache": b.v.float()}
    wide = {n: torch.zeros(*t.shape[:-1], 264, dtype=t.dtype, device=DEV) for n, t in (("q", b.q), ("out", out), ("k_cache", b.k), ("v_cache", b.v))}
    for kw in (single, wide):
        with pytest.raises(srs.SrsError):
            ctx.cache_attention(**{**good, **kw})
    torch.cuda.synchronize()
    assert bool((out == 9.0).all()) and ctx.status() == 0


def test_a_synchronisation_and_what_follows(ctx):
    """The calls together: requests are admitted and decode step by step; then their weights change, every cached key and value is
    computed again in chunks in the same pages, and decoding goes on.  Against attention over plain dense keys in 64 bits."""
    from paper_2605_07330_amd import srs
    R, hq, hkv, d, page, width, hidden = 5, 8, 2, 64, 16, 12, 32
    g = torch.Generator(device=DEV).manual_seed(5)
    i32 = dict(dtype=torch.int32, device=DEV)
    inv, magnitude = srs.rope_frequencies(d, 1e4, device=DEV)
    free, left = torch.randperm(40, generator=g, device=DEV).int(), torch.tensor([40], **i32)
    held, table = torch.zeros(R, **i32), torch.full((R, width), -1, **i32)
    kc, vc = (torch.full((40, page, hkv, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    W = (torch.randn(hidden, (hq + 2 * hkv) * d, generator=g, device=DEV) * hidden**-0.5).bfloat16()
    W_roll = W.clone()
    tokens = torch.randn(R, width * page, hidden, generator=g, device=DEV).bfloat16()        # of every request, in order

    def project(x):
        return (x.float() @ W_roll.float()).bfloat16().view(-1, hq + 2 * hkv, d)

    def step(start, count, padded):
        T = sum(count)
        begin, slots, positions = torch.zeros(R + 1, **i32), torch.zeros(padded, dtype=torch.int64, device=DEV), torch.zeros(padded, **i32)
        at = torch.tensor(start, **i32)
        ctx.cache_tables(at, torch.tensor(count, **i32), page, held, table, free, left, begin, slots, positions)
        x = torch.cat([tokens[r, s:s + c] for r, (s, c) in enumerate(zip(start, count))] + [tokens[0, :padded - T]])
        rows = project(x)
        q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        turned = torch.empty(padded, hq, d, dtype=torch.bfloat16, device=DEV)
        ctx.cache_write(k, v, kc, vc, slots, q=q, q_out=turned, positions=positions, inv_freq=inv, magnitude=magnitude)
        out = torch.full_like(turned, 9.0)
        ctx.cache_attention(turned, out, kc, vc, table, begin, at)
        assert ctx.status() == 0
        assert bool((out[T:] == 9.0).all())
        # dense: every token of each request so far, projected with the weights as they are
        t = 0
        for r, (s, c) in enumerate(zip(start, count)):
            n = s + c
            if not c:
                continue
            allrows = project(tokens[r, :n]).double()
            a = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * inv[None]
            co, si = a.cos()[:, None], a.sin()[:, None]

            def turn(y):
                y1, y2 = y[..., :d // 2], y[..., d // 2:]
                return torch.cat([y1 * co - y2 * si, y2 * co + y1 * si], -1)
            Q, K, V = turn(allrows[:, :hq])[s:], turn(allrows[:, hq:hq + hkv]), allrows[:, hq + hkv:]
            K, V = K.repeat_interleave(hq // hkv, 1), V.repeat_interleave(hq // hkv, 1)
            score = torch.matmul(Q.transpose(0, 1), K.permute(1, 2, 0).contiguous()) * d**-0.5
            hide = torch.arange(n, device=DEV)[None] > (s + torch.arange(c, device=DEV))[:, None]
            size = torch.matmul(Q.transpose(0, 1).abs(), K.permute(1, 2, 0).abs().contiguous()) * d**-0.5
            w = score.masked_fill(hide, -math.inf).softmax(-1)
            want, A = (w @ V.transpose(0, 1)).transpose(0, 1), (w @ V.transpose(0, 1).abs()).transpose(0, 1)
            B = size.masked_fill(hide, 0.0).amax(-1).transpose(0, 1)[..., None]
            h = 2.0**-8
            # queries and keys are rounded once each after turning: scores off by 2 h B (and the h^2), weights by e^2 of it; then as above
            tol = h * want.abs() + A * (2 * h + torch.expm1(2 * (2 * h + h * h) * B) + (d + 8) * 2.0**-23 * B + 2.0**-20)
            off = ((out[t:t + c].double() - want).abs() - tol).max()
            assert off <= 0, (r, s, c, off.item())
            t += c

    length = [30, 0, 17, 64, 5]
    step([0] * R, length, 130)                                       # prompts
    for _ in range(6):
        count = [1, 0, 1, 1, 1]
        step(length, count, 8)
        length = [a + b for a, b in zip(length, count)]
    pages_before, held_before = table.clone(), held.clone()
    # the synchronisation: one weight in ten changes, and travels as indices and values
    new = torch.where(torch.rand(W.shape, generator=g, device=DEV) < 0.1, (W.float() * 1.5 + 0.05).bfloat16(), W)
    I, V, counts = srs.alloc_payload(1, W.numel(), DEV)
    ctx.extract(W.view(-1), new.view(-1), W.numel(), I, V, counts, W.numel())
    ctx.apply(W_roll.view(-1), W.numel(), I, V, counts, W.numel())
    assert torch.equal(W_roll, new) and ctx.status() == 0
    done = [0] * R                                                   # every token again, in chunks
    while done != length:
        count = [min(n - a, 25) for n, a in zip(length, done)]
        step(done, count, 128)
        done = [a + b for a, b in zip(done, count)]
    assert torch.equal(table, pages_before) and torch.equal(held, held_before)
    for _ in range(3):
        step(length, [1] * R, 5)
        length = [a + 1 for a in length]
    ctx.cache_release(torch.zeros(R, **i32), held, table, free, left)
    assert ctx.status() == 0 and left.item() == 40 and sorted(free.tolist()) == list(range(40)) and not bool(held.any())
