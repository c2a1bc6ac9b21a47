"""Attention's weights over their whole range, and in the two parts that few new tokens are promised, against 64 bits.

How far a result may be off, with A = sum_j p_j |v_j| over a row's normalised weights, B its largest |score| and n its keys:
* the queries here have one element that is not 0, so scores are single products, which binary32 holds; the exponential's argument in
  another base adds 2^-22 B, the exponential 2^-22; weights are off by that relatively, so twice it with the sum's;
* a weight is rounded once to the element type where a request has many new tokens, half a step h, relatively, and the same again in
  the sum at worst: 2 h.  Where it has few it is carried as value and remainder, each rounded: 2 h^2;
* sums add n 2^-24, joining and division 2^-21;
* the output is rounded once: h |o|, or 2^-25 where a half has no smaller steps;
* weights below 2^-126 of the largest are 0.
None of it depends on how far a weight lies below the largest, as long as that is not beyond 2^126."""
import math

import pytest
import torch

from test_gpu_cache_attention import DEV, HALF_STEP, Batch, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def dense(b, r):
    page, place, _ = b.places(r)
    return page, place


def exact(b, r, scale, parts):
    """out and bound of request r, rows by heads by d, in 64 bits."""
    page, place = dense(b, r)
    h, group, start = HALF_STEP[b.dtype], b.hq // b.hkv, b.start[r]
    begin = int(b.begin[r])
    q = b.q[begin:begin + b.count[r]].double()
    k, v = b.k[page, place].double(), b.v[page, place].double()
    j = torch.arange(k.shape[0], device=DEV)
    seen = j[None] <= start + torch.arange(q.shape[0], device=DEV)[:, None]
    out, tol = torch.zeros_like(q), torch.zeros_like(q)
    for head in range(b.hq):
        kk, vv = k[:, head // group], v[:, head // group]
        s = (q[:, head] @ kk.t().contiguous() * scale).masked_fill(~seen, -math.inf)
        B = (q[:, head].abs() @ kk.abs().t().contiguous() * abs(scale)).masked_fill(~seen, 0.0).amax(1, keepdim=True)
        p = s.softmax(1)
        o, A = p @ vv, p @ vv.abs()
        score = 2.0**-22 * B + 2.0**-22
        n = seen.sum(1, keepdim=True)
        out[:, head] = o
        tol[:, head] = h * o.abs() + A * ((2 * h * h if parts else 2 * h) + 2 * score + n * 2.0**-24 + 2.0**-21) + 2.0**-126 * vv.abs().sum(0)
        if b.dtype == torch.float16:
            tol[:, head] += 2.0**-25
    return out, tol


def compare(ctx, b, scale, **kw):  # noqa: F811
    out, _ = b.call(ctx, scale=scale, **kw)
    narrow = max(1, 16 // (b.hq // b.hkv))
    for r in range(len(b.start)):
        begin = int(b.begin[r])
        want, tol = exact(b, r, scale, b.count[r] <= narrow)
        off = ((out[begin:begin + b.count[r]].double() - want).abs() - tol).max().item()
        assert off <= 0, f"request {r}: off by {off} beyond the bound"
    assert ctx.status() == 0


KINDS = [([8000], [1]), ([300, 8000], [1, 2]), ([8000], [40]), ([500], [130])]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("gap", [6, 11, 14, 17, 20, 24, 30, 36])
@pytest.mark.parametrize("start,count", KINDS)
def test_one_key_takes_the_weight_and_adds_nothing(ctx, dtype, gap, start, count):  # noqa: F811
    """The first key's value is 0 and its weight the largest; what the others add, e^-gap and less each, is the whole result."""
    b = Batch(start, count, 8, 2, 64, 16, dtype, seed=gap)
    g = torch.Generator(device=DEV).manual_seed(gap)
    b.q.zero_()
    b.q[..., 0] = 1.0
    b.k.zero_()
    b.k[..., 0] = -(gap + torch.rand(b.k.shape[:3], generator=g, device=DEV) * 2).to(dtype)
    b.v[:] = (1000 * (1 + torch.rand(b.v.shape, generator=g, device=DEV))).to(dtype)
    for r in range(len(start)):
        page, place = dense(b, r)
        b.k[page[0], place[0]], b.v[page[0], place[0]] = 0.0, 0.0
    compare(ctx, b, 1.0)
    compare(ctx, b, 1.0, most_tokens=max(count), most_keys=max(start) + max(count))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 128, 16), (4, 4, 64, 24), (6, 2, 80, 16), (4, 2, 256, 64)])
@pytest.mark.parametrize("start,count", KINDS[1:])
def test_weights_of_every_size(ctx, dtype, hq, hkv, d, page, start, count):  # noqa: F811
    """Scores over 60 nats; the larger a weight, the smaller its value, so that no few keys decide."""
    b = Batch(start, count, hq, hkv, d, page, dtype, seed=3)
    g = torch.Generator(device=DEV).manual_seed(9)
    b.q.zero_()
    b.q[..., 1] = 1.0
    b.k.zero_()
    score = -60.0 * torch.rand(b.k.shape[:3], generator=g, device=DEV)
    b.k[..., 1] = score.to(dtype)
    grow = (60000.0 * torch.exp(-score - 30.0)).clamp(max=60000.0)[..., None]
    b.v[:] = (grow * torch.rand(b.v.shape, generator=g, device=DEV)).to(dtype)
    compare(ctx, b, 1.0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hq,hkv,d,start", [(8, 2, 128, [3, 20, 50]), (32, 8, 128, [40]), (4, 4, 64, [7, 60]), (16, 1, 256, [33, 12]), (6, 2, 80, [30])])
def test_few_tokens_have_weights_in_two_parts(ctx, dtype, hq, hkv, d, start):  # noqa: F811
    """Values come in pairs of opposite sign behind keys that are nearly alike, so that the result is small beside what it is the sum of and its own
    rounding hides nothing: weights rounded once would be seen, which the oracle with such weights shows first."""
    b = Batch(start, [1] * len(start), hq, hkv, d, 16, dtype, seed=d)
    g = torch.Generator(device=DEV).manual_seed(d)
    b.q.zero_()
    b.q[..., 2] = 1.0
    b.k.zero_()
    b.k[..., 2] = (-2.0 * torch.rand(b.k.shape[:3], generator=g, device=DEV)).to(dtype)
    for r in range(len(start)):
        page, place = dense(b, r)
        n = page.numel() // 2 * 2
        b.k[page[1:n:2], place[1:n:2], :, 2] = 1.03125 * b.k[page[0:n:2], place[0:n:2], :, 2]
        b.v[page[1:n:2], place[1:n:2]] = -b.v[page[0:n:2], place[0:n:2]]
        if page.numel() % 2:
            b.v[page[-1], place[-1]] = 0.0
    for r in range(len(start)):
        want, tol = exact(b, r, 1.0, True)
        page, place = dense(b, r)
        seen = False
        for head in range(hq):
            s = b.q[r:r + 1, head].double() @ b.k[page, place, head // (hq // hkv)].double().t().contiguous()
            p = (s - s.amax()).exp()
            once = p.to(dtype).double() @ b.v[page, place, head // (hq // hkv)].double() / p.sum()
            seen |= bool(((once - want[:, head]).abs() > tol[:, head]).any())
        assert seen, "the data would not show weights that are rounded once"
    compare(ctx, b, 1.0)
