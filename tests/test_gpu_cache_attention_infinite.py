"""Values that are not finite behind weights that are next to nothing, against 64 bits: a row that sees such a value is itself not finite there,
whichever way its keys are shared out and however far the value's score lies below the row's largest.  Bounds as in
test_gpu_cache_attention."""
import math

import pytest
import torch

from test_gpu_cache_attention import DEV, Batch, check, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


def sloped(start, count, hq, hkv, d, page, dtype, gap, top, seed=0):
    """Scores of -gap to -gap - 1, of 0 at key `top` of each request."""
    b = Batch(start, count, hq, hkv, d, page, dtype, seed=seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    b.q.zero_()
    b.q[..., 3] = 1.0
    b.k.zero_()
    b.k[..., 3] = (-gap - torch.rand(b.k.shape[:3], generator=g, device=DEV)).to(dtype)
    for r in range(len(start)):
        page_of, place, _ = b.places(r)
        b.k[page_of[top], place[top]] = 0.0
    return b


def put(b, r, key, head, element, value):
    page, place, _ = b.places(r)
    b.v[page[key], place[key], head, element] = value


# few and many new tokens, with and without parts, and a last round that is shared out
SHAPES = [([300, 90], [1, 2], 8, 2, 128, 16), ([9000, 700], [1, 1], 8, 2, 64, 16), ([700], [3], 4, 2, 80, 24), ([600], [1], 4, 2, 256, 16),
          ([300, 400], [40, 130], 8, 2, 128, 16), ([300], [70], 6, 2, 72, 24), ([4000], [40], 8, 2, 64, 16), ([500], [40], 4, 2, 256, 16),
          ([1000], [1029], 64, 64, 128, 16)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("gap", [4, 26, 60, 100])
@pytest.mark.parametrize("top", [2, 80])
@pytest.mark.parametrize("start,count,hq,hkv,d,page", SHAPES)
def test_infinite_values_of_small_weight(ctx, dtype, gap, top, start, count, hq, hkv, d, page):  # noqa: F811
    """In front of the row's largest score and behind it, in its tile and in others, alone and of both signs."""
    b = sloped(start, count, hq, hkv, d, page, dtype, gap, top, seed=gap)
    for r in range(len(start)):
        last = start[r] - 1
        put(b, r, 5, 0, 1, math.inf)
        put(b, r, last, 0, 2, -math.inf)
        put(b, r, 0, hkv - 1, 4, math.inf)
        put(b, r, last - 20, hkv - 1, 4, -math.inf)
        put(b, r, 70, 0, d - 1, math.nan)
    check(ctx, b, scale=1.0, hints=(True,) if count == [1029] else (True, False))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("count", [1, 60])
def test_infinite_values_under_a_window(ctx, dtype, count):  # noqa: F811
    b = sloped([2000], [count], 8, 2, 128, 16, dtype, 100, 1900, seed=count)
    for key, element in ((1, 0), (1200, 1), (1930, 2), (1999, 3), (2000 + count - 1, 4)):
        put(b, 0, key, 1, element, math.inf)
    check(ctx, b, scale=1.0, window=700, sinks=3)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("start,count,hq,hkv,d,page", SHAPES[:-1])
def test_scores_of_minus_infinity(ctx, dtype, start, count, hq, hkv, d, page):  # noqa: F811
    """Keys with such scores weigh nothing; a row with no others is taken as one that sees no key."""
    b = sloped(start, count, hq, hkv, d, page, dtype, 5, 2)
    for r in range(len(start)):
        page_of, place, _ = b.places(r)
        b.k[page_of[::3], place[::3], :, 3] = -math.inf
    check(ctx, b, scale=1.0)
    b.k[..., 3] = -math.inf
    out, lse = b.call(ctx, scale=1.0)
    assert not bool(out.any()) and bool((lse == -math.inf).all()) and ctx.status() == 0
