"""Sizes beyond 32 bits at the cache calls, through the C++ checks and through ctypes: refused, and nothing is written."""
import pytest
import torch

srs = pytest.importorskip("paper_2605_07330_amd.srs")

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("size", [2**31, 2**32 + 16, 2**64 + 16])
def test_refused(monkeypatch, native, size):
    if not native:
        monkeypatch.setattr(srs, "_native", lambda *a: False)
    ctx, i32 = srs.Context(0), dict(dtype=torch.int32, device=DEV)
    start, count, held, table = torch.tensor([0, 3], **i32), torch.tensor([2, 1], **i32), torch.zeros(2, **i32), torch.full((2, 4), -1, **i32)
    free, left, begin = torch.arange(6, **i32), torch.tensor([6], **i32), torch.zeros(3, **i32)
    slots, positions = torch.full((3,), 7, dtype=torch.int64, device=DEV), torch.full((3,), 7, **i32)
    q, out = torch.ones(3, 4, 64, dtype=torch.bfloat16, device=DEV), torch.full((3, 4, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    cache = torch.ones(6, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    begin[1:] = torch.tensor([2, 3], **i32)
    attention = dict(table=table, token_begin=begin, start=start)
    calls = [lambda: ctx.cache_tables(start, count, size, held, table, free, left, begin, slots, positions),
             lambda: ctx.cache_attention(q, out, cache, cache, **attention, window=size),
             lambda: ctx.cache_attention(q, out, cache, cache, **attention, window=4, sinks=size)]
    if size >= 2**64:
        calls += [lambda: ctx.cache_attention(q, out, cache, cache, **attention, most_tokens=size), lambda: ctx.cache_attention(q, out, cache, cache, **attention, most_keys=size)]
    for call in calls:
        with pytest.raises(srs.SrsError) as e:
            call()
        assert e.value.code == srs.ERR_INVALID
    torch.cuda.synchronize()
    assert bool((slots == 7).all() and (positions == 7).all() and (table == -1).all() and (out == 9.0).all()) and left.item() == 6
    assert ctx.status() == 0
    ctx.close()
