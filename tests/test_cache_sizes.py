"""Sizes beyond 32 bits at the cache calls of the binding, without a GPU: they are refused, whatever their lower bits say.  The library gets 32
bits of each and could not tell; here it only records that it was called."""
import types

import pytest
import torch

BIG = 2**32


@pytest.fixture()
def srs(monkeypatch):
    from paper_2605_07330_amd import srs as module
    calls = []
    real = module._lib

    def recorder(name, result):
        return lambda *a: calls.append(name) or result
    fake = types.SimpleNamespace(srs_strerror=real.srs_strerror, srs_cache_attention_workspace=recorder("workspace", 0),
                                 **{n: recorder(n, module.OK) for n in ("srs_cache_tables", "srs_cache_release", "srs_rope", "srs_cache_write", "srs_cache_attention")})
    monkeypatch.setattr(module, "_lib", fake)
    monkeypatch.setattr(module, "_native", lambda *a: False)
    for name, stub in (("_stream", lambda self, s: 0), ("_here", lambda self, t, what, dtype, at_least=0: 0x1000),
                       ("_rows", lambda self, t, what, tokens, d, dtype: module.Rows(0x1000, 1, 8, 8)), ("_cache", lambda self, k, v: module.Cache(heads=2, page_tokens=16))):
        monkeypatch.setattr(module.Context, name, stub)
    ctx = module.Context.__new__(module.Context)
    ctx._h, ctx.device = None, 0
    yield types.SimpleNamespace(module=module, ctx=ctx, calls=calls)
    ctx._h = None
    monkeypatch.setattr(module, "_lib", real)


def refused(srs, call, name):
    with pytest.raises(srs.module.SrsError) as e:
        call()
    assert e.value.code == srs.module.ERR_INVALID and name not in srs.calls


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def wide(heads, dtype=torch.bfloat16):
    """[1, heads, 8] without the memory."""
    return torch.zeros(1, 1, 8, dtype=dtype).expand(1, heads, 8)


def test_tables(srs):
    call = lambda page, free=ints(4): srs.ctx.cache_tables(ints(3), ints(3), page, ints(3), ints(3, 4), free, ints(1), ints(4), torch.zeros(9, dtype=torch.int64), ints(9))
    call(16)
    assert srs.calls == ["srs_cache_tables"]
    srs.calls.clear()
    for page in (BIG + 16, 2**31, -16, 2**64 + 16):
        refused(srs, lambda: call(page), "srs_cache_tables")
    refused(srs, lambda: call(16, ints(1).expand(BIG + 4)), "srs_cache_tables")


def test_release(srs):
    refused(srs, lambda: srs.ctx.cache_release(ints(3), ints(3), ints(3, 4), ints(1).expand(BIG + 4), ints(1)), "srs_cache_release")


def test_rope(srs):
    freq = torch.zeros(4, dtype=torch.float64)
    srs.ctx.rope(wide(2), wide(2), ints(1), freq)
    assert srs.calls == ["srs_rope"]
    srs.calls.clear()
    refused(srs, lambda: srs.ctx.rope(wide(BIG + 2), wide(BIG + 2), ints(1), freq), "srs_rope")
    refused(srs, lambda: srs.ctx.rope(wide(2), wide(2), ints(1), freq[:1].expand(2**31 + 2)), "srs_rope")


def test_write(srs):
    cache, slots = torch.zeros(4, 16, 2, 8, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int64)
    srs.ctx.cache_write(wide(2), wide(2), cache, cache, slots)
    assert srs.calls == ["srs_cache_write"]
    srs.calls.clear()
    refused(srs, lambda: srs.ctx.cache_write(wide(BIG + 2), wide(2), cache, cache, slots), "srs_cache_write")
    refused(srs, lambda: srs.ctx.cache_write(wide(2), wide(2), cache[:1].expand(BIG + 4, 16, 2, 8), cache, slots), "srs_cache_write")
    freq = torch.zeros(4, dtype=torch.float64)
    refused(srs, lambda: srs.ctx.cache_write(wide(2), wide(2), cache, cache, slots, q=wide(BIG + 8), q_out=wide(BIG + 8), positions=ints(1), inv_freq=freq), "srs_cache_write")


def test_attention(srs):
    cache = torch.zeros(4, 16, 2, 8, dtype=torch.bfloat16)
    call = lambda heads=2, **kw: srs.ctx.cache_attention(wide(heads), wide(heads), cache, cache, ints(1, 4), ints(2), ints(1), **kw)
    call(window=5, sinks=2, most_tokens=2**62, most_keys=2**64 - 1)
    assert "srs_cache_attention" in srs.calls
    srs.calls.clear()
    for kw in ({"window": BIG + 16}, {"window": 4, "sinks": BIG}, {"window": 2**31}, {"most_tokens": 2**64 + 1}, {"most_keys": 2**64}, {"most_keys": -1}, {"window": -3}):
        refused(srs, lambda: call(**kw), "srs_cache_attention")
    refused(srs, lambda: call(heads=BIG + 2), "srs_cache_attention")


def test_workspace(srs):
    good = dict(nrequests=1, tokens=1, q_heads=4, kv_heads=2, head_dim=64, table_width=8192, page_tokens=16)
    srs.module.attention_workspace(**good)
    assert srs.calls == ["workspace"]
    srs.calls.clear()
    for kw in [{n: v + BIG} for n, v in good.items()] + [{"window": BIG + 5}, {"sinks": BIG}, {"tokens": -1}, {"most_keys": 2**64 + 3}]:
        refused(srs, lambda: srs.module.attention_workspace(**{**good, **kw}), "workspace")
