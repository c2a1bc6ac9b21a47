"""Refusals of the cache calls at the C entry, without a GPU: every argument is checked before anything touches a device.  The handle is a
block of zeros, which names device 0 and nothing else; a call whose arguments are accepted then ends at the device that is not there."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would reach the device with addresses that are none")


@pytest.fixture(scope="module")
def srs():
    from paper_2605_07330_amd import srs as module
    return module


CTX = C.create_string_buffer(4096)
A = 0x100000                    # an address, aligned to everything


def refused(srs, name, good, changes, accepted):
    call = getattr(srs._lib, name)
    assert call(*good.values()) == srs.ERR_HIP, "the call that should be accepted"
    for change in accepted:
        assert call(*{**good, **change}.values()) in (srs.ERR_HIP, srs.OK), change
    for change in changes:
        assert call(*{**good, **change}.values()) == srs.ERR_INVALID, change


def test_tables(srs):
    good = dict(ctx=CTX, start=A, count=A, n=3, page=16, held=A, table=A, width=4, free=A, left=A, cap=9, begin=A, slots=A, positions=A, most=20, stream=None)
    refused(srs, "srs_cache_tables", good,
            [{"ctx": None}, {"start": None}, {"count": None}, {"held": None}, {"table": None}, {"free": None}, {"left": None}, {"begin": None},
             {"slots": None}, {"positions": None}, {"page": 0}, {"width": 2**28}, {"most": 2**31}, {"cap": 2**31}, {"n": 2**31},
             {"slots": A + 4}, {"start": A + 2}, {"table": A + 1}, {"begin": A + 2}],
            [{"n": 0, "start": None, "count": None, "held": None, "table": None}, {"width": 0, "table": None}, {"cap": 0, "free": None},
             {"most": 0, "slots": None, "positions": None}, {"width": 2**27 - 1}])


def test_release(srs):
    good = dict(ctx=CTX, keep=A, n=3, held=A, table=A, width=4, free=A, left=A, cap=9, stream=None)
    refused(srs, "srs_cache_release", good,
            [{"ctx": None}, {"keep": None}, {"held": None}, {"table": None}, {"free": None}, {"left": None}, {"keep": A + 1}, {"cap": 2**31}, {"n": 2**31}],
            [{"n": 0}, {"width": 0, "table": None}, {"cap": 0, "free": None}])


def rows(srs, p=A, heads=4, token=256, head=64):
    return C.byref(srs.Rows(p, heads, token, head))


def test_rope(srs):
    good = dict(ctx=CTX, dtype=0, x=rows(srs), out=rows(srs), tokens=5, d=64, positions=A, freq=A, rot=64, flags=0, magnitude=1.0, stream=None)
    refused(srs, "srs_rope", good,
            [{"ctx": None}, {"dtype": 3}, {"dtype": -1}, {"x": None}, {"out": None}, {"x": rows(srs, heads=3)}, {"x": rows(srs, p=None)}, {"x": rows(srs, p=A + 1)},
             {"positions": None}, {"freq": None}, {"freq": A + 4}, {"rot": 63}, {"rot": 66}, {"flags": 4}, {"magnitude": float("nan")}, {"tokens": 2**31},
             {"d": 0}, {"x": rows(srs, heads=0), "out": rows(srs, heads=0)}, {"out": rows(srs, token=2**41)}, {"dtype": 2, "x": rows(srs, p=A + 2)}],
            [{"tokens": 0, "x": None, "out": None}, {"rot": 0, "positions": None, "freq": None}, {"dtype": 2}, {"flags": 3}, {"x": rows(srs, p=A + 2, token=-3, head=0)}])


def cache(srs, **kw):
    return C.byref(srs.Cache(**{**dict(k=A, v=A, dtype=0, pages=7, page_tokens=16, heads=2, head_dim=64, k_page=2048, k_token=128, k_head=64,
                                       v_page=2048, v_token=128, v_head=64), **kw}))


def test_write(srs):
    two = rows(srs, heads=2)
    good = dict(ctx=CTX, cache=cache(srs), k=two, v=two, tokens=5, slots=A, q=rows(srs), q_out=rows(srs), positions=A, freq=A, rot=64, flags=0, magnitude=1.0, stream=None)
    refused(srs, "srs_cache_write", good,
            [{"ctx": None}, {"cache": None}, {"cache": cache(srs, k=None)}, {"cache": cache(srs, dtype=5)}, {"cache": cache(srs, page_tokens=0)}, {"cache": cache(srs, heads=0)},
             {"cache": cache(srs, head_dim=0)}, {"cache": cache(srs, v=A + 1)}, {"cache": cache(srs, pages=2**31)}, {"k": rows(srs)}, {"v": rows(srs)}, {"k": None}, {"slots": None},
             {"slots": A + 4}, {"q_out": None}, {"q_out": rows(srs, heads=3)}, {"positions": None}, {"freq": None}, {"rot": 65}, {"rot": 66}, {"flags": 8}, {"tokens": 2**31},
             {"cache": cache(srs, k_page=2**41)}],
            [{"tokens": 0}, {"q": None, "q_out": None}, {"rot": 0, "positions": None, "freq": None, "q_out": None}, {"cache": cache(srs, pages=0)}, {"cache": cache(srs, k=A + 2, k_token=129)}])


def test_attention(srs):
    good = dict(ctx=CTX, cache=cache(srs), q=rows(srs), out=rows(srs), lse=A, tokens=5, begin=A, start=A, table=A, width=4, n=3, scale=0.1, flags=0, window=0, sinks=0,
                most_tokens=5, most_keys=64, workspace=A, bytes=1 << 30, stream=None)
    refused(srs, "srs_cache_attention", good,
            [{"ctx": None}, {"cache": None}, {"cache": cache(srs, dtype=2)}, {"cache": cache(srs, k=A + 8)}, {"cache": cache(srs, head_dim=60)}, {"cache": cache(srs, head_dim=264)},
             {"cache": cache(srs, k_token=132)}, {"cache": cache(srs, v_head=4)}, {"cache": cache(srs, heads=3)}, {"q": None}, {"out": None}, {"q": rows(srs, p=A + 8)},
             {"q": rows(srs, token=260)}, {"out": rows(srs, heads=2)}, {"begin": None}, {"start": None}, {"table": None}, {"lse": A + 2}, {"scale": float("inf")}, {"flags": 2},
             {"sinks": 3}, {"flags": 1, "window": 5}, {"window": 2**31}, {"tokens": 2**31}, {"n": 2**31}, {"width": 2**28}, {"begin": A + 2}],
            [{"tokens": 0}, {"n": 0}, {"lse": None}, {"window": 5, "sinks": 3}, {"flags": 1}, {"most_tokens": 0, "most_keys": 0}, {"most_tokens": 2**62, "most_keys": 2**62},
             {"cache": cache(srs, pages=0)}, {"width": 0, "table": None}])


def test_a_split_needs_its_workspace(srs):
    """One row over a long axis."""
    shape = dict(nrequests=1, tokens=1, q_heads=4, kv_heads=2, head_dim=64, table_width=8192, page_tokens=16)
    need = srs.attention_workspace(**shape, most_tokens=1, most_keys=100000)
    assert srs.attention_workspace(**{**shape, "tokens": 0}) == srs.attention_workspace(**{**shape, "nrequests": 0}) == 0
    assert srs.attention_workspace(**shape, most_tokens=1, most_keys=10) == 0
    good = dict(ctx=CTX, cache=cache(srs), q=rows(srs), out=rows(srs), lse=A, tokens=1, begin=A, start=A, table=A, width=8192, n=1, scale=0.1, flags=0, window=0, sinks=0,
                most_tokens=1, most_keys=100000, workspace=A, bytes=need, stream=None)
    call = srs._lib.srs_cache_attention
    assert call(*good.values()) == srs.ERR_HIP
    if need:
        for change in ({"bytes": need - 1}, {"workspace": None}, {"workspace": A + 8}):
            assert call(*{**good, **change}.values()) == srs.ERR_INVALID
