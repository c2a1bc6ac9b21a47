"""Attention's scale at the C entry, without a GPU: the kernels take it times log2(e), so one that is finite, but not so, is refused."""
import pytest
import torch

from test_cache_arguments import A, CTX, cache, rows, srs  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="accepted calls would reach the device with addresses that are none")


@pytest.mark.parametrize("scale,code", [(2.3e38, "ERR_HIP"), (-2.3e38, "ERR_HIP"), (2.4e38, "ERR_INVALID"), (-2.4e38, "ERR_INVALID"), (3.4e38, "ERR_INVALID"), (0.0, "ERR_HIP")])
def test_scale(srs, scale, code):  # noqa: F811
    got = srs._lib.srs_cache_attention(CTX, cache(srs), rows(srs), rows(srs), A, 5, A, A, A, 4, 3, scale, 0, 0, 0, 5, 64, A, 1 << 30, None)
    assert got == getattr(srs, code)
