"""The cache's calls on a stream that is not the current one.  Everything that a call reads or writes is made, and ordered before it, first; the
other stream is kept busy so that its calls run late, while the current stream fills fresh memory of a workspace's size: a workspace that
belonged to the current stream would be among it."""
import pytest
import torch

from test_gpu_cache_attention import DEV, Batch, compare, ctx  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("start,count", [([900, 400, 9000], [1, 1, 1]), ([900, 400, 9000], [1, 20, 1]), ([6000], [40])])
def test_attention(ctx, monkeypatch, native, start, count):  # noqa: F811
    from paper_2605_07330_amd import srs
    if not native:
        monkeypatch.setattr(srs, "_native", lambda *a: False)
    b = Batch(start, count, 8, 2, 128, 16)
    want = b.expect()
    most = {"most_tokens": max(count), "most_keys": max(s + c for s, c in zip(start, count))}
    need = srs.attention_workspace(len(start), sum(count), 8, 2, 128, b.table.shape[1], 16, **most)
    assert need
    side, current = torch.cuda.Stream(), torch.cuda.current_stream()
    work = torch.randn(4096, 4096, device=DEV)
    results = [(torch.full_like(b.q, 9.0), torch.full(b.q.shape[:2], 9.0, device=DEV)) for _ in range(3)]
    busy = torch.empty_like(work)
    side.wait_stream(current)
    with torch.cuda.stream(side):
        for _ in range(4):
            torch.mm(work, work, out=busy)
    junk = []
    for out, lse in results:
        b.call(ctx, out=out, lse=lse, stream=side, **most)
        junk += [torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(4)]
    current.wait_stream(side)
    for got in results:
        compare(got, want)
    assert ctx.status() == 0
    with torch.cuda.stream(side):                                       # and where it is the current one
        side.wait_stream(current)
        got = b.call(ctx, **most)
    current.wait_stream(side)
    compare(got, want)
    assert ctx.status() == 0


@pytest.mark.parametrize("native", [True, False])
def test_a_step(ctx, monkeypatch, native):  # noqa: F811
    """Tables, rows into the cache and attention one after the other, their order the stream's own."""
    from paper_2605_07330_amd import srs
    if not native:
        monkeypatch.setattr(srs, "_native", lambda *a: False)
    i32, side, current = dict(dtype=torch.int32, device=DEV), torch.cuda.Stream(), torch.cuda.current_stream()

    def state():
        g = torch.Generator(device=DEV).manual_seed(11)
        rows = torch.randn(60, 12, 64, generator=g, device=DEV).bfloat16()
        return dict(start=torch.tensor([0, 5, 0], **i32), count=torch.tensor([40, 1, 17], **i32), held=torch.tensor([0, 1, 0], **i32),
                    table=torch.tensor([[-1] * 4, [30, -1, -1, -1], [-1] * 4], **i32), free=torch.arange(20, **i32), left=torch.tensor([20], **i32), begin=torch.zeros(4, **i32),
                    slots=torch.zeros(60, dtype=torch.int64, device=DEV), positions=torch.zeros(60, **i32), rows=rows, turned=torch.zeros(60, 8, 64, dtype=torch.bfloat16, device=DEV),
                    k=torch.ones(31, 16, 2, 64, dtype=torch.bfloat16, device=DEV), v=torch.ones(31, 16, 2, 64, dtype=torch.bfloat16, device=DEV),
                    out=torch.zeros(60, 8, 64, dtype=torch.bfloat16, device=DEV), freq=srs.rope_frequencies(64, device=DEV)[0])

    def step(s, **kw):
        ctx.cache_tables(s["start"], s["count"], 16, s["held"], s["table"], s["free"], s["left"], s["begin"], s["slots"], s["positions"], **kw)
        ctx.cache_write(s["rows"][:, 8:10], s["rows"][:, 10:], s["k"], s["v"], s["slots"], q=s["rows"][:, :8], q_out=s["turned"], positions=s["positions"], inv_freq=s["freq"], **kw)
        ctx.rope(s["turned"], s["turned"], s["positions"], s["freq"], transpose=True, **kw)
        ctx.cache_attention(s["turned"], s["out"], s["k"], s["v"], s["table"], s["begin"], s["start"], **kw)
        ctx.cache_release(s["start"], s["held"], s["table"], s["free"], s["left"], **kw)
    one, two = state(), state()
    step(one)
    work = torch.randn(4096, 4096, device=DEV)
    busy = torch.empty_like(work)
    side.wait_stream(current)
    with torch.cuda.stream(side):
        for _ in range(4):
            torch.mm(work, work, out=busy)
    step(two, stream=side)
    current.wait_stream(side)
    for name in one:
        assert torch.equal(one[name], two[name]), name
    assert ctx.status() == 0
