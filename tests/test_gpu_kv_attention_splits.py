"""Partial results of workgroups along the keys and their join: on two streams at once, captured and replayed."""
import pytest
import torch

from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, Batch

pytestmark = pytest.mark.gpu
SETS = [([1, 1], [5000, 300], 2, 8, 128), ([3], [7000], 2, 4, 64), ([12, 1], [2500, 6000], 1, 4, 256)]


def batch(new, ctx, H, Hq, D, seed):
    print("splits", new, ctx, H, Hq, D, flush=True)
    b = Batch(new, ctx, H, D, seed)
    b.fill()
    n = B.lib().kv_pages_attention_workspace_bytes(b.T, len(new), Hq, H, D, b.max_pages)
    assert n > 0
    g = torch.Generator().manual_seed(seed)
    return b, n, lambda: torch.randn(b.T, Hq, D, generator=g).to(BF16).cuda()


@pytest.mark.parametrize("new,ctx,H,Hq,D", SETS)
def test_two_streams(new, ctx, H, Hq, D):
    b, n, query = batch(new, ctx, H, Hq, D, 101)
    pages, table, qs, ln = b.dev()
    Q = [query() for _ in range(8)]
    want = [B.kv_pages_attention(q, pages, table, qs, ln, H) for q in Q]
    ws = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None] * 8
    for i, q in enumerate(Q):
        with torch.cuda.stream(streams[i % 2]):
            got[i] = B.kv_pages_attention(q, pages, table, qs, ln, H, ws=ws[i % 2])
    torch.cuda.synchronize()
    for a, w in zip(got, want):
        assert torch.equal(a, w)


@pytest.mark.parametrize("new,ctx,H,Hq,D", SETS)
def test_captured_and_replayed(new, ctx, H, Hq, D):
    """Queries and lengths change between the replays, down to lengths of which most workgroups have no page, and what the workspace
    holds is overwritten."""
    b, n, query = batch(new, ctx, H, Hq, D, 103)
    pages, table, qs, ln = b.dev()
    Q, ws = query(), torch.zeros(n, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(Q)
    B.kv_pages_attention(Q, pages, table, qs, ln, H, ws=ws, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_pages_attention(Q, pages, table, qs, ln, H, ws=ws, out=out)
    full = ln.clone()
    for k, short in enumerate((0, 129, 2000, 10 ** 6, 1)):
        Q.copy_(query())
        ln.copy_(torch.maximum(full - short, qs[1:] - qs[:-1]))
        ws.fill_(255)
        out.fill_(float("nan"))
        graph.replay()
        want = B.kv_pages_attention(Q, pages, table, qs, ln, H)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and bool(torch.isfinite(out).all()), k
