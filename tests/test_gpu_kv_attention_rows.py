"""Attention over the paged cache with enough rows that a workgroup takes 128 or 256 of one head, against the oracle's float64."""
import numpy as np
import pytest
import torch

from paper_2411_04965_amd import binding as B
from tests.attention_util import F32, Batch
from tests.test_gpu_kv_attention import run

pytestmark = pytest.mark.gpu

# new, ctx, H, Hq, width of the page table
FEW = ([300, 1, 77, 130], [100, 37, 0, 900], 16, 64, None)           # workgroups of 128 rows: of three sequences at most
MANY = ([500, 1, 523], [300, 700, 0], 14, 56, 20)                    # of 256 rows: two turns of the chip with 128, one with 256
SETS = [FEW + (64,), FEW + (100,), FEW + (128,), FEW + (256,), MANY + (64,), MANY + (128,), MANY + (34,), MANY + (160,)]


def batch(new, ctx, H, Hq, pages, D, seed):
    print("rows", new, ctx, H, Hq, D, flush=True)
    b = Batch(new, ctx, H, D, seed, max_pages=pages, extra_rows=3)
    b.fill()
    assert B.lib().kv_pages_attention_workspace_bytes(b.T, len(new), Hq, H, D, b.max_pages) == 0
    return b


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", SETS)
def test_rows_of_several_sequences(new, ctx, H, Hq, pages, D):
    b = batch(new, ctx, H, Hq, pages, D, 31)
    run(b, Hq, rope=True)
    run(b, Hq, zero=True)                                            # every visible value with the same weight
    run(b, Hq, q_bits=4, q_dtype=F32)


@pytest.mark.parametrize("window,sinks", [(1, 0), (130, 3), (256, 200)])
@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", [SETS[0], SETS[2], SETS[4], SETS[5]])
def test_windows(new, ctx, H, Hq, pages, D, window, sinks):
    run(batch(new, ctx, H, Hq, pages, D, 32), Hq, window=window, sinks=sinks)


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", [SETS[0], SETS[2], SETS[4], SETS[5]])
def test_pages_and_rows_that_are_not_there(new, ctx, H, Hq, pages, D):
    b = batch(new, ctx, H, Hq, pages, D, 33)
    b.table[0, 0] = -1                                               # the first page, one inside, all of a sequence, the last
    b.table[-1, 1] = len(b.pool.raw)
    b.table[1, :] = -1
    b.table[0, (b.total[0] - 1) // 128] = -1
    run(b, Hq)
    run(b, Hq, zero=True)
    b.kv_len[0] = new[0] - 100                                       # a hundred of its rows have no position
    run(b, Hq, zero=True)
    b.kv_len[:] = 0
    run(b, Hq)


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", [SETS[0], SETS[2], SETS[4], SETS[5]])
def test_value_scales_of_any_size(new, ctx, H, Hq, pages, D):
    b = batch(new, ctx, H, Hq, pages, D, 34)
    n = b.pool.n_codes
    for s in range(len(new)):
        for k, f in ((0, 2.0 ** -60), (1, 2.0 ** 40), (2, 0.0)):
            if b.table[s, k] >= 0:
                b.pool.floats[b.table[s, k], :, 2 * n + 128:2 * n + 256] *= np.float32(f)
    run(b, Hq)


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", [SETS[0], SETS[2], SETS[4], SETS[5]])
def test_masked_places_may_hold_anything(new, ctx, H, Hq, pages, D):
    """Positions that the later rows of a workgroup see and the earlier ones do not, with infinities and NaN there: the earlier rows'
    results stand."""
    b = batch(new, ctx, H, Hq, pages, D, 35)
    n = b.pool.n_codes
    s, at = 0, b.total[0] - 40                                       # seen by the last 40 rows of sequence 0
    f = b.pool.floats[b.table[s, at // 128]]
    keep = f.copy()
    clean = run(b, Hq).float().cpu().numpy()
    f[:, 2 * n + at % 128] = np.inf
    f[:, 2 * n + 128 + at % 128] = np.nan
    pages_d, table, qs, ln = b.dev()
    Q = torch.randn(b.T, Hq, D, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    bad = B.kv_pages_attention(Q, pages_d, table, qs, ln, H).float().cpu().numpy()
    f[:] = keep
    pages_d, table, qs, ln = b.dev()
    good = B.kv_pages_attention(Q, pages_d, table, qs, ln, H).float().cpu().numpy()
    rows = new[0] - 40
    assert np.array_equal(bad[:rows], good[:rows]) and np.isfinite(clean[:b.q_start[-1]]).all()


@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", [SETS[1], SETS[5], SETS[3]])
def test_captured_and_replayed(new, ctx, H, Hq, pages, D):
    """The graph takes the queries and lengths that stand there at each replay."""
    b = batch(new, ctx, H, Hq, pages, D, 36)
    pages_d, table, qs, ln = b.dev()
    g = torch.Generator().manual_seed(5)
    Q = torch.randn(b.T, Hq, D, generator=g).to(torch.bfloat16).cuda()
    out = torch.zeros(b.T, Hq, D, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.kv_pages_attention(Q, pages_d, table, qs, ln, H, window=200, sinks=1, out=out)
    full = ln.clone()
    for k in range(4):
        Q.copy_(torch.randn(b.T, Hq, D, generator=g))
        ln.copy_(full - 30 * k)
        graph.replay()
        want = B.kv_pages_attention(Q, pages_d, table, qs, ln, H, window=200, sinks=1)
        torch.cuda.synchronize()
        rows = int(b.q_start[-1])
        assert torch.equal(out[:rows], want[:rows]), k
