"""Queries of which one channel stands far above the others: what the others say is kept."""
import numpy as np
import pytest
import torch

from oracle import attention_block as A
from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, F32, Batch, fast_put
from tests.gpu_util import dev, host
from tests.test_gpu_kv_attention import tolerance
from tests.test_gpu_kv_attention_rows import FEW, MANY

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("new,ctx,H,Hq,pages,D", [([1, 1], [700, 30], 2, 4, None, 128), ([2], [200], 2, 6, None, 64), ([40, 3], [300, 30], 2, 4, None, 128),
                                                  ([9], [100], 2, 2, None, 34), ([1], [700], 1, 4, None, 256), ([20], [300], 1, 4, None, 160),
                                                  FEW + (64,), FEW + (128,), MANY + (128,), FEW + (256,)])
def test_an_outlying_channel(new, ctx, H, Hq, pages, D, dtype):
    """Channel 0 is 7680, where the keys are zero; the others are multiples of a half, which is 1 / 15360 of the largest: exact in the
    three digits, so that a score loses what float32 loses and nothing else."""
    print("outlying channel", new, ctx, D, dtype, flush=True)
    b = Batch(new, ctx, H, D, 111, max_pages=pages)
    for s, t in enumerate(b.total):
        x = b.g.standard_normal((2, t, H, D)).astype(np.float32)
        x[0, ..., 0] = 0.0
        fast_put(b.pool, b.table[s], x)
    Q = (b.g.integers(-6, 7, (b.T, Hq, D)) * 0.5).astype(np.float32)
    Q[..., 0] = 7680.0 * np.where(b.g.random((b.T, Hq)) < 0.5, -1, 1)
    scale = float(np.float32(D ** -0.5))
    d = b.dev()
    got = host(B.kv_pages_attention(dev(Q, dtype), *d, H, scale=scale))
    o, a, mass, unit, n = A.attention(Q, b.pool, b.table, b.q_start, b.kv_len, None, scale)
    tol = tolerance(o, a, mass, unit, n, D, 4)                       # (4: without the term for a query's fixed-point step)
    err = np.abs(got - o)
    assert (err <= tol).all(), "err / tol %.3g" % (err / tol).max()


@pytest.mark.parametrize("D,dtype", [(64, F32), (128, F32), (256, F32), (128, BF16)])
def test_every_channel_and_level_of_a_query(D, dtype):
    """Row i's query has one channel beside the largest, which keys do not have: its score with the one key that is not zero, and so that
    key's weight against two others of score 0, gives it back to half a step, 1 / 30720 of the largest, for numbers of all sizes down
    to a 20000th of it."""
    b = Batch([D], [1], 1, D, 113)
    x = np.zeros((2, D + 1, 1, D), np.float32)
    x[0, 1, 0, 1:] = 3.0                                             # key 1; key 0 and the rows' own keys and values are zero
    x[1, 1] = 3.0
    fast_put(b.pool, b.table[0], x)
    g = np.random.default_rng(5)
    Q = np.zeros((D, 1, D), np.float32)
    Q[np.arange(D), 0, np.arange(D)] = np.exp(g.uniform(np.log(5e-5), 0.0, D)) * np.where(g.random(D) < 0.5, -1, 1)
    Q[:, 0, 0] = 1.0
    qd = dev(Q, dtype)
    q = host(qd)[np.arange(D), 0, np.arange(D)].astype(float)
    got = host(B.kv_pages_attention(qd, *b.dev(), 1, scale=1000.0, window=1, sinks=2))[:, 0, 1].astype(float)
    k1, v1 = (float(A.cached(b.pool, b.table, 0, 0, v)[0][1, 1]) for v in (0, 1))
    with np.errstate(over="ignore"):
        for i in range(1, D):
            lo, mid, hi = (v1 / (1 + 2 * np.exp(-1000 * (q[i] + e) * k1)) for e in (-1 / 30720 - 1e-6, 0.0, 1 / 30720 + 1e-6))
            slack = 2.0 ** -7 * mid + 1e-36                          # the weight's rounding, the output's, and where float32 ends
            assert lo - slack <= got[i] <= hi + slack, (i, q[i], got[i])
