"""Weights far below a row's largest: a key that takes nearly all of the softmax and whose value is next to nothing, so that the output
is made of the others' values."""
import numpy as np
import pytest
import torch

from oracle import attention_block as A
from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, Batch, fast_put
from tests.gpu_util import dev, host

pytestmark = pytest.mark.gpu
AT = 5                                                               # the key's position


@pytest.mark.parametrize("nats", [9.0, 14.0, 17.0, 25.0])
@pytest.mark.parametrize("new,ctx,H,Hq,D", [([1], [500], 2, 4, 128), ([3], [400], 1, 2, 64), ([30], [450], 1, 4, 128), ([1], [500], 1, 2, 256),
                                            ([1], [9000], 1, 4, 64), ([300, 140], [700, 0], 16, 32, 256), ([300, 140], [700, 0], 16, 64, 128)])
def test_a_dominant_key_without_a_value(new, ctx, H, Hq, D, nats):
    """Per term: 2^-8 of its own for the weight's 8 significand bits, and 2^-22 of the page's largest p * scale where the parts of an E4M3
    pair end, which over a page's 128 tokens and 3 levels is at most 2^-15 of the sum of p * max |v|.  Every key but one has a score of
    next to nothing, and a query's fixed-point step moves a score by x as in the other tests."""
    print("dominant key", new, ctx, D, nats, flush=True)
    b = Batch(new, ctx, H, D, 95)
    scale = float(np.float32(D ** -0.5))
    for s, t in enumerate(b.total):
        x = b.g.standard_normal((2, t, H, D)).astype(np.float32)
        x[0] *= 1e-3
        x[0, AT] = nats / (D * scale)                                # q is all ones: q . k = nats / scale
        x[1, AT] *= 1e-12
        fast_put(b.pool, b.table[s], x)
    Q = np.ones((b.T, Hq, D), np.float32)
    pages, table, qs, ln = b.dev()
    got = host(B.kv_pages_attention(dev(Q, BF16), pages, table, qs, ln, H, scale=scale))
    G = Hq // H
    for s in range(len(new)):
        r0, pos = A.rows_of(b.q_start, b.kv_len, s)
        for h in range(H):
            k, there = A.cached(b.pool, b.table, s, h, 0)
            v, _ = A.cached(b.pool, b.table, s, h, 1)
            n = b.total[s]
            k, v = k[:n].astype(float), v[:n].astype(float)
            z = np.where(np.arange(n) <= pos[:, None], scale * k.sum(1), -np.inf)
            p = np.exp(z - z.max(1, keepdims=True))
            l = p.sum(1, keepdims=True)
            o, a, w = p @ v / l, p @ np.abs(v) / l, p @ np.abs(v).max(1)[:, None] / l
            x = (scale * (np.abs(k).sum(1) * ((D + 8) * 2.0 ** -24 + 2.0 ** -22 + 1 / 7680))).max()
            e = (2 * np.expm1(x) + 2.0 ** -8 + 2.0 ** -16) * a + 2.0 ** -15 * w
            e = e + 2.0 ** -8 * (np.abs(o) + e) + 1e-30
            for g in range(h * G, (h + 1) * G):
                err = np.abs(got[r0:r0 + len(pos), g] - o)
                assert (err <= e).all(), "err / tol %.3g" % (err / e).max()
