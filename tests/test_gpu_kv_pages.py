"""The paged cache's bytes against the oracle, and its values read back."""
import numpy as np
import pytest
import torch

from oracle import attention_block as A
from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, F32, Batch, states
from tests.gpu_util import dev, host

pytestmark = pytest.mark.gpu
EPS = 1e-5


def check(b, dtype, rope, strided=False):
    """Appends the batch's rows on both sides: all bytes of the pool, and the values read back, have to be the same."""
    K, V = states(b.g, (b.T, b.H, b.D), dtype), states(b.g, (b.T, b.H, b.D), dtype)
    pages, table, qs, ln = b.dev()
    if strided:
        wide = torch.full((b.T, 3 * b.H * b.D + 8), float("nan"), dtype=dtype, device="cuda")
        n = b.H * b.D
        kd, vd = wide[:, n:2 * n].view(b.T, b.H, b.D), wide[:, 2 * n:3 * n].view(b.T, b.H, b.D)
        kd.copy_(dev(K, dtype))
        vd.copy_(dev(V, dtype))
    else:
        kd, vd = dev(K, dtype), dev(V, dtype)
    B.kv_pages_append(kd, vd, pages, table, qs, ln, rope=b.rope_d if rope else None, eps=EPS)
    A.append(b.pool, K, V, b.table, b.q_start, b.kv_len, b.rope if rope else None, EPS)
    got = pages.cpu().numpy()
    # the padding channels' value codes are zero where a token was written; the oracle leaves them: compare what stands for something
    want = b.pool
    mine = A.Pages(got, b.H, b.D)
    for s in range(len(b.new)):
        for k in range(b.max_pages):
            if not 0 <= b.table[s, k] < len(got):
                continue
            for h in range(b.H):
                for v in (0, 1):
                    (q0, d0), (q1, d1) = want.get(b.table[s, k], h, v, k == 0), mine.get(b.table[s, k], h, v, k == 0)
                    assert np.array_equal(q0, q1), "levels: sequence %d page %d head %d values %d" % (s, k, h, v)
                    assert np.array_equal(d0, d1, equal_nan=True), "scales"
    untouched = np.setdiff1d(np.arange(len(got)), b.table[b.table >= 0])
    assert np.array_equal(got[untouched], want.raw[untouched])
    for odt in (F32, BF16):
        out = [torch.full((b.T, b.H, b.D), -7.0, dtype=odt, device="cuda") for _ in range(2)]
        B.kv_pages_read(pages, table, qs, ln, b.T, b.H, b.D, out=out)
        for v, o in enumerate(out):
            ref = np.full((b.T, b.H, b.D), -7.0, np.float32)
            for s in range(len(b.new)):
                r0, pos = A.rows_of(b.q_start, b.kv_len, s)
                for h in range(b.H):
                    val, there = A.cached(want, b.table, s, h, v)
                    for i, p in enumerate(pos):
                        if 0 <= p < len(there) and there[p]:
                            ref[r0 + i, h] = val[p]
            assert torch.equal(o, dev(ref, odt)), "read back"


@pytest.mark.parametrize("new,ctx,H,D,dtype,rope", [
    ([1], [0], 1, 2, BF16, True), ([1], [0], 2, 128, BF16, True), ([1, 1, 1], [127, 128, 500], 3, 64, BF16, True),
    ([130], [0], 1, 128, F32, True), ([5, 0, 300, 1], [126, 4, 100, 0], 2, 100, BF16, True), ([140, 3], [250, 0], 2, 256, F32, True),
    ([257], [127], 1, 96, BF16, False), ([17], [3], 2, 30, F32, True), ([64, 64, 64], [0, 64, 128], 1, 32, BF16, False),
    ([2] * 70, list(range(70)), 1, 34, BF16, True), ([128, 128], [0, 128], 1, 160, BF16, True)])
def test_append_and_read(new, ctx, H, D, dtype, rope):
    print("append", new[:4], ctx[:4], H, D, dtype, flush=True)
    b = Batch(new, ctx, H, D, 1)
    b.fill(0)
    check(b, dtype, rope)


def test_rows_of_a_fused_product():
    b = Batch([9, 1], [120, 40], 2, 64, 2)
    b.fill(0)
    check(b, BF16, True, strided=True)


def test_rows_and_pages_that_are_not_there():
    """Rows behind the last sequence, rows before position 0, positions past the table, entries outside the pool."""
    b = Batch([3, 200, 1, 4], [0, 100, 300, 2], 2, 64, 3, max_pages=2, extra_rows=5)
    b.kv_len[3] = 2                                      # four rows, two positions: the first two rows have none
    b.table[1, 0] = -1
    b.table[0, 0] = len(b.pool.raw)                      # one behind the pool
    check(b, BF16, True)


def test_zero_and_extreme_states():
    b = Batch([4], [0], 1, 64, 4)
    pages, table, qs, ln = b.dev()
    K = np.zeros((4, 1, 64), np.float32)
    K[1] = 1e-30
    K[2, 0, 5] = 3e38
    K[3, 0] = -2.0
    B.kv_pages_append(dev(K), dev(-K), pages, table, qs, ln, eps=EPS)
    k, v = B.kv_pages_read(pages, table, qs, ln, 4, 1, 64)
    want = []
    for x in (K, -K):
        q, d = A.levels(x, np.arange(4), EPS)
        want.append((q.astype(np.float32) * d[:, :, None]))
    assert np.array_equal(host(k), want[0]) and np.array_equal(host(v), want[1])


def test_two_calls_and_one_give_the_same_pages():
    """A page filled token by token has the codes of a page filled at once."""
    b = Batch([150], [0], 2, 128, 5)
    X = states(b.g, (2, 150, 2, 128), BF16)
    pages, table, qs, ln = b.dev()
    one = pages.clone()
    B.kv_pages_append(dev(X[0], BF16), dev(X[1], BF16), one, table, qs, ln, rope=b.rope_d)
    for lo, hi in ((0, 1), (1, 2), (2, 60), (60, 129), (129, 130), (130, 150)):
        q = torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda")
        n = torch.tensor([hi], dtype=torch.int32, device="cuda")
        B.kv_pages_append(dev(X[0, lo:hi], BF16), dev(X[1, lo:hi], BF16), pages, table, q, n, rope=b.rope_d)
    assert torch.equal(pages, one)
