"""NaN and infinities that a row of the paged attention meets: in its query, or in a state that it sees.  The row is no number; every
other row keeps its bits."""
import numpy as np
import pytest
import torch

from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, F32, Batch
from tests.test_gpu_kv_attention_rows import FEW, MANY

pytestmark = pytest.mark.gpu

# new, ctx, H, Hq, width of the page table, D: tiles of 4, 8 and 16 rows (one workgroup along the keys, or several), whole rows of 128 and
# 256, and of more than 128 channels
FORMS = [([1, 1], [700, 30], 2, 4, None, 128), ([2, 1], [200, 30], 2, 4, None, 64), ([40, 3], [1500, 30], 2, 4, None, 128),
         ([1], [2000], 1, 8, None, 256), ([9, 1], [100, 0], 2, 2, None, 34), ([20], [300], 1, 4, None, 160),
         FEW + (64,), FEW + (100,), MANY + (128,), FEW + (256,)]
IDS = ["%dx%d_D%d" % (len(f[0]), f[0][0], f[5]) for f in FORMS]


def batch(form, seed):
    new, ctx, H, Hq, pages, D = form
    print("not finite", new, ctx, H, Hq, D, flush=True)
    b = Batch(new, ctx, H, D, seed, max_pages=pages)
    b.fill()
    return b, Hq


def queries(b, Hq, dtype=BF16):
    return torch.randn(b.T, Hq, b.D, generator=torch.Generator().manual_seed(9)).to(dtype).cuda()


def attend(b, Q, **kw):
    pages, table, qs, ln = b.dev()
    return B.kv_pages_attention(Q, pages, table, qs, ln, b.H, **kw)


@pytest.mark.parametrize("q_bits,dtype", [(16, BF16), (16, F32), (4, BF16)])
@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_a_query_that_is_not_finite(form, q_bits, dtype):
    b, Hq = batch(form, 81)
    Q = queries(b, Hq, dtype)
    clean = attend(b, Q, q_bits=q_bits)
    bad = torch.zeros(b.T, Hq, dtype=torch.bool, device="cuda")
    last = int(b.q_start[1]) - 1
    for (t, h, c), v in {(0, 0, 1): np.nan, (last, Hq - 1, b.D - 1): np.inf, (b.T - 1, 0, b.D // 2): -np.inf}.items():
        Q[t, h, c] = v
        bad[t, h] = True
    Q[last, 0] = float("nan")                                        # all of a row
    bad[last, 0] = True
    out = attend(b, Q, q_bits=q_bits)
    assert bool(torch.isnan(out[bad]).all())
    assert torch.equal(out[~bad], clean[~bad])


def test_such_a_query_that_sees_nothing():
    """Zeros, as for any query: no position, or only pages that are not there."""
    for new, H, Hq in (([4, 3], 2, 4), ([300, 77], 16, 64)):
        b = Batch(new, [0, 200], H, 64, 82)
        b.fill()
        b.kv_len[0] = new[0] - 2                                     # the first two rows have no position
        b.table[1, :] = -1
        Q = queries(b, Hq)
        Q[0], Q[b.T - 1] = float("nan"), float("inf")
        out = attend(b, Q)
        assert bool((out[:2] == 0).all()) and bool((out[new[0]:] == 0).all()) and bool(torch.isfinite(out).all())


def spoiled(b, at, key=None, value=None, head=0):
    """The scale of head 0 at position `at` of sequence 0 in the pool's bytes."""
    n = b.pool.n_codes
    f = b.pool.floats[b.table[0, at // 128], head]
    if key is not None:
        f[2 * n + at % 128] = key
    if value is not None:
        f[2 * n + 128 + at % 128] = value


@pytest.mark.parametrize("key,value", [(np.nan, None), (np.inf, None), (None, np.nan), (None, np.inf)])
@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_a_state_that_is_not_finite(form, key, value):
    b, Hq = batch(form, 83)
    Q, G = queries(b, Hq), Hq // b.H
    n0, ctx = b.new[0], form[1][0]
    for at in (0, ctx + n0 - 1 - n0 // 3):                           # the sequence's first state, and one of the new rows'
        kept = b.pool.raw.copy()
        clean = attend(b, Q)
        spoiled(b, at, key, value)
        out = attend(b, Q)
        b.pool.raw[:] = kept
        bad = torch.zeros(b.T, Hq, dtype=torch.bool, device="cuda")
        bad[max(at - ctx, 0):n0, :G] = True                          # the rows of sequence 0 that see it
        assert bool(torch.isnan(out[bad]).all()), at
        assert torch.equal(out[~bad], clean[~bad]), at


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_whatever_the_weight_or_the_values(form):
    """A value of next to no weight, a key beside values that are all zero."""
    b, Hq = batch(form, 84)
    Q, n0, G = queries(b, Hq) * 50, b.new[0], Hq // b.H
    spoiled(b, 1 if form[1][0] else 0, value=np.nan)
    assert bool(torch.isnan(attend(b, Q)[:n0, :G]).all())
    n = b.pool.n_codes
    b.fill()
    b.pool.floats[b.table[0, 0], 0, 2 * n + 128:2 * n + 256] = 0.0
    spoiled(b, 0, key=np.nan)
    assert bool(torch.isnan(attend(b, Q)[:n0, :G]).all())
