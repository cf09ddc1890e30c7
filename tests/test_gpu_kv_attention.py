"""Attention over the paged cache against the oracle's float64."""
import numpy as np
import pytest
import torch

from oracle import attention_block as A
from paper_2411_04965_amd import binding as B
from tests.attention_util import BF16, F32, Batch, states
from tests.gpu_util import dev, host

pytestmark = pytest.mark.gpu


def tolerance(o, a, mass, unit, n, D, q_bits):
    """A score loses at most (D + 8) 2^-24 of sum |q| |k| in float32.  A query that is not quantized is kept in steps of 1 / 3840 of its
    largest channel (largest = 15, three digits of a sixteenth each): every channel is off by half a step, the score by that times
    sum |k|, and by 2^-22 of sum |q| |k| for the two roundings of the division and the product.  That shifts every term by a factor
    exp(x), numerator and denominator alike: 2 (exp(x) - 1) of sum p |v| / sum p.  A term is rounded to 8 significand bits (2^-8; the
    parts end at 2^-22 of the largest value scale: 3 levels, n terms), exp2, the float32 sums and their rescalings take 2^-16 more;
    the output its bfloat16 rounding 2^-8."""
    x = mass[..., 0] * ((D + 8) * 2.0 ** -24 + 2.0 ** -22) + (mass[..., 1] / 7680 if q_bits == 16 else 0.0)
    e = (2 * np.expm1(x)[..., None] + 2.0 ** -8 + 2.0 ** -16) * a + n[..., None] * 2.0 ** -22 * 2 * unit[..., None]
    return e + 2.0 ** -8 * (np.abs(o) + e) + 1e-30


def run(b, Hq, q_dtype=BF16, rope=False, window=0, sinks=0, q_bits=16, scale=None, zero=False, strided=False, Q=None):
    if Q is None:
        Q = states(b.g, (b.T, Hq, b.D), q_dtype) * (0.0 if zero else 2.0)
    scale = b.D ** -0.5 if scale is None else scale
    pages, table, qs, ln = b.dev()
    qd = dev(Q, q_dtype)
    if strided:
        wide = torch.full((b.T, Hq * b.D + 64), float("nan"), dtype=q_dtype, device="cuda")
        wide[:, 64:] = qd.view(b.T, -1)
        qd = wide[:, 64:].view(b.T, Hq, b.D)
    out = torch.full((b.T, Hq, b.D), 7.0, dtype=BF16, device="cuda")
    B.kv_pages_attention(qd, pages, table, qs, ln, b.H, rope=b.rope_d if rope else None, scale=scale, window=window, sinks=sinks,
                         q_bits=q_bits, out=out)
    o, a, mass, unit, n = A.attention(Q, b.pool, b.table, b.q_start, b.kv_len, b.rope if rope else None, float(np.float32(scale)), window,
                                      sinks, q_bits)
    got = host(out)
    rows = int(b.q_start[-1])
    assert (got[rows:] == 7.0).all(), "rows of no sequence"
    got, o, a, mass, unit, n = (t[:rows] for t in (got, o, a, mass, unit, n))
    assert np.isfinite(got).all()
    assert (got[n == 0] == 0).all(), "rows that see nothing"
    tol = tolerance(o, a, mass, unit, n, b.D, q_bits)
    err = np.abs(got - o)
    assert (err <= tol).all(), "err / tol %.3g at %s" % ((err / tol).max(), np.argwhere(err > tol)[:4].tolist())
    return out


CASES = [
    # new, ctx, H, Hq, D
    ([1], [0], 1, 1, 32), ([1], [0], 2, 2, 128), ([1], [127], 1, 4, 128), ([1], [128], 2, 2, 64), ([1, 1, 1], [5, 700, 129], 2, 8, 128),
    ([1], [2000], 1, 1, 256), ([7], [0], 1, 3, 64), ([40, 1, 0, 130], [90, 383, 60, 0], 2, 4, 128), ([33], [250], 2, 10, 96),
    ([20, 2], [140, 3], 1, 5, 100), ([3], [300], 1, 17, 34), ([50], [100], 1, 1, 2), ([200], [60], 1, 2, 160)]


@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("new,ctx,H,Hq,D", CASES)
def test_chunks_and_single_tokens(new, ctx, H, Hq, D, zero):
    """Random queries, and zero queries: every visible value with the same weight, whatever its place."""
    print("attention", new, ctx, H, Hq, D, zero, flush=True)
    b = Batch(new, ctx, H, D, 11)
    b.fill()
    run(b, Hq, zero=zero)


@pytest.mark.parametrize("q_bits,q_dtype,rope", [(4, BF16, False), (4, F32, True), (16, F32, False), (16, BF16, True), (16, F32, True)])
@pytest.mark.parametrize("new,ctx,H,Hq,D", [CASES[4], CASES[7], CASES[9], CASES[12], CASES[5]])
def test_query_forms(new, ctx, H, Hq, D, q_bits, q_dtype, rope):
    print("query form", new, ctx, D, q_bits, q_dtype, rope, flush=True)
    b = Batch(new, ctx, H, D, 12)
    b.fill()
    run(b, Hq, q_dtype=q_dtype, rope=rope, q_bits=q_bits)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (60, 0), (128, 4), (129, 130), (300, 128), (100000, 3)])
@pytest.mark.parametrize("new,ctx,H,Hq,D", [([1, 1], [700, 3], 2, 4, 64), ([150], [200], 1, 2, 128), ([30, 5], [0, 600], 2, 2, 100)])
def test_windows_and_sinks(new, ctx, H, Hq, D, window, sinks):
    print("window", new, ctx, D, window, sinks, flush=True)
    b = Batch(new, ctx, H, D, 13)
    b.fill()
    for zero in (False, True):
        run(b, Hq, window=window, sinks=sinks, zero=zero)


def test_many_rows_take_the_row_tiles():
    """Enough rows that the keys are not split over workgroups."""
    b = Batch([900, 200], [100, 37], 32, 32, 14)
    b.fill()
    assert B.lib().kv_pages_attention_workspace_bytes(b.T, 2, 64, 32, 32, b.max_pages) == 0
    run(b, 64, window=200, sinks=2)
    b = Batch([300, 1, 77], [100, 37, 0], 32, 128, 15)
    b.fill()
    run(b, 64, rope=True)
    run(b, 64, q_bits=4)


def test_long_sequence_split_over_workgroups():
    b = Batch([1], [40000], 1, 64, 16)
    b.fill()
    run(b, 8)
    run(b, 8, window=20000, sinks=4, zero=True)


def test_strided_rows_and_scales():
    b = Batch([5, 1], [200, 9], 2, 64, 17)
    b.fill()
    run(b, 4, strided=True, rope=True)
    run(b, 4, scale=1e-4)
    run(b, 4, scale=2.0)                                 # all weight on a few keys


def test_rows_and_pages_that_are_not_there():
    b = Batch([4, 60, 3, 2], [1, 300, 100, 500], 2, 64, 18, max_pages=3, extra_rows=9)
    b.fill()
    b.kv_len[0] = 2                                      # two of its four rows have no position
    b.table[1, 1] = -1                                   # a hole
    b.table[2, 0] = len(b.pool.raw)                      # all it would see lies outside the pool
    for zero in (False, True):
        run(b, 4, zero=zero)
    run(b, 4, window=100, sinks=2)                       # sequence 3 ends past the table: rows that see nothing of their window
    b.kv_len[:] = 0
    run(b, 4)


def test_an_empty_cache_place_may_hold_anything():
    """Infinite and NaN scales in places no row sees, codes of any kind."""
    b = Batch([1, 20], [130, 0], 1, 128, 19)
    b.fill()
    n = b.pool.n_codes
    for s, page in ((0, 1), (1, 0)):
        f = b.pool.floats[b.table[s, page], 0]
        live = b.total[s] - 128 * page
        for part in (0, 1):
            f[2 * n + 128 * part + live:2 * n + 128 * (part + 1)] = np.where(np.arange(128 - live) % 2, np.inf, np.nan)
    run(b, 2)


def test_value_scales_of_any_size():
    b = Batch([1, 9], [300, 130], 1, 64, 20)
    b.fill()
    n = b.pool.n_codes
    for k, f in ((0, 2.0 ** -60), (1, 2.0 ** 40), (2, 0.0)):
        for s in range(2):
            if 0 <= b.table[s, min(k, b.max_pages - 1)] and k < b.max_pages:
                b.pool.floats[b.table[s, k], 0, 2 * n + 128:2 * n + 256] *= np.float32(f)
    run(b, 2)


def test_one_visible_key_is_returned_as_it_is():
    b = Batch([130], [0], 2, 64, 21)
    b.fill()
    out = host(run(b, 2, window=1))
    for h in range(2):
        v, _ = A.cached(b.pool, b.table, 0, h, 1)
        # its weight is exactly 1 and its levels are small integers: scale * level, split in two parts, loses 2^-8, bfloat16 2^-8
        assert (np.abs(out[:, h] - v[:130]) <= (2.0 ** -7 + 2.0 ** -16) * np.abs(v[:130])).all()


def test_key_of_every_place_is_found():
    """A query that singles out one key of the page: its value comes out, for every place."""
    b = Batch([128], [128], 1, 128, 22)
    b.fill()
    k, _ = A.cached(b.pool, b.table, 0, 0, 0)
    Q = np.zeros((128, 1, 128), np.float32)
    Q[:, 0] = k[128:256]                                 # the row's own key: |k|^2 stands far above k . k'
    from paper_2411_04965_amd.synth import snap_bf16
    run(b, 1, Q=snap_bf16(Q), scale=1.0)
