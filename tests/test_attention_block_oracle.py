"""The oracle of the norm, the paged cache and its attention, pinned without itself: hand-worked words, the single-sequence cache's
oracle, differences, closed forms."""
import numpy as np
import pytest

from oracle import attention_block as A
from oracle import bitnet_a48 as O


def rng(*k):
    return np.random.default_rng([19, *k])


def test_words_of_a_hand_worked_token():
    pool = A.Pages(np.zeros((1, A.page_bytes(1, 32)), np.uint8), 1, 32)
    q = np.zeros(32, int)
    q[0], q[1], q[9], q[17], q[31] = 3, -2, 1, -3, -1
    pool.put(0, 0, 0, 21, q, 0.5, False)                 # token 21 = 64*0 + 16*1 + 4*1 + 1: slot 16*1 + 4*1 + 1
    w = pool.words[0, 0, 21 * 3:21 * 3 + 3]
    # code 0: bits 0, 1; code 1: bits 4, 5; code 9: bits 6, 7 | code 17: bits 4, 5; code 31: bits 30, 31 | signs: 4 (i % 8) + 3 - i / 8
    assert [int(x) for x in w] == [3 | 2 << 4 | 1 << 6, 3 << 4 | 1 << 30, 1 << 7 | 1 << 5 | 1 << 28]
    pool.put(0, 0, 0, 6, q, 1.0, False)                  # token 6 = 4*1 + 2: slot 16*1 + 2
    assert int(pool.words[0, 0, 18 * 3]) == int(w[0])
    pool.put(0, 0, 1, 37, q, 0.25, False)                # values: channel 0, tokens 32 .. 63: group 1, code 5
    assert int(pool.words[0, 0, A.PAGE * 3 + 3]) == 3 << 20
    assert pool.floats[0, 0, 2 * A.PAGE * 3 + 21] == 0.5 and pool.floats[0, 0, 2 * A.PAGE * 3 + A.PAGE + 37] == 0.25
    q[0], q[1] = 7, -4                                   # a first token: magnitudes 3 (+ 1), 2 (+ 0)
    pool.put(0, 0, 0, 0, q, 1.0, True)
    assert int(pool.words[0, 0, 0]) & 0x3F == 3 | 2 << 4
    assert int(pool.words[0, 0, 2 * A.PAGE * 3 + 2 * A.PAGE]) & 0x88 == 1 << 3


@pytest.mark.parametrize("H,D,T", [(1, 32, 5), (2, 64, 131), (1, 96, 129)])
def test_pages_hold_what_the_single_sequence_cache_holds(H, D, T):
    X = rng(H, D, T).standard_normal((T, H, D)).astype(np.float32)
    raw, d = O.kv_cache_pack(X)
    want = O.kv_cache_unpack(raw, d, T, H, D)
    mp = (T + 127) // 128
    table = np.arange(mp)[::-1].reshape(1, mp)
    pool = A.Pages(rng(1).integers(0, 256, (mp, A.page_bytes(H, D))).astype(np.uint8), H, D)
    for n in (T - 3, T):                                 # in two goes: new tokens leave older ones as they are
        lo = 0 if n < T else T - 3
        A.append(pool, X[lo:n], X[lo:n][:, :, ::-1], table, [0, n - lo], [n], None, O.DEFAULT_EPS)
    for h in range(H):
        assert np.array_equal(A.cached(pool, table, 0, h, 0)[0][:T], want[:, h])
        assert np.array_equal(A.cached(pool, table, 0, h, 1)[0][:T], _values(X[:, :, ::-1])[:, h])


def _values(X):
    q, d = A.levels(X, np.arange(len(X)), O.DEFAULT_EPS)
    return q.astype(np.float32) * d[:, :, None]


def test_rotation_keeps_lengths_and_differences_of_angles():
    D = 64
    inv = 10000.0 ** (-2.0 * np.arange(D // 2) / D)
    ang = np.arange(50)[:, None] * inv
    tab = np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)
    x = rng(5).standard_normal((2, 1, D)).astype(np.float32)
    dots = []
    for a, b in ((3, 10), (20, 27), (0, 7)):
        r = A.rotate(x, tab, np.array([a, b]))
        dots.append(float(r[0, 0].astype(float) @ r[1, 0].astype(float)))
        assert np.allclose((r.astype(float) ** 2).sum(2), (x.astype(float) ** 2).sum(2), rtol=1e-5)
    assert np.allclose(dots, dots[0], atol=1e-4)         # a matter of the distance alone


def test_norm_gradient_against_differences():
    g = rng(7)
    M, K = 3, 11
    X, R, dY, ga = (g.standard_normal(s) for s in ((M, K), (M, K), (M, K), (K,)))
    def loss(x, ga):
        return float((dY * (x / np.sqrt((x * x).mean(1, keepdims=True) + 1e-5)) * ga).sum() + (R * x).sum())
    rstd = 1 / np.sqrt((X * X).mean(1) + 1e-5)
    # the formula drops nothing: d(rstd)/dh = -h rstd^3 / K holds with eps inside rstd
    dX, dga = A.rmsnorm_backward(dY, X, rstd, ga, R)
    e = 1e-6
    for m in range(M):
        for k in range(K):
            p, n = X.copy(), X.copy()
            p[m, k] += e
            n[m, k] -= e
            assert abs((loss(p, ga) - loss(n, ga)) / (2 * e) - dX[m, k]) < 1e-7
    for k in range(K):
        p, n = ga.copy(), ga.copy()
        p[k] += e
        n[k] -= e
        assert abs((loss(X, p) - loss(X, n)) / (2 * e) - dga[k]) < 1e-7


def test_attention_closed_forms():
    H, D, T = 1, 32, 140
    g = rng(9)
    X = g.standard_normal((T, H, D)).astype(np.float32)
    table = np.array([[1, 0]])
    pool = A.Pages(np.zeros((2, A.page_bytes(H, D)), np.uint8), H, D)
    A.append(pool, X, X, table, [0, T], [T], None, O.DEFAULT_EPS)
    v = A.cached(pool, table, 0, 0, 1)[0][:T].astype(float)
    o, *_ = A.attention(np.zeros((T, 2, D)), pool, table, [0, T], [T], None, 0.2)
    for i in (0, 1, 127, 128, 139):                      # no preference: the mean of what is visible
        assert np.allclose(o[i, 1], v[:i + 1].mean(0))
    o, *_, n = A.attention(np.zeros((T, 1, D)), pool, table, [0, T], [T], None, 0.2, window=3, sinks=2)
    assert list(n[:7, 0]) == [1, 2, 3, 4, 5, 5, 5]
    assert np.allclose(o[139, 0], v[[0, 1, 137, 138, 139]].mean(0))
    o, *_ = A.attention(np.zeros((2, 1, D)), pool, np.array([[-1, 5]]), [0, 2], [T], None, 0.2)
    assert not o.any()                                   # no page is there
