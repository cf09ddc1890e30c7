"""What the norm and the paged cache's calls refuse, on the host, before anything is enqueued (no GPU: pointers are numbers)."""
import pytest

from paper_2411_04965_amd import binding as B

P = 4096                                                 # a 128-byte aligned address that nothing reads
INF = float("inf")


@pytest.fixture(scope="module")
def L():
    import os

    from paper_2411_04965_amd import build
    if not os.path.exists(B.LIB_PATH):
        build.build(verbose=False)
    return B.lib()


def append(L, K=P, ldk=256, V=P, ldv=256, dt=1, T=4, H=2, D=128, qs=P, kl=P, S=1, tab=P, mp=2, rope=None, n_pos=0, eps=1e-5, pages=P,
           n_pages=4):
    return L.kv_pages_append(K, ldk, V, ldv, dt, T, H, D, qs, kl, S, tab, mp, rope, n_pos, eps, pages, n_pages, None)


def read(L, K=P, V=P, dt=1, T=4, H=2, D=128, qs=P, kl=P, S=1, tab=P, mp=2, pages=P, n_pages=4):
    return L.kv_pages_read(pages, n_pages, qs, kl, S, tab, mp, T, H, D, K, V, dt, None)


def attend(L, Q=P, ldq=512, dt=1, T=4, Hq=4, H=2, D=128, bits=16, qs=P, kl=P, S=1, tab=P, mp=2, rope=None, n_pos=0, scale=0.1, eps=1e-5,
           window=0, sinks=0, pages=P, n_pages=4, O=P, ws=P, wsb=1 << 30):
    return L.kv_pages_attention(Q, ldq, dt, T, Hq, H, D, bits, qs, kl, S, tab, mp, rope, n_pos, scale, eps, window, sinks, pages, n_pages, O,
                                ws, wsb, None)


@pytest.mark.parametrize("call", [append, read, attend])
@pytest.mark.parametrize("bad,status", [
    (dict(qs=None), -1), (dict(kl=None), -1), (dict(tab=None), -1), (dict(pages=None), -1), (dict(dt=2), -1), (dict(T=0), -1),
    (dict(S=0), -1), (dict(mp=0), -1), (dict(n_pages=0), -1), (dict(H=0), -1), (dict(D=0), -1), (dict(D=127), -2), (dict(D=258), -2),
    (dict(T=1 << 31), -2), (dict(S=1 << 31), -2), (dict(mp=1 << 25), -2), (dict(n_pages=1 << 31), -2), (dict(pages=P + 64), -3),
    (dict(qs=P + 2), -3), (dict(kl=P + 1), -3), (dict(tab=P + 2), -3)])
def test_shared_refusals(L, call, bad, status):
    assert call(L, **bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(K=None), -1), (dict(V=None), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(ldk=255), -1), (dict(ldv=0), -1),
    (dict(ldk=-256), -1), (dict(ldv=1 << 50), -1), (dict(K=P + 1), -3), (dict(V=P + 2, dt=0), -3), (dict(rope=P, n_pos=255), -2),
    (dict(rope=P + 2, n_pos=256), -3)])
def test_append_refusals(L, bad, status):
    assert append(L, **bad) == status


@pytest.mark.parametrize("bad,status", [(dict(K=None, V=None), -1), (dict(K=P + 8), -3), (dict(V=P + 4), -3)])
def test_read_refusals(L, bad, status):
    assert read(L, **bad) == status


@pytest.mark.parametrize("bad,status", [
    (dict(Q=None), -1), (dict(O=None), -1), (dict(bits=8), -1), (dict(bits=3), -1), (dict(eps=-1.0), -1), (dict(scale=0.0), -1),
    (dict(scale=-0.1), -1), (dict(scale=INF), -1), (dict(scale=float("nan")), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
    (dict(Hq=3), -1), (dict(Hq=0), -1), (dict(ldq=511), -1), (dict(ldq=1 << 50), -1), (dict(Q=P + 1), -3), (dict(Q=P + 2, dt=0), -3), (dict(O=P + 2), -3),
    (dict(rope=P, n_pos=255), -2), (dict(T=(1 << 30) - 1, Hq=8, ldq=1024), -2),
    (dict(mp=64, ws=None), -4), (dict(mp=64, wsb=64), -4), (dict(mp=64, ws=P + 8), -3)])
def test_attention_refusals(L, bad, status):
    assert attend(L, **bad) == status


def test_page_and_workspace_sizes(L):
    assert L.kv_page_bytes(1, 128) == 2 * 128 * 48 + 1024 + 128 and L.kv_page_bytes(8, 100) == 8 * L.kv_page_bytes(1, 128)
    assert L.kv_page_bytes(3, 2) == 3 * (2 * 128 * 12 + 1152) and L.kv_page_bytes(1, 256) % 128 == 0
    for bad in ((0, 128), (2, 0), (2, 3), (2, 258), (-1, 64), (1 << 40, 64)):
        assert L.kv_page_bytes(*bad) == 0
    ws = L.kv_pages_attention_workspace_bytes
    assert ws(1, 1, 8, 8, 128, 1) == 0                   # one page: nothing to split
    assert ws(1, 1, 8, 8, 128, 1024) > 0
    assert ws(1 << 20, 1, 8, 8, 128, 1024) == 0          # many rows: nothing to join
    for bad in ((0, 1, 8, 8, 128, 9), (1, 0, 8, 8, 128, 9), (1, 1, 9, 8, 128, 9), (1, 1, 8, 0, 128, 9), (1, 1, 8, 8, 300, 9), (1, 1, 8, 8, 64, 0)):
        assert ws(*bad) == 0


def norm(L, X=P, R=None, dt=1, M=4, K=256, gamma=P, ne=1e-5, mode=0, eps=1e-5, H=None, rstd=None, q=P, scale=P):
    return L.rmsnorm_quantize(X, R, dt, M, K, gamma, ne, mode, eps, H, rstd, q, scale, None)


@pytest.mark.parametrize("bad,status", [
    (dict(X=None), -1), (dict(gamma=None), -1), (dict(q=None), -1), (dict(scale=None), -1), (dict(dt=5), -1), (dict(mode=9), -1),
    (dict(eps=-1.0), -1), (dict(ne=-1.0), -1), (dict(ne=float("nan")), -1), (dict(M=0), -1), (dict(K=0), -1), (dict(K=32769), -2),
    (dict(M=1 << 31), -2), (dict(mode=2), -6), (dict(mode=4), -6), (dict(mode=5), -6), (dict(mode=6), -6), (dict(mode=7), -6),
    (dict(X=P + 2), -3), (dict(R=P + 8), -3), (dict(H=P + 4), -3), (dict(q=P + 4), -3), (dict(gamma=P + 2), -3), (dict(rstd=P + 1), -3),
    (dict(scale=P + 2), -3)])
def test_norm_refusals(L, bad, status):
    assert norm(L, **bad) == status


def grad(L, dY=P, H=P, rstd=P, gamma=P, dH=None, dt=1, M=4, K=256, dX=P, dg=P, ws=P, wsb=1 << 30):
    return L.rmsnorm_backward(dY, H, rstd, gamma, dH, dt, M, K, dX, dg, ws, wsb, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dY=None), -1), (dict(H=None), -1), (dict(rstd=None), -1), (dict(gamma=None), -1), (dict(dX=None), -1), (dict(dg=None), -1),
    (dict(dt=3), -1), (dict(M=0), -1), (dict(K=-1), -1), (dict(K=40000), -2), (dict(ws=None), -4), (dict(wsb=100), -4), (dict(ws=P + 8), -3),
    (dict(dY=P + 2), -3), (dict(dH=P + 2), -3), (dict(dX=P + 8), -3), (dict(dg=P + 2), -3)])
def test_gradient_refusals(L, bad, status):
    assert grad(L, **bad) == status


def test_binding_refuses_what_the_library_cannot_see():
    import torch
    t = torch.zeros((4, 256))
    with pytest.raises(ValueError):                      # host tensors
        B.rmsnorm_quantize(t, torch.ones(256), B.BL_ACT_INT4_ABSMEAN)
    with pytest.raises(ValueError):
        B.kv_pages_append(t.view(4, 2, 128), t.view(4, 2, 128), t, t, t, t)
    with pytest.raises(B.BitlinearError):
        B.kv_pages_new(4, 2, 258, "cpu")
