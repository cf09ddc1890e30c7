"""The marshalling module's norm, cache and attention against the general way through ctypes: the same outputs, the same errors, and
calls it leaves alone."""
import numpy as np
import pytest
import torch

from paper_2411_04965_amd import binding as B
from tests.test_gpu_marshal import BF16, Quiet, Refuses, Sub, both

pytestmark = pytest.mark.gpu
H, HQ, D, T = 2, 4, 64, 5


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def setting():
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((T, (HQ + 2 * H) * D), generator=g, device="cuda")
    rope = torch.randn((256, D), generator=g, device="cuda")
    return x, rope, i32(1, 0).view(1, 2), i32(0, T), i32(T)


def same(a, b):
    if isinstance(a, dict):
        assert list(a) == list(b)
        return all(same(a[k], b[k]) for k in a)
    return type(a) is type(b) and a.dtype == b.dtype and torch.equal(a, b) and a.requires_grad == b.requires_grad


def compare(monkeypatch, calls):
    for i, call in enumerate(calls):
        with monkeypatch.context() as mp:
            n, c = both(mp, call)
        assert n[0] == c[0], (i, n, c)
        if n[0] == "value":
            assert same(n[1], c[1]), i
        elif issubclass(n[0], B.BitlinearError) or n[0] in (ValueError, TypeError):
            assert n[1] == c[1], i


def test_norm(monkeypatch):
    X = torch.randn((7, 200), device="cuda")
    gamma = torch.rand(200, device="cuda")
    modes = (B.BL_ACT_INT4_ABSMEAN, B.BL_ACT_INT4_ABSMEAN_MX6, B.BL_ACT_TOPK_INT8_ABSMAX)

    def codes(x, m, r):                                  # (the bytes of a block's tokens behind M are nobody's)
        d = B.rmsnorm_quantize(x, gamma, m, residual=r)
        return dict(d, q=B.unpack_act(d["q"], m, *x.shape))

    calls = [lambda x=x, r=r, m=m: codes(x, m, r) for m in modes
             for x in (X, X.to(BF16)) for r in (None, x * 2)]
    for x in (torch.nn.Parameter(X), X.as_subclass(Sub), X.half(), X.T, X.cpu(), X[0], X[:0]):
        calls += [lambda x=x: B.rmsnorm_quantize(x, gamma, 0)]
    calls += [lambda: B.rmsnorm_quantize(X, gamma[:100], 0), lambda: B.rmsnorm_quantize(X, gamma.to(BF16), 0),
              lambda: B.rmsnorm_quantize(X, gamma, 2), lambda: B.rmsnorm_quantize(X, gamma, 99), lambda: B.rmsnorm_quantize(X, gamma, -1),
              lambda: B.rmsnorm_quantize(X, gamma, 0, residual=X.to(BF16)), lambda: B.rmsnorm_quantize(X, gamma, 0, residual=X[:3]),
              lambda: B.rmsnorm_quantize(X, gamma, 0, residual=X.cpu()), lambda: B.rmsnorm_quantize(X, gamma, 0, norm_eps=-1.0),
              lambda: B.rmsnorm_quantize(X, gamma, 0, eps=0), lambda: B.rmsnorm_quantize(X, gamma.cpu(), 0)]
    compare(monkeypatch, calls)
    assert B.rmsnorm_quantize(X, gamma, 0)["h"] is X


def test_cache_and_attention(monkeypatch):
    x, rope, table, qs, ln = setting()
    xb = x.to(BF16)

    def q(t):
        return t[:, :HQ * D].view(T, HQ, D)

    def kv(t):
        return t[:, HQ * D:(HQ + H) * D].view(T, H, D), t[:, (HQ + H) * D:].view(T, H, D)

    def append(t=xb, pages=None, **k):
        k = dict(dict(page_table=table, q_start=qs, kv_len=ln, rope=rope), **k)
        p = B.kv_pages_new(2, H, D, "cuda") if pages is None else pages
        a, b = kv(t) if torch.is_tensor(t) else t
        B.kv_pages_append(a, b, p, **k)
        return p

    pages = append()
    k_, v_ = kv(xb)
    compare(monkeypatch, [append, lambda: append(x), lambda: append(rope=None), lambda: append((k_.contiguous(), v_)), lambda: append(eps=0),
                          lambda: append(eps=-1.0), lambda: append((k_, v_.float())), lambda: append((k_[:3], v_)),
                          lambda: append((k_.half(), v_.half())), lambda: append((k_.transpose(1, 2), v_)), lambda: append((k_.cpu(), v_)),
                          lambda: append(page_table=table.long()), lambda: append(page_table=table[0]), lambda: append(q_start=qs[:1]),
                          lambda: append(kv_len=ln.cpu()), lambda: append(rope=rope[:100]), lambda: append(rope=rope[:, :32]),
                          lambda: append(pages=pages[:, :-128].contiguous()), lambda: append(pages=pages.view(torch.int8))])

    def attend(t=xb, pages=pages, H=H, **k):
        k = dict(dict(rope=rope), **k)
        return B.kv_pages_attention(q(t) if t.dim() == 2 else t, pages, table, qs, ln, H, **k)

    out = torch.empty((T, HQ, D), dtype=BF16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    compare(monkeypatch, [attend, lambda: attend(x), lambda: attend(rope=None, scale=0.5), lambda: attend(q_bits=4, window=3, sinks=1),
                          lambda: attend(out=out), lambda: attend(ws=ws), lambda: attend(ws=ws[:0]), lambda: attend(ws=ws.cpu()),
                          lambda: attend(ws=ws.view(-1, 2)[:, 0]), lambda: attend(out=out.float()), lambda: attend(out=out[:2]),
                          lambda: attend(scale=1), lambda: attend(scale=-1.0), lambda: attend(window=-1), lambda: attend(sinks=2.5),
                          lambda: attend(q_bits=8), lambda: attend(H=3), lambda: attend(H=0), lambda: attend(H=np.int64(H)),
                          lambda: attend(q(xb).as_subclass(Sub)), lambda: attend(torch.nn.Parameter(x)), lambda: attend(xb.half()),
                          lambda: attend(q(xb)[..., ::2]), lambda: attend(q(xb)[:0]), lambda: attend(pages=pages.cpu())])
    assert attend(out=out) is out


def test_plain_calls_only():
    x, rope, table, qs, ln = setting()
    q, k, v = x[:, :HQ * D].view(T, HQ, D), x[:, HQ * D:(HQ + H) * D].view(T, H, D), x[:, (HQ + H) * D:].view(T, H, D)
    pages, m, gamma = B.kv_pages_new(2, H, D, "cuda"), B._native(), torch.ones(D, device="cuda")
    n = x[:, :D].contiguous()
    args = (pages, table, qs, ln, H, rope, None, 0, 0, 16, 1e-5, None, None)
    assert m.kv_append(k, v, pages, table, qs, ln, rope, 1e-5) == 0
    assert torch.is_tensor(m.kv_attention(q, *args))
    assert type(m.norm(n, gamma, 0, None, 1e-5, 1e-5)) is dict
    with Quiet():
        assert m.kv_append(k, v, pages, table, qs, ln, rope, 1e-5) is None
        assert m.kv_attention(q, *args) is None and m.norm(n, gamma, 0, None, 1e-5, 1e-5) is None
    ref = B.kv_pages_attention(q, pages, table, qs, ln, H, rope=rope)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = B.kv_pages_attention(q, pages, table, qs, ln, H, rope=rope)
    torch.cuda.current_stream().wait_stream(s)
    y.record_stream(torch.cuda.current_stream())
    assert torch.equal(y, ref)


def test_errors_of_a_dispatch_mode(monkeypatch):
    x, rope, table, qs, ln = setting()
    q, pages, gamma = x[:, :HQ * D].contiguous().view(T, HQ, D), B.kv_pages_new(2, H, D, "cuda"), torch.ones(D, device="cuda")
    n = x[:, :D].contiguous()
    for call in (lambda: B.kv_pages_attention(q, pages, table, qs, ln, H), lambda: B.rmsnorm_quantize(n, gamma, 0, residual=n)):
        def inside(call=call):
            with Refuses():
                return call()
        with monkeypatch.context() as mp:
            a, c = both(mp, inside)
        assert a == c and a[0] is KeyError, (a, c)
