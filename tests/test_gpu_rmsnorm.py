"""RMS norm with codes, and its gradient, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import attention_block as A
from oracle import bitnet_a48 as O
from paper_2411_04965_amd import binding as B
from paper_2411_04965_amd import synth as S
from tests.gpu_util import decode_int4, decode_int4_mx6, decode_int8, dev, host

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def inputs(M, K, dtype, seed, residual=True):
    g = np.random.default_rng([23, M, K, seed])
    snap = S.snap_bf16 if dtype == BF16 else (lambda x: x.astype(np.float32))
    x = snap((g.standard_normal((M, K)) * np.exp2(g.integers(-3, 4, (M, 1)))).astype(np.float32))
    if M > 2:
        x[2] = 0.0                                       # a row of zeros
    r = snap(g.standard_normal((M, K)).astype(np.float32)) if residual else None
    if residual and M > 2:
        r[2] = 0.0
    return x, r, (1 + 0.3 * g.standard_normal(K)).astype(np.float32)


@pytest.mark.parametrize("mode", [B.BL_ACT_INT4_ABSMEAN, B.BL_ACT_INT4_ABSMEAN_MX6, B.BL_ACT_TOPK_INT8_ABSMAX])
@pytest.mark.parametrize("M,K,dtype,residual", [
    (1, 1, F32, False), (3, 7, BF16, True), (5, 256, BF16, True), (33, 1000, F32, True), (9, 1537, BF16, False), (40, 2048, BF16, True),
    (4, 4096, F32, True), (3, 5460, BF16, True), (5, 8191, BF16, False), (3, 16384, F32, False), (3, 11008, BF16, True),
    (4, 20001, BF16, True), (3, 32768, F32, True)])
def test_rmsnorm_quantize(M, K, dtype, residual, mode):
    print("rmsnorm_quantize M=%d K=%d %s mode %d" % (M, K, dtype, mode), flush=True)
    x, r, ga = inputs(M, K, dtype, mode, residual)
    h, rstd, y = A.rmsnorm(x, r, ga, EPS, dtype == BF16)
    q, d = O.quant_int8(y, EPS) if mode == B.BL_ACT_TOPK_INT8_ABSMAX else O.quant_int4(y, EPS)
    got = B.rmsnorm_quantize(dev(x, dtype), dev(ga), mode, residual=None if r is None else dev(r, dtype), norm_eps=EPS, eps=EPS)
    raw = host(got["q"])
    codes = {B.BL_ACT_INT4_ABSMEAN: decode_int4, B.BL_ACT_INT4_ABSMEAN_MX6: decode_int4_mx6, B.BL_ACT_TOPK_INT8_ABSMAX: decode_int8}[mode](raw, M, K)
    assert np.array_equal(host(got["h"]), h)
    assert np.array_equal(host(got["rstd"]), rstd)
    assert np.array_equal(host(got["scale"]), d)
    assert np.array_equal(codes, q)


def test_codes_are_those_of_the_quantizer_and_feed_the_product():
    M, N, K = 37, 200, 1000
    x, r, ga = inputs(M, K, BF16, 1)
    W = S.latent_weights(N, K, 5)
    for mode, layout in ((B.BL_ACT_INT4_ABSMEAN, B.BL_W_GEMM), (B.BL_ACT_INT4_ABSMEAN_MX6, B.BL_W_MX2), (B.BL_ACT_TOPK_INT8_ABSMAX, B.BL_W_GEMM)):
        got = B.rmsnorm_quantize(dev(x, BF16), dev(ga), mode, residual=dev(r, BF16))
        y = dev(A.rmsnorm(x, r, ga, 1e-5, True)[2])
        want = B.quantize_act(y, mode, topk=K)
        p, a = B.pack_ternary(dev(W), EPS, layout)
        ya = B.bitlinear_gemm(got["q"], got["scale"], mode, M, K, p, a, N, layout)
        yb = B.bitlinear_gemm(want["q"], want["scale"], mode, M, K, p, a, N, layout)
        assert torch.equal(got["scale"], want["scale"]) and torch.equal(ya, yb)
        assert torch.equal(B.unpack_act(got["q"], mode, M, K), B.unpack_act(want["q"], mode, M, K))


def test_residual_in_place_and_nullable_outputs():
    M, K = 6, 777
    x, r, ga = inputs(M, K, BF16, 2)
    X, R, G = dev(x, BF16), dev(r, BF16), dev(ga)
    want = B.rmsnorm_quantize(X, G, B.BL_ACT_INT4_ABSMEAN, residual=R)
    L = B.lib()
    for inplace in (X.clone(), R.clone()):
        a, b = (inplace, R) if torch.equal(inplace, X) else (X, inplace)
        q, sc = torch.empty_like(want["q"]), torch.empty_like(want["scale"])
        assert L.rmsnorm_quantize(a.data_ptr(), b.data_ptr(), B.BL_BF16, M, K, G.data_ptr(), 1e-5, 0, 1e-5, inplace.data_ptr(), None,
                                  q.data_ptr(), sc.data_ptr(), B._stream()) == 0
        torch.cuda.synchronize()
        assert torch.equal(inplace, want["h"]) and torch.equal(q, want["q"]) and torch.equal(sc, want["scale"])


def bound_backward(dY, H, rstd, ga, dH, dx, dg, out_eps):
    """What float32 steps can lose.  xh, a: one rounding each (2^-24 relative); a sum of n float32 products, however ordered, loses at
    most n 2^-24 of the sum of magnitudes; a few more single roundings; then the output's own."""
    u = 2.0 ** -24
    M, K = H.shape
    xh = np.abs(H * rstd[:, None])
    a = np.abs(dY * ga)
    mean = (a * xh).mean(1, keepdims=True)
    ex = rstd[:, None] * (6 * u * a + xh * mean * (16 + 8 + 6) * u)       # a thread adds 16 to 64 products, then float64
    ex = rstd[:, None] * (6 * u * a + xh * mean * (64 + 8) * u) + 2 * u * (0 if dH is None else np.abs(dH)) + 2 * u * np.abs(dx)
    eg = (np.abs(dY) * xh).sum(0) * (M + 4) * u
    return ex + out_eps * (np.abs(dx) + ex) + 1e-37, eg + 1e-37


@pytest.mark.parametrize("M,K,dtype,residual", [
    (1, 1, F32, True), (2, 9, BF16, True), (7, 1024, BF16, False), (600, 300, F32, True), (1030, 513, BF16, True), (5, 4096, F32, False),
    (3, 5460, BF16, True), (4, 16384, F32, True), (3, 16385, BF16, True), (2, 32768, F32, False)])
def test_rmsnorm_backward(M, K, dtype, residual):
    print("rmsnorm_backward M=%d K=%d %s" % (M, K, dtype), flush=True)
    x, r, ga = inputs(M, K, dtype, 3)
    h, rstd, _ = A.rmsnorm(x, None, ga, EPS, dtype == BF16)
    g = np.random.default_rng([29, M, K])
    snap = S.snap_bf16 if dtype == BF16 else (lambda t: t)
    dy = snap(g.standard_normal((M, K)).astype(np.float32))
    dh = r if residual else None
    dx, dg = A.rmsnorm_backward(dy, h, rstd, ga, dh)
    ex, eg = bound_backward(dy.astype(float), h.astype(float), rstd.astype(float), ga.astype(float), dh, dx, dg,
                            2.0 ** -8 if dtype == BF16 else 2.0 ** -24)
    args = (dev(dy, dtype), dev(h, dtype), dev(rstd), dev(ga))
    got = B.rmsnorm_backward(*args, dH=None if dh is None else dev(dh, dtype))
    assert (np.abs(host(got[0]) - dx) <= ex).all()
    assert (np.abs(host(got[1]) - dg) <= eg).all()
    again = B.rmsnorm_backward(*args, dH=None if dh is None else dev(dh, dtype))
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])          # a fixed order


def test_gradient_against_differences_of_the_forward_pass():
    """d loss / d X of loss = sum(w * y): differences of the kernel's own rstd and h in float64."""
    M, K = 2, 40
    x, _, ga = inputs(M, K, F32, 4, False)
    w = np.random.default_rng(31).standard_normal((M, K)).astype(np.float32)
    rstd = B.rmsnorm_quantize(dev(x), dev(ga), B.BL_ACT_INT4_ABSMEAN)["rstd"]
    dx, _ = B.rmsnorm_backward(dev(w), dev(x), rstd, dev(ga))

    def loss(t):
        return float((w * t / np.sqrt((t * t).mean(1, keepdims=True) + 1e-5) * ga).sum())
    e = 1e-5
    for m in range(M):
        for k in range(0, K, 7):
            p, n = x.astype(float), x.astype(float)
            p[m, k] += e
            n[m, k] -= e
            # the difference's own error is e^2 / 6 of the third derivative, and 2^-52 loss / e: both below 1e-8 here
            assert abs((loss(p) - loss(n)) / (2 * e) - float(dx[m, k])) < 1e-5
