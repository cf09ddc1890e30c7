"""The operators together, as a program uses them: norm, product, cache, attention, product; in a captured graph; on other streams."""
import numpy as np
import pytest
import torch

from oracle import attention_block as A
from oracle import bitnet_a48 as O
from paper_2411_04965_amd import binding as B
from paper_2411_04965_amd import synth as S
from tests.attention_util import BF16, rope_table
from tests.gpu_util import dev, host

pytestmark = pytest.mark.gpu
EPS = 1e-5
HIDDEN, HQ, H, D = 256, 4, 2, 64


class Block:
    """norm -> qkv (W1.58A4) -> cache -> attention -> o (sparse W1.58A8), weights packed once."""

    def __init__(self, n_pages=8):
        W = S.latent_weights((HQ + 2 * H) * D, HIDDEN, 3), S.latent_weights(HIDDEN, HQ * D, 4)
        self.W = W
        self.qkv, self.o = (B.pack_ternary(dev(w), EPS) for w in W)
        self.gamma_h = (1 + 0.1 * np.random.default_rng(5).standard_normal(HIDDEN)).astype(np.float32)
        self.gamma = dev(self.gamma_h)
        self.rope_h = rope_table(512, D)
        self.rope = dev(self.rope_h)
        self.pages = B.kv_pages_new(n_pages, H, D, "cuda")

    def step(self, x, r, table, qs, ln, window=0, sinks=0):
        M = x.shape[0]
        n = B.rmsnorm_quantize(x, self.gamma, B.BL_ACT_INT4_ABSMEAN, residual=r)
        y = B.bitlinear_gemm(n["q"], n["scale"], B.BL_ACT_INT4_ABSMEAN, M, HIDDEN, *self.qkv, (HQ + 2 * H) * D)
        q, k, v = (y[:, a * D:b * D].view(M, -1, D) for a, b in ((0, HQ), (HQ, HQ + H), (HQ + H, HQ + 2 * H)))
        B.kv_pages_append(k, v, self.pages, table, qs, ln, rope=self.rope)
        a = B.kv_pages_attention(q, self.pages, table, qs, ln, H, rope=self.rope, window=window, sinks=sinks, q_bits=4)
        return n["h"], y, a, B.bitlinear_a8_sparse(a.view(M, HQ * D), HQ * D // 2, *self.o, HIDDEN)


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_prompt_then_tokens_against_the_oracle():
    """Two sequences: a prompt each, then single tokens; every stage against the oracle's of the same inputs."""
    blk = Block()
    g = np.random.default_rng(41)
    table_h = np.array([[5, 2, 0, -1], [7, 1, -1, -1]], np.int32)
    table = torch.from_numpy(table_h).cuda()
    pool = A.Pages(np.zeros((8, A.page_bytes(H, D)), np.uint8), H, D)
    length = np.zeros(2, np.int32)
    for new in ([130, 40], [1, 1], [1, 1], [3, 90], [1, 0]):
        length = length + np.array(new, np.int32)
        qs_h = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        M = int(qs_h[-1])
        x, r = (S.snap_bf16(g.standard_normal((M, HIDDEN)).astype(np.float32)) for _ in range(2))
        h, y, a, out = blk.step(dev(x, BF16), dev(r, BF16), table, i32(*qs_h), i32(*length), window=100, sinks=1)
        hh, _, yn = A.rmsnorm(x, r, blk.gamma_h, 1e-5, True)
        q4, d4 = O.quant_int4(yn, EPS)
        T, alpha = O.ternarize(blk.W[0], EPS)[:2]
        acc = q4.astype(np.int64) @ T.astype(np.int64).T
        yo = O.bf16_round(((acc.astype(np.float32) * d4[:, None]).astype(np.float32) * np.float32(alpha)).astype(np.float32))
        assert np.array_equal(host(h), hh) and np.array_equal(host(y), yo)
        q, k, v = (yo[:, s * D:e * D].reshape(M, -1, D) for s, e in ((0, HQ), (HQ, HQ + H), (HQ + H, HQ + 2 * H)))
        A.append(pool, k, v, table_h, qs_h, length, blk.rope_h, EPS)
        o, ab, mass, unit, n = A.attention(q, pool, table_h, qs_h, length, blk.rope_h, float(np.float32(D ** -0.5)), 100, 1, 4)
        from tests.test_gpu_kv_attention import tolerance
        assert (np.abs(host(a) - o) <= tolerance(o, ab, mass, unit, n, D, 4)).all()
        ref = O.bitlinear_a8_sparse(host(a).reshape(M, -1), blk.W[1], HQ * D // 2, EPS, "bf16")["y"]
        assert np.array_equal(host(out), ref)


def test_captured_step_replayed():
    """A decode step in a graph; tokens, lengths and pages change between the replays, eager work runs in between."""
    blk, eager = Block(), Block()
    table = i32(3, 1, 6, -1).view(1, 4)
    g = np.random.default_rng(43)
    prompt = [dev(g.standard_normal((120, HIDDEN)), BF16) for _ in range(2)]
    for bl in (blk, eager):
        bl.step(*prompt, table, i32(0, 120), i32(120))
    x, r, tb, qs, ln = torch.zeros_like(prompt[0][:1]), torch.zeros_like(prompt[0][:1]), table.clone(), i32(0, 1), i32(121)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        blk.step(x, r, tb, qs, ln)                       # warm: allocations of the binding
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = blk.step(x, r, tb, qs, ln)
    for t in range(121, 135):                            # across the first page's end
        xn, rn = (dev(g.standard_normal((1, HIDDEN)), BF16) for _ in range(2))
        x.copy_(xn)
        r.copy_(rn)
        ln.fill_(t)
        for o in got:
            o.fill_(float("nan"))
        graph.replay()
        want = eager.step(xn, rn, table, qs, i32(t))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), "token %d" % t
    assert torch.equal(blk.pages[[3, 1]], eager.pages[[3, 1]])


def test_captured_norm_gradient():
    M, K = 70, 300
    g = np.random.default_rng(47)
    h, dy, ga = dev(g.standard_normal((M, K)), BF16), dev(g.standard_normal((M, K)), BF16), dev(g.standard_normal(K))
    rstd = torch.ones(M, device="cuda")
    ws = torch.empty(B.lib().rmsnorm_backward_workspace_bytes(M, K), dtype=torch.uint8, device="cuda")
    B.rmsnorm_backward(dy, h, rstd, ga, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.rmsnorm_backward(dy, h, rstd, ga, ws=ws)
    for k in range(4):
        dy.copy_(dev(g.standard_normal((M, K)), BF16))
        ws.fill_(255)
        graph.replay()
        want = B.rmsnorm_backward(dy, h, rstd, ga)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_streams_with_their_own_workspaces():
    """Calls that overlap in time give what they give alone."""
    blk = Block()
    table, g = i32(3, 1, 6, 2).view(1, 4), np.random.default_rng(53)
    blk.step(dev(g.standard_normal((500, HIDDEN)), BF16), None, table, i32(0, 500), i32(500))
    qs, ln = i32(0, 1), i32(500)
    Q = [dev(g.standard_normal((1, HQ, D)), BF16) for _ in range(8)]
    want = [B.kv_pages_attention(q, blk.pages, table, qs, ln, H, rope=blk.rope) for q in Q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None] * 8
    for i, q in enumerate(Q):
        with torch.cuda.stream(streams[i % 2]):
            got[i] = B.kv_pages_attention(q, blk.pages, table, qs, ln, H, rope=blk.rope)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_workspace_of_another_device_is_refused():
    h, rstd, gamma = (torch.ones(s, device="cuda") for s in ((3, 64), (3,), (64,)))
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.rmsnorm_backward(h, h, rstd, gamma, ws=ws)
    pages, table = B.kv_pages_new(1, 1, 64, "cuda"), i32(0).view(1, 1)
    q = torch.zeros((1, 1, 64), dtype=BF16, device="cuda")
    with pytest.raises(ValueError):
        B.kv_pages_attention(q, pages, table, i32(0, 1), i32(1), 1, ws=ws)
