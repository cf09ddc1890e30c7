"""Batches for the paged cache's GPU tests."""
import numpy as np
import torch

from oracle import attention_block as A
from paper_2411_04965_amd import binding as B
from paper_2411_04965_amd import synth as S
from tests.gpu_util import dev

BF16, F32 = torch.bfloat16, torch.float32


def rope_table(n, D):
    inv = 10000.0 ** (-2.0 * np.arange(D // 2) / D)
    a = np.arange(n)[:, None] * inv
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


class Batch:
    """Sequences with `new` rows each behind `ctx` cached positions; pages of the pool in any order, garbage in what nothing wrote."""

    def __init__(self, new, ctx, H, D, seed, max_pages=None, extra_rows=0):
        g = self.g = np.random.default_rng([37, seed, H, D, len(new)])
        self.H, self.D, self.new = H, D, list(new)
        self.total = [a + b for a, b in zip(new, ctx)]
        counts = [max(0, (t + 127) // 128) for t in self.total]
        self.max_pages = max_pages or max(max(counts), 1)
        n_pages = sum(counts) + 2
        ids = g.permutation(n_pages)[:sum(counts)]
        self.table = np.full((len(new), self.max_pages), -1, np.int32)
        at = 0
        for s, c in enumerate(counts):
            c = min(c, self.max_pages)
            self.table[s, :c] = ids[at:at + c]
            at += c
        self.q_start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.kv_len = np.array(self.total, np.int32)
        self.T = int(self.q_start[-1]) + extra_rows
        raw = g.integers(0, 256, (n_pages, A.page_bytes(H, D))).astype(np.uint8)
        self.pool = A.Pages(raw, H, D)
        w = self.pool.n_codes
        self.pool.floats[:, :, 2 * w:2 * w + 256] = np.nan           # scales of places that nothing wrote
        self.rope = rope_table(self.max_pages * 128, D)

    def fill(self, upto=None):
        """Cached positions of every sequence (all, or those before its new rows), straight into the pool's bytes."""
        for s, t in enumerate(self.total):
            n = t if upto is None else t - self.new[s]
            n = min(n, self.max_pages * 128)
            if n <= 0:
                continue
            x = self.g.standard_normal((2, n, self.H, self.D)).astype(np.float32)
            fast_put(self.pool, self.table[s], x)

    def dev(self):
        self.pages_d = torch.from_numpy(self.pool.raw.copy()).cuda()
        self.table_d, self.q_d, self.len_d = (torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in (self.table, self.q_start, self.kv_len))
        self.rope_d = dev(self.rope)
        return self.pages_d, self.table_d, self.q_d, self.len_d


def fast_put(pool, pages, x):
    """Positions 0 .. n - 1 of one sequence from x [2, n, H, D], quantized by the oracle, packed array-wise."""
    n, D, U = x.shape[1], pool.D, pool.U
    i = np.arange(32)
    mb, sb = 4 * (i % 8) + 2 * (i // 8 % 2), 4 * (i % 8) + 3 - i // 8
    slots = np.array([A.slot(t) for t in range(128)])
    nc = pool.n_codes
    for values in (0, 1):
        q, d = A.levels(x[values], np.arange(n), 1e-5)
        for k in range((n + 127) // 128):
            lo, hi = 128 * k, min(n, 128 * k + 128)
            lv = np.zeros((128, pool.H, 32 * U), np.int64)
            lv[:hi - lo, :, :D] = q[lo:hi]
            mag, neg = np.abs(lv), (lv < 0).astype(np.int64)
            low = mag[0] & 1
            if k == 0:
                mag[0] >>= 1
            for h in range(pool.H):
                w = pool.words[pages[k], h]
                if values:
                    m, s = (t[:, h].T.reshape(32 * U, 4, 32) for t in (mag, neg))
                else:
                    m, s = (t[:, h].reshape(128, U, 32) for t in (mag, neg))
                words = np.stack([(m[..., :16] << mb[:16]).sum(-1), (m[..., 16:] << mb[16:]).sum(-1), (s << sb).sum(-1)], -1)
                if not values:
                    by_slot = np.empty_like(words)
                    by_slot[slots] = words
                    words = by_slot
                w[values * nc:(values + 1) * nc] = words.reshape(-1).astype(np.uint32)
                if k == 0:
                    at = 2 * nc + 256 + values * U
                    w[at:at + U] = (low[h].reshape(U, 32) << sb).sum(-1).astype(np.uint32)
                f = pool.floats[pages[k], h]
                f[2 * nc + 128 * values:2 * nc + 128 * values + hi - lo] = d[lo:hi, h]


def states(g, shape, dtype):
    x = g.standard_normal(shape).astype(np.float32)
    return S.snap_bf16(x) if dtype == BF16 else x
