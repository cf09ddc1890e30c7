"""CPU oracle of what stands around the quantized linears in a decoder's attention half: the RMS norm with codes and its gradient,
the paged low-bit key / value cache, and attention over it.  numpy; float32 single operations where the kernels' integers depend on
them, float64 elsewhere; formats written from include/bitlinear.h.  Test infrastructure: the library does not use it."""
import numpy as np

from oracle import bitnet_a48 as O

F32, F64 = np.float32, np.float64
PAGE = 128


# ---------------------------------------------------------------- norm
def rmsnorm(X, R, gamma, norm_eps, bf16):
    """(h, rstd, y): h = X + R in the stream's type, rstd from float64, y = (h * rstd) * gamma in float32 steps."""
    h = np.asarray(X, F32)
    if R is not None:
        h = (h + np.asarray(R, F32)).astype(F32)
        h = O.bf16_round(h) if bf16 else h
    ms = (h.astype(F64) ** 2).mean(1)
    rstd = (1.0 / np.sqrt(ms + F64(F32(norm_eps)))).astype(F32)
    y = ((h * rstd[:, None]).astype(F32) * np.asarray(gamma, F32)).astype(F32)
    return h, rstd, y


def rmsnorm_backward(dY, H, rstd, gamma, dH=None):
    """float64 (dX, dgamma) with the given rstd."""
    dY, H, rstd, gamma = (np.asarray(t, F64) for t in (dY, H, rstd, gamma))
    xh = H * rstd[:, None]
    a = dY * gamma
    dX = rstd[:, None] * (a - xh * (a * xh).mean(1, keepdims=True))
    return dX if dH is None else dX + np.asarray(dH, F64), (dY * xh).sum(0)


# ---------------------------------------------------------------- pages
def rotate(x, table, pos):
    """float32 [T, H, D] rotated with the table's rows `pos`: pairs (i, i + D / 2), single float32 operations."""
    half = x.shape[2] // 2
    c, s = table[pos][:, None, :half].astype(F32), table[pos][:, None, half:].astype(F32)
    a, b = x[..., :half].astype(F32), x[..., half:].astype(F32)
    return np.concatenate([(a * c).astype(F32) - (b * s).astype(F32), (b * c).astype(F32) + (a * s).astype(F32)], 2).astype(F32)


def levels(x, pos, eps):
    """Levels int [T, H, D] and scales float32 [T, H] of head vectors at positions `pos`: 4 bits at position 0, else 3."""
    q, d = np.zeros(x.shape, np.int64), np.zeros(x.shape[:2], F32)
    for bits, at in ((4, pos == 0), (3, pos != 0)):
        if at.any():
            codes, dd = O.quant_heads(x[at], bits, eps)
            q[at], d[at] = codes.astype(np.int64) - 2 ** (bits - 1), dd
    return q, d


def page_bytes(H, D):
    return H * (2 * PAGE * 12 * ((D + 31) // 32) + 2 * PAGE * 4 + 128)


def slot(t):
    a, b, c, d = t // 64, t // 16 % 4, t // 4 % 4, t % 4
    return 64 * a + 16 * c + 4 * b + d


class Pages:
    """A page pool as bytes, written and read code by code."""

    def __init__(self, raw, H, D):
        self.raw = np.ascontiguousarray(raw, np.uint8)
        self.H, self.D, self.U = H, D, (D + 31) // 32
        self.words = self.raw.view("<u4").reshape(self.raw.shape[0], H, -1)
        self.floats = self.raw.view("<f4").reshape(self.raw.shape[0], H, -1)
        self.n_codes = PAGE * self.U * 3

    def _group(self, values, tok, ch):
        """(first word of the code's three, the code's number of the 32)"""
        if values:
            return self.n_codes + (ch * 4 + tok // 32) * 3, tok % 32
        return (slot(tok) * self.U + ch // 32) * 3, ch % 32

    def _low(self, values, ch):
        i = ch % 32
        return 2 * self.n_codes + 2 * PAGE + values * self.U + ch // 32, 4 * (i % 8) + 3 - i // 8

    def put(self, page, h, values, tok, q, scale, first):
        """Levels q [D] of one token; the padding channels' codes become 0 with them."""
        w = self.words[page, h]
        for ch in range(32 * self.U if not values else self.D):
            v = int(q[ch]) if ch < self.D else 0
            m = abs(v) // 2 if first else abs(v)
            at, i = self._group(values, tok, ch)
            mb, sb = 4 * (i % 8) + 2 * (i // 8 % 2), 4 * (i % 8) + 3 - i // 8
            w[at + i // 16] = (int(w[at + i // 16]) & ~(3 << mb)) | (m << mb)
            w[at + 2] = (int(w[at + 2]) & ~(1 << sb)) | ((v < 0) << sb)
            if first:
                lw, lb = self._low(values, ch)
                w[lw] = (int(w[lw]) & ~(1 << lb)) | ((abs(v) % 2) << lb)
        self.floats[page, h, 2 * self.n_codes + values * PAGE + tok] = scale

    def get(self, page, h, values, first_page):
        """(levels int [128, D], scales [128]) of a head's keys or values."""
        w = self.words[page, h].astype(np.int64)
        out = np.zeros((PAGE, self.D), np.int64)
        tok = np.arange(PAGE)
        for ch in range(self.D):
            at, i = self._group(values, tok, ch) if values else ((slot(tok) * self.U + ch // 32) * 3, np.full(PAGE, ch % 32))
            m = (w[at + i // 16] >> (4 * (i % 8) + 2 * (i // 8 % 2))) & 3
            neg = (w[at + 2] >> (4 * (i % 8) + 3 - i // 8)) & 1
            if first_page:
                lw, lb = self._low(values, ch)
                m[0] = 2 * m[0] + ((w[lw] >> lb) & 1)
            out[:, ch] = np.where(neg == 1, -m, m)
        s = 2 * self.n_codes + values * PAGE
        return out, self.floats[page, h, s:s + PAGE].copy()


def rows_of(q_start, kv_len, s):
    """(first row, positions of the rows) of sequence s."""
    n = int(q_start[s + 1]) - int(q_start[s])
    return int(q_start[s]), int(kv_len[s]) - n + np.arange(n)


def append(pool, K, V, table, q_start, kv_len, rope, eps):
    """Writes a batch into the pool (K already float32 values of the input type)."""
    for s in range(len(kv_len)):
        r0, pos = rows_of(q_start, kv_len, s)
        ok = np.array([p >= 0 and p // PAGE < table.shape[1] and 0 <= table[s, p // PAGE] < pool.raw.shape[0] for p in pos], bool)
        if not ok.any():
            continue
        rows, pos = r0 + np.nonzero(ok)[0], pos[ok]
        k = K[rows] if rope is None else rotate(K[rows], rope, pos)
        for values, x in ((0, k), (1, V[rows])):
            q, d = levels(x, pos, eps)
            for i, p in enumerate(pos):
                for h in range(pool.H):
                    pool.put(table[s, p // PAGE], h, values, p % PAGE, q[i, h], d[i, h], p == 0)


def cached(pool, table, s, h, values):
    """float32 values [128 max_pages, D] of a sequence's head, and which places have a page."""
    out = np.zeros((table.shape[1] * PAGE, pool.D), F32)
    there = np.zeros(table.shape[1] * PAGE, bool)
    for k, page in enumerate(table[s]):
        if 0 <= page < pool.raw.shape[0]:
            q, d = pool.get(page, h, values, k == 0)
            with np.errstate(invalid="ignore", over="ignore"):
                out[PAGE * k:PAGE * (k + 1)] = q.astype(F32) * d[:, None]
            there[PAGE * k:PAGE * (k + 1)] = True
    return out, there


# ---------------------------------------------------------------- attention
def attention(Q, pool, table, q_start, kv_len, rope, scale, window=0, sinks=0, q_bits=16, eps=O.DEFAULT_EPS):
    """float64 outputs [T, Hq, D] (NaN in rows of no sequence), and what a tolerance needs: sum p |v| / sum p [T, Hq, D], the largest
    scale * sum |q| |k| and scale * max |q| * sum |k| over visible keys [T, Hq, 2], largest |v| over sum p [T, Hq], visible keys [T, Hq]."""
    T, Hq, D = Q.shape
    G = Hq // pool.H
    o, a = np.full((T, Hq, D), np.nan), np.zeros((T, Hq, D))
    mass, unit, seen_n = np.zeros((T, Hq, 2)), np.zeros((T, Hq)), np.zeros((T, Hq), int)
    for s in range(len(kv_len)):
        r0, pos = rows_of(q_start, kv_len, s)
        if not len(pos):
            continue
        q = np.asarray(Q[r0:r0 + len(pos)], F32)
        if rope is not None:
            q = rotate(q, rope, np.clip(pos, 0, len(rope) - 1))
        if q_bits == 4:
            c, d = O.quant_heads(q, 4, eps)
            q = (c.astype(F64) - 8) * d[:, :, None].astype(F64)
        q = q.astype(F64)
        for h in range(pool.H):
            k, there = cached(pool, table, s, h, 0)
            v, _ = cached(pool, table, s, h, 1)
            j = np.arange(len(there))
            see = there & (j <= pos[:, None])
            if window:
                see &= (j > pos[:, None] - window) | (j < sinks)
            any_ = see.any(0)
            k, v = np.where(any_[:, None], k, 0).astype(F64), np.where(any_[:, None], v, 0).astype(F64)
            for g in range(h * G, (h + 1) * G):
                z = np.where(see, q[:, g] @ k.T * scale, -np.inf)
                top = z.max(1, keepdims=True)
                p = np.exp(z - np.where(np.isinf(top), 0, top))
                l = np.where(see.any(1), p.sum(1), 1)
                at = slice(r0, r0 + len(pos))
                o[at, g], a[at, g] = (p @ v) / l[:, None], (p @ np.abs(v)) / l[:, None]
                mass[at, g, 0] = np.where(see, scale * (np.abs(q[:, g]) @ np.abs(k).T), 0).max(1)
                mass[at, g, 1] = np.where(see, scale * np.abs(q[:, g]).max(1, keepdims=True) * np.abs(k).sum(1), 0).max(1)
                unit[at, g] = np.abs(v).max() / l
                seen_n[at, g] = see.sum(1)
    return o, a, mass, unit, seen_n
