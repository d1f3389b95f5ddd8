"""The cache in 4 bits and in pages, from its definition: numpy, one head, row and page at a time, in float64. Shares no code with
the kernels. The pool is held as bytes, in the layout of audiokv_pages, so that it can be compared with the device's byte for byte.
"""
from __future__ import annotations

import math

import numpy as np

MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def scale_byte(block: np.ndarray) -> int:
    """e of a block of 32 values: the smallest with max|x| <= 7 * 2^(e - 127), within 2 and 252; 255 for an infinity or NaN."""
    top = np.abs(np.asarray(block, dtype=np.float64)).max()
    if not np.isfinite(top):
        return 255
    e = 2
    while e < 252 and top > 7 * math.ldexp(1.0, e - 127):
        e += 1
    return e


def code_of(y: float) -> int:
    """The nearest magnitude's code; in the middle between two the even code; the sign in bit 3."""
    distance = np.abs(MAGNITUDES - abs(y))
    near = np.flatnonzero(distance == distance.min())
    c = int(near[0]) if len(near) == 1 else int(next(i for i in near if i % 2 == 0))
    return c + (8 if math.copysign(1.0, y) < 0 else 0)


def encode_block(block: np.ndarray):
    e = scale_byte(block)
    if e == 255:
        return np.zeros(32, dtype=np.uint8), e
    return np.array([code_of(math.ldexp(float(x), 127 - e)) for x in block], dtype=np.uint8), e


def encode(rows: np.ndarray):
    """[n, d] -> codes [n, d / 2] (the even channel low), e [n, d / 32], bytes. Blocks of the same values are worked out once."""
    n, d = rows.shape
    codes, es = np.zeros((n, d), dtype=np.uint8), np.zeros((n, d // 32), dtype=np.uint8)
    blocks = np.ascontiguousarray(rows, dtype=np.float64).reshape(n, d // 32, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(blocks).max(-1)
    for i in range(n):
        for b in range(d // 32):
            e = es[i, b] = scale_byte(blocks[i, b]) if not np.isfinite(top[i, b]) or top[i, b] == 0 else _scale_fast(top[i, b])
            if e != 255:
                y = np.ldexp(blocks[i, b], 127 - int(e))
                z = np.abs(y)[:, None] - MAGNITUDES
                z = np.abs(z)
                near = z == z.min(-1, keepdims=True)
                first = near.argmax(-1)
                c = np.where((near.sum(-1) == 2) & (first % 2 == 1), first + 1, first)
                codes[i, b * 32:(b + 1) * 32] = c + 8 * np.signbit(y)
    return codes[:, ::2] | codes[:, 1::2] << 4, es


def _scale_fast(top: float) -> int:
    m, e = math.frexp(top / 7)                     # top / 7 = m 2^e: the smallest power of two that is not below it
    k = e - 1 if m == 0.5 else e
    return min(max(k + 127, 2), 252)


def decode(codes: np.ndarray, es: np.ndarray) -> np.ndarray:
    """Bytes as encode gives them -> the values that they stand for."""
    c = np.empty((*codes.shape[:-1], codes.shape[-1] * 2), dtype=np.uint8)
    c[..., ::2], c[..., 1::2] = codes & 15, codes >> 4
    value = np.where(c >= 8, -1.0, 1.0) * MAGNITUDES[c & 7]
    e = np.repeat(es.astype(np.int64), 32, axis=-1)
    return np.where(e == 255, math.nan, np.ldexp(value, e - 127))


def pages_of(rows: int, P: int) -> int:
    return -(-rows // P)


class Cache:
    def __init__(self, n_seqs: int, H: int, d: int, n_pages: int, max_pages: int, P: int, pool=None):
        self.n_seqs, self.H, self.d, self.n_pages, self.max_pages, self.P = n_seqs, H, d, n_pages, max_pages, P
        self.page_bytes = P * d * 17 // 16
        self.pool = np.zeros((n_pages, self.page_bytes), dtype=np.uint8) if pool is None else pool.copy()
        self.table = np.zeros((n_seqs * H, max_pages), dtype=np.int32)
        self.lengths = np.zeros(n_seqs * H, dtype=np.int32)
        self.refs = np.zeros(n_pages, dtype=np.int32)
        self.free, self.search = n_pages, 0

    # -- a row's bytes
    def _row(self, page: int, row: int):
        P, d, b = self.P, self.d, self.pool[page]
        at = [0, P * d // 2, P * d, P * d + P * d // 32]
        size = [d // 2, d // 2, d // 32, d // 32]
        return [b[a + row * n:a + (row + 1) * n] for a, n in zip(at, size)]

    def _copy_row(self, page, row, to_page, to_row):
        for a, b in zip(self._row(page, row), self._row(to_page, to_row)):
            b[:] = a

    def value(self, head: int, row: int):
        kc, vc, ke, ve = self._row(self.table[head, row // self.P], row % self.P)
        return decode(kc, ke), decode(vc, ve)

    # -- pages
    def _plan(self):
        """Free pages as they are taken."""
        return [p for p in ((self.search + i) % self.n_pages for i in range(self.n_pages)) if self.refs[p] == 0]

    def _taken(self, pages):
        if pages:
            self.search = (pages[-1] + 1) % self.n_pages
        for p in pages:
            self.refs[p] += 1

    def _given_back(self, pages):
        for p in pages:
            self.refs[p] -= 1
        self.free = int((self.refs == 0).sum())

    def state(self):
        return np.array([self.free, self.search], dtype=np.int32)

    # -- the operators
    def append(self, items, seqs=None) -> int:
        """items: per item a list over KV heads of (K rows, V rows) [n, d]. Returns the number of heads refused."""
        P, H = self.P, self.H
        plan, taken, back, asked, refused = self._plan(), [], [], 0, 0
        seqs = list(range(len(items))) if seqs is None else list(seqs)
        shared = {p for p in range(self.n_pages) if self.refs[p] > 1}
        for i, heads in enumerate(items):
            x = seqs[i]
            if not 0 <= x < self.n_seqs or x in seqs[:i]:
                continue
            needs = []
            for h, (k, _) in enumerate(heads):
                n, more = int(self.lengths[x * H + h]), len(k)
                copies = more > 0 and n % P != 0 and self.table[x * H + h, n // P] in shared
                needs.append(pages_of(n + more, P) - pages_of(n, P) + copies)
            if any(len(k) and pages_of(int(self.lengths[x * H + h]) + len(k), P) > self.max_pages for h, (k, _) in enumerate(heads)):
                refused += sum(len(k) > 0 for k, _ in heads)
                continue
            asked += sum(needs)
            if sum(needs) > 0 and asked > len(plan):
                refused += sum(len(k) > 0 for k, _ in heads)
                continue
            for h, (k, v) in enumerate(heads):
                g, n = x * H + h, int(self.lengths[x * H + h])
                if len(k) and n % P and self.table[g, n // P] in shared:
                    old, new = int(self.table[g, n // P]), plan[len(taken)]
                    taken.append(new)
                    back.append(old)
                    for r in range(n % P):
                        self._copy_row(old, r, new, r)
                    self.table[g, n // P] = new
                (kc, ke), (vc, ve) = encode(k), encode(v)
                for t in range(len(k)):
                    r = n + t
                    if r % P == 0:
                        self.table[g, r // P] = plan[len(taken)]
                        taken.append(plan[len(taken)])
                    for to, what in zip(self._row(self.table[g, r // P], r % P), (kc[t], vc[t], ke[t], ve[t])):
                        to[:] = what
                self.lengths[g] = n + len(k)
        self._taken(taken)
        self._given_back(back)
        return refused

    def fork(self, parents=None, drop=None):
        P, H = self.P, self.H
        table, lengths = self.table.copy(), self.lengths.copy()
        for x in range(self.n_seqs):
            parent = x if parents is None else int(parents[x])
            for h in range(H):
                g, n = x * H + h, 0
                if 0 <= parent < self.n_seqs:
                    n = max(0, int(lengths[parent * H + h]) - max(0, 0 if drop is None else int(drop[x])))
                for j in range(pages_of(int(lengths[g]), P)):
                    self.refs[table[g, j]] -= 1
                for j in range(pages_of(n, P)):
                    self.table[g, j] = table[parent * H + h, j]
                    self.refs[self.table[g, j]] += 1
                self.lengths[g] = n
        self.free = int((self.refs == 0).sum())

    def keep(self, kept) -> int:
        """kept: the indices of every head, ascending. Returns the number of heads refused."""
        P = self.P
        plan, taken, back, asked, refused = self._plan(), [], [], 0, 0
        for g, index in enumerate(kept):
            n, b = int(self.lengths[g]), len(index)
            if b >= n:
                continue
            same = 0
            while (same + 1) * P <= b and list(index[same * P:(same + 1) * P]) == list(range(same * P, (same + 1) * P)):
                same += 1
            need = pages_of(b, P) - same
            asked += need
            if need > 0 and asked > len(plan):
                refused += 1
                continue
            old = self.table[g].copy()
            new = [plan[len(taken) + j] for j in range(need)]
            taken += new
            for t in range(same * P, b):
                i = min(max(int(index[t]), 0), n - 1)
                self._copy_row(old[i // P], i % P, new[t // P - same], t % P)
            back += [int(p) for p in old[same:pages_of(n, P)]]
            self.table[g, same:same + need] = new
            self.lengths[g] = b
        self._taken(taken)
        self._given_back(back)
        return refused

    def read(self, first, counts):
        """K and V [sum of counts, d]."""
        out = [[], []]
        for g, (f, n) in enumerate(zip(first, counts)):
            for r in range(f, f + n):
                there = 0 <= r < self.lengths[g]
                for which, x in enumerate(self.value(g, r) if there else (np.zeros(self.d),) * 2):
                    out[which].append(x)
        return [np.array(x).reshape(-1, self.d) for x in out]

    def rows(self, g):
        """All rows of a head, K and V."""
        n, P, d = int(self.lengths[g]), self.P, self.d
        pages = self.pool[self.table[g, :pages_of(n, P)]]
        at = [0, P * d // 2, P * d, P * d + P * d // 32, P * d + P * d // 16]
        kc, vc, ke, ve = (pages[:, a:b].reshape(len(pages) * P, (b - a) // P)[:n] for a, b in zip(at, at[1:]))
        return decode(kc, ke), decode(vc, ve)

    def attend(self, q, scale):
        """q [n_seqs, n_q_heads, d] -> output of its shape, log-sum-exp [n_seqs, n_q_heads]."""
        out, lse = np.zeros(q.shape), np.full(q.shape[:2], -math.inf)
        G = q.shape[1] // self.H
        with np.errstate(invalid="ignore", over="ignore"):
            for x in range(self.n_seqs):
                for h in range(self.H):
                    k, v = self.rows(x * self.H + h)
                    if len(k) == 0:
                        continue
                    for j in range(h * G, (h + 1) * G):
                        z = k @ q[x, j] * scale
                        if (z == -math.inf).all():
                            continue
                        m = z.max()
                        p = np.exp(z - m)
                        out[x, j] = p @ v / p.sum()
                        lse[x, j] = m + math.log(p.sum()) if p.sum() > 0 else math.nan
        return out, lse
