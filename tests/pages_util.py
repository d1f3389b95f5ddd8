"""What the tests of the cache in pages share: a random cache, the same on both sides, and the comparison of all of it."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import pages_oracle as O


def bf16(x) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def values(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().double().numpy()


def cache(rng, n_seqs, H, d, P, lengths, *, spare=4, max_pages=None, n_pages=None, scales=(110, 140), highest=False) -> O.Cache:
    """A cache whose heads have random rows in random pages (`highest`: the last ones of the pool); what no head has is noise, too."""
    lengths = np.resize(np.array(lengths, dtype=np.int32), n_seqs * H)
    used = sum(O.pages_of(int(n), P) for n in lengths)
    n_pages = n_pages or used + spare
    c = O.Cache(n_seqs, H, d, 1, max_pages or max(1, O.pages_of(int(lengths.max(initial=0)), P)) + 2, P)
    c.n_pages, c.refs = n_pages, np.zeros(n_pages, dtype=np.int32)
    c.pool = rng.integers(0, 256, (n_pages, c.page_bytes), dtype=np.uint8)
    c.pool[:, P * d:] = rng.integers(*scales, (n_pages, P * d // 16), dtype=np.uint8)
    order = n_pages - 1 - np.arange(used) if highest else rng.permutation(n_pages)[:used]
    at = 0
    c.table[:] = rng.integers(-5, n_pages + 5, c.table.shape)
    for g, n in enumerate(lengths):
        k = O.pages_of(int(n), P)
        c.table[g, :k] = order[at:at + k]
        at += k
    c.lengths = lengths.copy()
    c.refs[order] = 1
    c.free, c.search = n_pages - used, int(rng.integers(n_pages))
    return c


def share(c: O.Cache, x: int, parent: int):
    """Sequence x (without rows so far) has the pages of another."""
    parents = list(range(c.n_seqs))
    parents[x] = parent
    c.fork(parents)


def params(A, c: O.Cache, G=2, **more):
    return A.Params(c.H * G, c.H, c.d, 0, **more)


def upload(A, c: O.Cache):
    def dev(x, dtype=np.int32):
        return torch.from_numpy(np.ascontiguousarray(x, dtype=dtype)).cuda()
    return A.Pages(dev(c.pool, np.uint8).view(-1), dev(c.table), dev(c.lengths), dev(c.refs), dev(c.state()), c.P)


def same(c: O.Cache, pages, pool=True):
    """Table, lengths, counts, state and the pool, byte for byte."""
    torch.cuda.synchronize()
    for name, mine in (("lengths", c.lengths), ("refs", c.refs), ("state", c.state())):
        assert np.array_equal(getattr(pages, name).cpu().numpy(), mine), name
    table = pages.table.cpu().numpy()
    for g, n in enumerate(c.lengths):
        k = O.pages_of(int(n), c.P)
        assert np.array_equal(table[g, :k], c.table[g, :k]), g
    if pool:
        got = pages.pool.cpu().numpy().reshape(c.pool.shape)
        assert np.array_equal(got, c.pool), np.argwhere((got != c.pool).any(1))[:5]


class Source:
    """K and V of items as the library takes them: lengths, a layout, rows that each head takes (None: all)."""

    def __init__(self, rng, H, d, lens, kept=None, layout="head", scale=1.0):
        self.H, self.d, self.lens, self.layout = H, d, list(lens), layout
        self.k = [values(bf16(rng.standard_normal((H, L, d)) * scale * np.exp(rng.standard_normal((H, L, 1))))) for L in lens]
        self.v = [values(bf16(rng.standard_normal((H, L, d)) * scale)) for L in lens]
        self.index = None
        if kept is not None:
            self.index = [np.sort(rng.choice(L, min(n, L), replace=False)) for L, n in
                          zip(np.repeat(lens, H), np.resize(np.array(kept), len(lens) * H))]

    def items(self):
        def take(x, i, h):
            return x[i][h] if self.index is None else x[i][h][self.index[i * self.H + h]]
        return [[(take(self.k, i, h), take(self.v, i, h)) for h in range(self.H)] for i in range(len(self.lens))]

    def lay(self, blocks):
        H, d = self.H, self.d
        if self.layout == "strided":
            T = max(self.lens) + 2
            big = np.full((len(blocks), H, T, d + 8), np.nan)
            for i, b in enumerate(blocks):
                big[i, :, :b.shape[1], :d] = b
            return bf16(big).cuda()
        return bf16(np.concatenate([(b if self.layout == "head" else b.transpose(1, 0, 2)).reshape(-1) for b in blocks])).cuda()

    def params(self):
        if self.layout == "strided":
            T, row = max(self.lens) + 2, self.d + 8
            return dict(kv_stride_item=self.H * T * row, kv_stride_head=T * row, kv_stride_tok=row)
        return dict(kv_layout=1 if self.layout == "token" else 0)

    def call(self, A, c, pages, seqs=None, **more):
        """pages_append on the device; the number of heads refused."""
        def dev(x):
            return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
        given = {}
        if self.index is not None:
            given = dict(indices=dev(np.concatenate(self.index)), cu_budgets=dev(np.concatenate([[0], np.cumsum([len(x) for x in self.index])])),
                         total_rows=sum(len(x) for x in self.index))
        refused = torch.full((1,), -7, dtype=torch.int32, device="cuda")
        A.pages_append(params(A, c, **self.params()), pages, self.lay(self.k), self.lay(self.v), self.lens,
                       seqs=None if seqs is None else dev(seqs), refused=refused, **given, **more)
        return int(refused)


def attend_error(c: O.Cache, q, scale, out, lse=None):
    """Nothing is off by more than arithmetic in 32 bits allows. For a query whose logits z_t = scale q.k_t are sums of d products in
    fp32, each is off by at most dz = (d + 4) 2^-24 scale sum |q k| (the products of bf16 numbers are exact, their sum and the scaling
    round d + 1 times, exp2's argument and result about as much again); a weight so by dz + 2^-21 of itself, and for its product with V
    by 2^-16; sums of n terms by n 2^-24; and the output is rounded to bf16, 2^-8 of itself. A weight below fp32's normal numbers,
    2^-126 of the largest, may be zero: n of them take 2^-126 |v| each."""
    ref, ref_lse = c.attend(q, scale)
    G = q.shape[1] // c.H
    for x in range(c.n_seqs):
        for h in range(c.H):
            k, v = c.rows(x * c.H + h)
            n = len(k)
            for j in range(h * G, (h + 1) * G):
                if n == 0 or not np.isfinite(ref_lse[x, j]):
                    assert np.array_equal(out[x, j], ref[x, j], equal_nan=True), (x, j)
                    assert lse is None or np.array_equal(lse[x, j], ref_lse[x, j], equal_nan=True), (x, j)
                    continue
                dz = (c.d + 4) * 2.0 ** -24 * scale * (np.abs(k) @ np.abs(q[x, j])).max()
                w = np.exp(k @ q[x, j] * scale - ref_lse[x, j])
                spread = w @ np.abs(v)
                tol = 2.0 ** -8 * np.abs(ref[x, j]) + (1 + 2.0 ** -8) * spread * (2 * dz + 2.0 ** -15 + 2 * n * 2.0 ** -24 + 2.0 ** -20) + n * 2.0 ** -126 * np.abs(v).max()
                off = np.abs(out[x, j] - ref[x, j])
                assert (off <= tol).all(), (x, j, (off / tol).max())
                if lse is not None:
                    assert abs(lse[x, j] - ref_lse[x, j]) <= dz + n * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -22 * abs(ref_lse[x, j]), (x, j)
    return math.nan
