"""Attention over a cache in pages against its definition, head by head: rows of pages that are none left out, NaN where the definition
has it, and every path of pages_attend by the sizes that choose it."""
from __future__ import annotations

import math

import numpy as np

from oracle import pages_oracle as O
from pages_util import cache

# Workgroups that attend is cut for, by head_dim. Heads in parts: tables of more than 2048 rows, or more than 512 heads.
WORKGROUPS = {64: 1024, 128: 768, 256: 512}
PATHS = ("whole", "aligned", "even", "even_long", "even_many")


def on_path(rng, path, d, P, lengths, **more) -> O.Cache:
    """A cache of one KV head a sequence whose first heads have `lengths`, with as many others, empty or short, and tables as wide as a path takes:
    a workgroup a head; shares that end with heads; even shares of fewer heads than workgroups (with few rows in all, and with so many that
    the other cut would have been chosen for fewer heads), and of more."""
    w, lengths = WORKGROUPS[d], list(lengths)
    if path == "whole":
        assert max(lengths) <= 512
        return cache(rng, len(lengths), 1, d, P, lengths, max_pages=512 // P, **more)
    n = {"aligned": len(lengths), "even": w * 3 // 4, "even_long": w // 2 - 4, "even_many": w + 100}[path]
    rest = n - len(lengths)
    short = np.where(rng.random(rest) < 0.8, 0, rng.integers(1, 70, rest))
    if path == "even_long":
        # w - n workgroups to share among, more than four units beyond an even share: total / (w - n) - 4 > total / w
        short = rng.integers(32 * 10, 32 * 14, rest)
        total = int(sum(-(-x // 32) for x in [*short, *lengths]))
        assert -(-total // (w - n)) - 4 > total // w
    return cache(rng, n, 1, d, P, [*lengths, *short], max_pages=max(4096, max(lengths) + P) // P, **more)


def rows_of(c: O.Cache, g: int):
    """K and V of a head, without the rows of pages that are none."""
    n, P, d = int(c.lengths[g]), c.P, c.d
    entries = c.table[g, :O.pages_of(n, P)]
    fine = (entries >= 0) & (entries < c.n_pages)
    pages = c.pool[np.where(fine, entries, 0)]
    at = [0, P * d // 2, P * d, P * d + P * d // 32, P * d + P * d // 16]
    there = np.repeat(fine, P)[:n]
    kc, vc, ke, ve = (pages[:, a:b].reshape(len(pages) * P, (b - a) // P)[:n][there] for a, b in zip(at, at[1:]))
    return O.decode(kc, ke), O.decode(vc, ve)


def compare(c: O.Cache, q, scale, out, lse, heads=None, large=False):
    """As pages_util.attend_error, which derives these bounds: dz for a logit, 2^-21 for its exponential, 2^-16 for its product with V, n 2^-24
    for sums of n terms, 2^-8 of the output for its rounding. A weight below fp32's normal numbers may be zero, and so may its product with V, or
    that of what one bf16 number leaves of it: 2^-126 |v| and 2 * 2^-126 for each of n rows. `large`: V's scales reach the largest, 2^125, and
    sums of n terms may be kept from overflowing by a reference that lies up to ceil(log2 n) octaves above the largest logit. What may be zero is
    as much larger then; and the distances of logits from it, and the logarithm of the weights' sum, are numbers of that size: each is rounded by
    2^-24 of it, or the hardware's logarithm by 2^-23, which together is less than octaves 2^-22."""
    G = q.shape[1] // c.H
    for g in range(c.n_seqs * c.H) if heads is None else heads:
        x, h = divmod(g, c.H)
        mine = slice(h * G, (h + 1) * G)
        k, v = rows_of(c, g)
        n = len(k)
        if n == 0:
            assert not out[x, mine].any() and (lse[x, mine] == -np.inf).all(), g
            continue
        octaves = math.ceil(math.log2(n)) if large else 0
        with np.errstate(invalid="ignore", over="ignore"):
            z = q[x, mine] @ k.T * scale
            m = z.max(-1, keepdims=True)
            w = np.exp(z - m)
            den = w.sum(-1, keepdims=True)
            w, ref_lse = w / den, (m + np.log(den))[:, 0]
            ref, spread, most = w @ v, w @ np.abs(v), np.abs(v).max(0)
            dz = (c.d + 4) * 2.0 ** -24 * scale * (np.abs(q[x, mine]) @ np.abs(k).T).max(-1)
            tol = 2.0 ** -8 * np.abs(ref) + (1 + 2.0 ** -8) * spread * (2 * dz + octaves * 2.0 ** -22 + 2.0 ** -15 + 2 * n * 2.0 ** -24 + 2.0 ** -20)[:, None] + n * 2.0 ** (octaves - 126) * (most + 2)
            off = np.abs(out[x, mine] - ref)
            lse_off = np.abs(lse[x, mine] - ref_lse)
        assert np.array_equal(np.isnan(out[x, mine]), np.isnan(ref)), g
        assert (off <= tol)[~np.isnan(ref)].all(), (g, np.nanmax(off / tol))
        assert np.array_equal(np.isnan(lse[x, mine]), np.isnan(ref_lse)), g
        assert (lse_off <= dz + octaves * 2.0 ** -22 + n * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -22 * np.abs(ref_lse))[~np.isnan(ref_lse)].all(), g
