"""Pins of the oracle of the cache in 4 bits and in pages: the format by brute force and by hand, pages and counts by their invariants
and by hand, attention against a softmax written out. CPU only."""
import math

import numpy as np
import pytest

from oracle import pages_oracle as O


def bf16_values():
    bits = np.arange(1 << 16, dtype=np.uint32) << 16
    x = bits.view(np.float32)
    return x[np.isfinite(x)].astype(np.float64)


def test_the_scale_is_the_smallest_that_reaches():
    for x in np.random.default_rng(0).choice(bf16_values(), 400):
        block = np.zeros(32)
        block[5] = x
        e = O.scale_byte(block)
        assert 2 <= e <= 252
        assert abs(x) <= 7 * 2.0 ** (e - 127) or e == 252
        assert e == 2 or abs(x) > 7 * 2.0 ** (e - 128)
        if x != 0:
            assert e == O._scale_fast(abs(x))


@pytest.mark.parametrize("top,e", [(7.0, 127), (7.03125, 128), (3.5, 126), (3.515625, 127), (1.0, 125), (0.0, 2), (2.0 ** -126, 2),
                                   (2.0 ** 127, 252), (math.inf, 255), (math.nan, 255)])
def test_scales_by_hand(top, e):
    assert O.scale_byte(np.array([0.0] * 31 + [top])) == e
    assert O.encode(np.array([[0.0] * 31 + [top]]))[1][0, 0] == e


@pytest.mark.parametrize("y,magnitude", [(0.25, 0), (0.2501, 0.5), (0.75, 1), (0.7499, 0.5), (1.25, 1), (1.75, 2), (2.5, 2), (2.51, 3),
                                         (3.5, 4), (3.49, 3), (5, 4), (5.01, 6), (7, 6), (100, 6)])
def test_codes_by_hand(y, magnitude):
    assert O.MAGNITUDES[O.code_of(y)] == magnitude
    assert O.code_of(-y) == O.code_of(y) + 8


def test_ties_of_rows_are_those_of_single_values():
    x = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, 6.5, 0.1, 0, 1, 2, 3, 4, 6])
    row = np.concatenate([x, -x, x / 8, -x / 4 * 1.5])
    codes, es = O.encode(row[None])
    c, e = O.encode_block(row[:32])
    assert es[0].tolist() == [127, O.scale_byte(row[32:])] and e == 127
    assert c.tolist() == [O.code_of(v) for v in row[:32]] and np.array_equal(codes[0, :16], c[::2] | c[1::2] << 4)


def test_what_is_held_is_the_nearest_that_can_be():
    """Against all 15 values that a block's scale allows; and twice through the format is once."""
    r = np.random.default_rng(1)
    x = r.standard_normal((40, 64)) * np.exp(3 * r.standard_normal((40, 1)))
    codes, es = O.encode(x)
    held = O.decode(codes, es)
    for i in range(40):
        for b in range(2):
            s = 2.0 ** (int(es[i, b]) - 127)
            allowed = np.concatenate([O.MAGNITUDES, -O.MAGNITUDES]) * s
            block = slice(b * 32, b * 32 + 32)
            nearest = np.abs(x[i, block, None] - allowed).min(-1)
            assert np.array_equal(np.abs(x[i, block] - held[i, block]), nearest)
            c, e = O.encode_block(x[i, block])
            assert e == es[i, b] and np.array_equal(c[::2] | c[1::2] << 4, codes[i, b * 16:b * 16 + 16])
    assert np.array_equal(O.decode(*O.encode(held)), held)


def test_a_block_that_is_not_finite_stands_for_nan():
    x = np.ones((2, 64))
    x[0, 3], x[1, 40] = math.inf, math.nan
    codes, es = O.encode(x)
    held = O.decode(codes, es)
    assert np.isnan(held[0, :32]).all() and np.isnan(held[1, 32:]).all()
    assert np.array_equal(held[0, 32:], np.ones(32)) and np.array_equal(held[1, :32], np.ones(32))
    assert not codes[0, :16].any()


def rows(r, n, d):
    return r.standard_normal((n, d)), r.standard_normal((n, d))


def sound(c):
    """Counts are those of the tables, and no page is at two places of a head."""
    count = np.zeros(c.n_pages, dtype=int)
    for g in range(c.n_seqs * c.H):
        mine = c.table[g, :O.pages_of(int(c.lengths[g]), c.P)]
        assert len(set(mine)) == len(mine)
        np.add.at(count, mine, 1)
    assert np.array_equal(count, c.refs) and c.free == (count == 0).sum()


def test_pages_and_counts_hold_together():
    r = np.random.default_rng(2)
    c = O.Cache(4, 2, 64, 30, 6, 32)
    held = {}
    for _ in range(60):
        do = r.integers(4)
        if do == 0:
            n = int(r.integers(0, 50))
            added = [[rows(r, n + int(r.integers(3)), 64) for _ in range(2)] for _ in range(2)]
            before = c.lengths.copy()
            refused = c.append(added, r.permutation(4)[:2])
            assert refused == 0 or (c.lengths == before).sum() >= refused
        elif do == 1:
            parents = r.integers(-1, 4, 4)
            c.fork(parents)
        elif do == 2:
            c.fork(None, r.integers(0, 9, 4))
        else:
            c.keep([np.sort(r.choice(n, int(r.integers(0, n + 1)), replace=False)) if n else [] for n in c.lengths])
        sound(c)
    assert not held


def test_a_fork_keeps_its_rows_when_either_side_grows():
    r = np.random.default_rng(3)
    c = O.Cache(2, 1, 64, 8, 4, 32)
    c.append([[rows(r, 40, 64)]], [0])
    c.fork([0, 0])
    assert c.free == 6 and c.refs.max() == 2
    before = c.rows(0)
    c.append([[rows(r, 1, 64)], [rows(r, 1, 64)]])
    sound(c)
    assert c.free == 5                                   # one whole page in common, a copy each; the begun page is free again
    for g in range(2):
        assert all(np.array_equal(a[:40], b) for a, b in zip(c.rows(g), before))
    assert not np.array_equal(c.rows(0)[0][40], c.rows(1)[0][40])


def test_keep_by_hand():
    r = np.random.default_rng(4)
    c = O.Cache(1, 1, 64, 9, 5, 32)
    c.append([[rows(r, 130, 64)]])
    k, v = c.rows(0)
    first = c.table[0, 0]
    index = list(range(32)) + [33, 40, 129]
    assert c.keep([index]) == 0
    sound(c)
    assert c.table[0, 0] == first and c.table[0, 1] == 5 and c.free == 7 and c.search == 6
    assert np.array_equal(c.rows(0)[0], k[index]) and np.array_equal(c.rows(0)[1], v[index])
    assert c.keep([list(range(40))]) == 0 and c.lengths[0] == 35


def test_kept_rows_are_those_that_were_asked_for():
    r = np.random.default_rng(8)
    c = O.Cache(1, 2, 64, 30, 6, 32)
    c.append([[rows(r, 130, 64), rows(r, 101, 64)]])
    before = [c.rows(0), c.rows(1)]
    index = [np.sort(r.choice(130, 97, replace=False)), np.arange(64)]
    assert c.keep(index) == 0
    sound(c)
    for g in range(2):
        assert all(np.array_equal(a, b[index[g]]) for a, b in zip(c.rows(g), before[g]))


def test_what_there_are_no_pages_for():
    r = np.random.default_rng(5)
    c = O.Cache(3, 1, 64, 4, 3, 32)
    assert c.append([[rows(r, 97, 64)]], [0]) == 1 and c.lengths[0] == 0            # more than its table row has
    assert c.append([[rows(r, 64, 64)], [rows(r, 96, 64)], [rows(r, 32, 64)]]) == 2  # two pages; five in all; six
    assert list(c.lengths) == [64, 0, 0] and c.free == 2
    assert c.append([[rows(r, 5, 64)], [rows(r, 5, 64)], [rows(r, 5, 64)]], [1, 1, 7]) == 0      # twice the same, and none
    assert list(c.lengths) == [64, 5, 0]


def test_a_copy_needs_a_page():
    r = np.random.default_rng(7)
    c = O.Cache(2, 1, 64, 2, 3, 32)
    c.append([[rows(r, 40, 64)]])
    c.fork([0, 0])
    assert c.append([[rows(r, 1, 64)]], [1]) == 1 and list(c.lengths) == [40, 40] and c.free == 0
    c.fork([0, -1])
    assert c.append([[rows(r, 1, 64)]], [0]) == 0 and c.lengths[0] == 41          # not shared any more


def test_attention_written_out():
    r = np.random.default_rng(6)
    c = O.Cache(2, 2, 64, 20, 4, 32)
    c.append([[rows(r, n, 64) for n in (33, 1)], [rows(r, n, 64) for n in (0, 60)]])
    q = r.standard_normal((2, 4, 64))
    out, lse = c.attend(q, 0.125)
    assert not out[1, :2].any() and (lse[1, :2] == -math.inf).all()
    k, v = c.rows(0)
    w = [math.exp(0.125 * float(k[t] @ q[0, 1])) for t in range(33)]
    assert math.isclose(lse[0, 1], math.log(sum(w)), rel_tol=1e-12)
    assert np.allclose(out[0, 1], sum(w[t] * v[t] for t in range(33)) / sum(w), rtol=1e-12)
    assert np.allclose(out[0, 2], c.rows(1)[1][0])       # one row: that row
    a, b = c.read([30, 0, 0, 2], [5, 1, 2, 1])
    assert np.array_equal(a[:3], k[30:]) and not a[3:5].any() and not a[6:8].any() and np.array_equal(b[8], c.rows(3)[1][2])
