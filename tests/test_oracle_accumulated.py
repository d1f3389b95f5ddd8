"""Pins for the oracle's accumulated weights and the eviction by them: brute force, closed forms, invariants."""
import math

import numpy as np
import pytest

from oracle import audiokv_oracle as O


def test_accumulate_brute_force():
    rng = np.random.default_rng(0)
    for H_q, H_kv, Q, L, causal in [(4, 2, 5, 9, True), (3, 1, 7, 7, True), (2, 2, 1, 6, True), (4, 2, 4, 6, False)]:
        q, k = rng.normal(size=(H_q, Q, 3)), rng.normal(size=(H_kv, L, 3))
        ref = np.zeros((H_kv, L))
        for j in range(H_q):
            for r in range(Q):
                seen = [t for t in range(L) if not causal or t <= L - Q + r]
                w = [math.exp(0.7 * sum(q[j][r][c] * k[j * H_kv // H_q][t][c] for c in range(3))) for t in seen]
                for t, x in zip(seen, w):
                    ref[j * H_kv // H_q][t] += x / sum(w)
        np.testing.assert_allclose(O.accumulate(q, k, causal=causal, scale=0.7), ref, rtol=1e-12)


def test_accumulate_closed_forms():
    rng = np.random.default_rng(1)
    q, k = rng.normal(size=(6, 8, 4)), rng.normal(size=(2, 11, 4))
    got = O.accumulate(q, k)
    np.testing.assert_allclose(got.sum(1), 3 * 8)                            # every query gives one in all
    # the last W queries alone are the window score before pooling
    np.testing.assert_allclose(O.accumulate(q[:, -5:], k), O.score(q[:, -5:], k, pool_kernel=1), rtol=1e-12)
    # two chunks add up to the whole: the first sees the tokens up to its last query
    first = O.accumulate(q[:, :3], k[:, :6])
    second = O.accumulate(q[:, 3:], k)
    second[:, :6] += first
    np.testing.assert_allclose(second, got, rtol=1e-12)
    # queries of zero: query r spreads evenly over the L - Q + r + 1 tokens that it sees
    zero = O.accumulate(np.zeros((1, 4, 4)), k[:1])
    np.testing.assert_allclose(zero[0], [sum(1 / (8 + r) for r in range(4) if t <= 7 + r) for t in range(11)])
    # tokens at -inf get nothing; a query that sees nothing else gives nothing
    k1 = np.ones((1, 3, 1))
    k1[0, 0] = -np.inf
    np.testing.assert_allclose(O.accumulate(np.ones((1, 3, 1)), k1), [[0, 1.5, 0.5]])


def test_decode_weights_is_decode_attend():
    rng = np.random.default_rng(2)
    q, rows = rng.normal(size=(6, 4)), [rng.normal(size=(n, 4)) for n in (3, 7)]
    out, w = O.decode_weights(q, rows, rows)
    np.testing.assert_allclose(out, O.decode_attend(q, rows, rows), rtol=1e-14)
    for h in range(2):
        np.testing.assert_allclose(w[h].sum(), 3)
        np.testing.assert_allclose(w[h], O.accumulate(q[3 * h:3 * h + 3, None], rows[h][None])[0], rtol=1e-12)
    out, w = O.decode_weights(q, [np.zeros((0, 4)), rows[1]], [np.zeros((0, 4)), rows[1]])
    assert not out[:3].any() and out[3:].all() and len(w[0]) == 0


@pytest.mark.parametrize("weights,positions,budget,recent,src", [
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 3, 0, [0, 4, 2]),             # slot 1 goes, the kept row of slot 4 takes it
    ([5, 1, 4, 2, 3], [0, 1, 2, 3, 4], 3, 2, [0, 3, 4]),             # the two newest stay whatever their weight
    ([1, 1, 1, 1], [0, 1, 2, 3], 2, 0, [0, 1]),                      # equal weights: the lower slots
    ([1, 1, 1, 1], [3, 2, 1, 0], 2, 1, [0, 1]),
    ([1, 9, 9, 9], [9, 2, 1, 0], 2, 1, [0, 1]),                      # slot 0 holds the newest
    ([math.nan, 0, -1, 2], [0, 1, 2, 3], 3, 0, [3, 1, 2]),           # NaN is worth least
    ([1, 2, 3], [0, 1, 2], 5, 1, [0, 1, 2]),                         # nothing to evict
    ([1, 2, 3], [0, 1, 2], 0, 1, []),
    ([1, 2, 3, 4], [7, 8, 9, 10], 2, 4, [0, 1]),                     # more recent rows than room: by slot
    ([0.0, -0.0, 1], [0, 1, 2], 2, 0, [0, 2]),                       # the zeros are equal
])
def test_evict_accumulated_by_hand(weights, positions, budget, recent, src):
    assert O.evict_accumulated(np.array(weights, dtype=float), np.array(positions), budget, recent) == src
