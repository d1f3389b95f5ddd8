"""pages_attend where V is as large as bf16 holds: the mean of finite values is finite, however its sums are formed."""
import numpy as np
import pytest
import torch

from pages_compare import PATHS, compare, on_path
from pages_util import bf16, params, upload, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def scales(c, of_k, of_v):
    """All scale bytes of K and of V, by functions of a shape."""
    P, d = c.P, c.d
    a, b, e = P * d, P * d + P * d // 32, P * d + P * d // 16
    c.pool[:, a:b] = of_k((c.n_pages, b - a))
    c.pool[:, b:e] = of_v((c.n_pages, e - b))


def attend(A, c, G, q):
    qt, lse = bf16(q).cuda(), torch.full(q.shape[:2], 77.0, device="cuda")
    out = A.pages_attend(params(A, c, G), upload(A, c), qt, lse=lse)
    return values(qt), values(out), values(lse)


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d,G", [(64, 7), (64, 16), (128, 1), (128, 9), (256, 8), (256, 12)])
def test_values_up_to_the_largest(A, path, d, G):
    """Scales of V over all of their range, logits over tens of octaves, so that weights lie above the running reference."""
    r = np.random.default_rng(d + G)
    lengths = [512, 1, 33, 300, 0, 64, 500] if path == "whole" else [3000, 1, 33, 2900, 0, 64, 1500]
    c = on_path(r, path, d, 64, lengths)
    scales(c, lambda s: np.full(s, 120), lambda s: np.where(r.random(s) < 0.5, r.integers(240, 253, s), r.integers(2, 253, s)))
    q, out, lse = attend(A, c, G, r.standard_normal((c.n_seqs, G, d)) * 2.0 ** 7)
    compare(c, q, d ** -0.5, out, lse, large=True)
    assert np.isfinite(out).all()


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_the_mean_of_equal_values_is_their_value(A, path, d):
    """6 * 2^125 in every channel of every row: sums of few terms of it are beyond fp32's numbers. Weights equal, and unequal."""
    r = np.random.default_rng(d)
    c = on_path(r, path, d, 32, [512, 40, 32, 7] if path == "whole" else [3000, 40, 32, 7])
    c.pool[:, c.P * d // 2:c.P * d] = 0x77
    scales(c, lambda s: np.full(s, 120), lambda s: np.full(s, 252))
    for q_scale in (2.0 ** -30, 2.0 ** 6):
        _, out, lse = attend(A, c, 4, r.standard_normal((c.n_seqs, 4, d)) * q_scale)
        there = c.lengths > 0
        assert (out[there] == 6 * 2.0 ** 125).all() and not out[~there].any() and np.isfinite(lse[there]).all()


def test_large_values_of_little_weight(A):
    """Rows with huge V far below the largest logit: they change nothing that fp32 could show, wherever in the head they are."""
    r = np.random.default_rng(3)
    for path in ("whole", "aligned"):
        c = on_path(r, path, 128, 32, [512] if path == "whole" else [3008])
        d, P = 128, 32
        scales(c, lambda s: np.full(s, 120), lambda s: np.full(s, 127))
        c.pool[:, :P * d // 2] = 0x22                                       # keys of 1, but every fifth page's rows are -1 with huge V
        at = c.table[0, :c.lengths[0] // P][2::5]
        c.pool[at, :P * d // 2] = 0xaa
        c.pool[at, P * d + P * d // 32:] = 252
        q, out, lse = attend(A, c, 4, np.full((1, 4, d), 2.0 ** 11))        # logits 181 2^4 / 2 to either side: weights of 2^-4178
        k, v = c.rows(0)
        near = (k > 0).all(1)
        assert np.allclose(out[0], v[near].mean(0), rtol=2.0 ** -7, atol=2.0 ** -12) and np.isfinite(lse).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_one_row_is_its_values(A, d):
    """Of all sizes at once, the smallest beside the largest: a single weight is one."""
    r = np.random.default_rng(d)
    for path in PATHS:
        c = on_path(r, path, d, 32, [1] * 7)
        scales(c, lambda s: np.full(s, 120), lambda s: r.integers(2, 253, s))
        q, out, lse = attend(A, c, 2, r.standard_normal((c.n_seqs, 2, d)))
        for x in range(7):
            assert np.array_equal(out[x], np.repeat(c.rows(x)[1], 2, 0))
