"""pages_attend by every way of cutting the work: what special values, pages that are none and moving references do to heads that several
workgroups share, whose parts go through the workspace and are joined there."""
import numpy as np
import pytest
import torch

from pages_compare import PATHS, compare, on_path, rows_of
from pages_util import bf16, params, upload, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def attend(A, c, G, q, large_pool=False):
    pages = upload(A, c)
    if large_pool:                                              # one that the memory-side cache does not hold: rows are streamed
        n = (300 << 20) // c.page_bytes
        pool = torch.zeros(n * c.page_bytes, dtype=torch.uint8, device="cuda")
        pool[:pages.pool.numel()] = pages.pool
        pages.pool, pages.refs = pool, torch.cat((pages.refs, torch.zeros(n - c.n_pages, dtype=torch.int32, device="cuda")))
    qt, lse = bf16(q).cuda(), torch.full(q.shape[:2], 77.0, device="cuda")
    out = A.pages_attend(params(A, c, G), pages, qt, out=torch.full_like(qt, 77.0), lse=lse)
    return values(qt), values(out), values(lse)


def noise_behind_the_last_rows(c):
    """Scales there that say NaN."""
    P, d = c.P, c.d
    for g, n in enumerate(c.lengths):
        if n % P:
            for section in (P * d, P * d + P * d // 32):
                c.pool[c.table[g, n // P], section + n % P * (d // 32):section + P * (d // 32)] = 255


@pytest.mark.parametrize("path,large_pool", [(path, large) for path in PATHS for large in (False, True) if not (large and path == "whole")])
@pytest.mark.parametrize("d,G", [(64, 4), (64, 16), (128, 1), (128, 12), (256, 8), (256, 9)])
def test_special_values(A, path, d, G, large_pool):
    """A scale that says NaN, in K and in V; pages that are none, some and all; keys that rise by many octaves, and fall; queries with NaN and with
    an infinity; heads without rows; ordinary heads beside them."""
    r = np.random.default_rng(d + G)
    P = 64
    lengths = [500, 500, 512, 510, 512, 400, 333, 500, 1, 0] if path == "whole" else [2900, 2950, 3000, 2901, 3136, 2000, 1500, 2600, 1, 0]
    c = on_path(r, path, d, P, lengths)
    noise_behind_the_last_rows(c)
    pages = [n // P for n in lengths]
    c.pool[c.table[0, pages[0] // 2], P * d + 17 * (d // 32) + 1] = 255                          # K of a row in the middle
    c.pool[c.table[1, pages[1] // 2], P * d + P * d // 32 + 17 * (d // 32)] = 255                # V of one: channels 0 to 31
    c.table[2, [0, 2, pages[2] // 2, pages[2] - 1]] = -1, c.n_pages, 2**31 - 1, -2**31
    for g in (3, 4):                                                                             # keys over 16 octaves, up and down
        up = np.arange(pages[g]) * 16 // pages[g]
        for j in range(pages[g]):
            c.pool[c.table[g, j], P * d:P * d + P * d // 32] = 114 + (up[j] if g == 3 else up[-1] - up[j])
    c.table[5, :pages[5] + 1] = -1
    q = r.standard_normal((c.n_seqs, G, d)) * 2.0 ** -5
    q[6, G - 1, 5], q[7, 0, 7] = np.nan, np.inf
    q, out, lse = attend(A, c, G, q, large_pool)
    compare(c, q, d ** -0.5, out, lse)
    assert np.isnan(out[0]).all() and np.isnan(out[1, :, :32]).all() and np.isfinite(out[1, :, 32:]).all() and np.isfinite(lse[1]).all()
    assert not out[5].any() and np.isnan(out[6, G - 1]).all() and np.isnan(out[7, 0]).all() and np.isfinite(out[8:]).all()


@pytest.mark.parametrize("path", PATHS)
@pytest.mark.parametrize("d,G", [(64, 9), (128, 4), (256, 2)])
def test_logits_of_minus_infinity(A, path, d, G):
    """Products that overflow: all of a head's, all but a few rows' far apart, those of whole parts of it; and of one query of a group only."""
    r = np.random.default_rng(d)
    P = 64
    n = 512 if path == "whole" else 3008
    c = on_path(r, path, d, P, [n, n, n, n, 70])
    c.pool[:, :P * d // 2] = 0x66                                              # 4 in every channel
    c.pool[:, P * d:P * d + P * d // 32] = 200
    left = {1: [n // 3, n - 70], 2: list(range(n // 2 // 32 * 32, n // 2 // 32 * 32 + 32)), 3: [0], 4: [69]}
    for g, rows in left.items():
        for t in rows:
            c.pool[c.table[g, t // P], P * d + t % P * (d // 32):P * d + (t % P + 1) * (d // 32)] = 127
    q = np.full((c.n_seqs, G, d), -2.0 ** 60)
    q[3, 1:] = -2.0 ** -80                                                     # (their logits are finite: 2^-5 and nothing)
    q[5:] = 0
    _, out, lse = attend(A, c, G, q)
    assert not out[0].any() and (lse[0] == -np.inf).all()
    for g, rows in left.items():
        v = rows_of(c, g)[1][rows]
        mine = out[g, :1] if g == 3 else out[g]
        assert (np.abs(mine - v.mean(0)) <= 2.0 ** -8 * np.abs(v.mean(0)) + 2.0 ** -15 * np.abs(v).mean(0)).all(), g
        assert np.isfinite(lse[g]).all()
    assert np.isfinite(out).all()
    compare(c, q, d ** -0.5, out, lse, heads=range(5, c.n_seqs))


@pytest.mark.parametrize("path", PATHS[1:])
def test_lengths_that_fill_parts_to_the_row(A, path):
    """Parts of one row, of whole units, of a row less and a row more."""
    r = np.random.default_rng(5)
    c = on_path(r, path, 128, 32, [32 * 4 * 20, 32 * 4 * 20 - 1, 32 * 4 * 20 + 1, 32 * 4, 32 * 4 + 1, 31, 33, 2049])
    q, out, lse = attend(A, c, 7, r.standard_normal((c.n_seqs, 7, 128)) * 2.0 ** -4)
    compare(c, q, 128 ** -0.5, out, lse)
