"""fork of tables by two launches, with heads of several hundred entries: more than a wave of 64, more than a workgroup of 256."""
import numpy as np
import pytest
import torch

from pages_util import cache, params, same, upload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("n,H,entries", [(4, 2, 300), (6, 1, 700), (3, 3, 1500), (16, 2, 400)])
def test_long_heads_grow_shrink_and_end(A, n, H, entries):
    """Sequences that take over longer ones, shorter ones, lose most of their rows, and end: lengths, owners and free pages."""
    r = np.random.default_rng(entries)
    long = r.integers(entries * 32 // 2, entries * 32 + 1, n * H)             # every other sequence is, in all of its heads
    c = cache(r, n, H, 64, 32, np.where(np.arange(n * H) // H % 2, r.integers(0, 200, n * H), long), max_pages=entries)
    pages = upload(A, c)
    by_length = np.argsort(c.lengths.reshape(n, H).sum(1), kind="stable")
    shorter, longer = np.empty(n, dtype=np.int64), np.empty(n, dtype=np.int64)
    shorter[by_length], longer[by_length] = np.roll(by_length, 1), np.roll(by_length, -1)
    for parents, drop in ((longer, None), (shorter, None), (np.arange(n), r.integers(0, entries * 32, n)), (r.integers(0, n, n), r.integers(0, 5000, n)),
                          (np.where(np.arange(n) % 2, -1, np.arange(n)), None), (np.zeros(n, dtype=np.int64), None), (np.full(n, -1), None)):
        A.pages_fork(params(A, c), pages, ints(parents), drop=None if drop is None else ints(drop))
        c.fork(parents, drop)
        same(c, pages)
    assert c.free == c.n_pages


@pytest.mark.parametrize("entries", [8, 600])
def test_an_entry_that_is_no_page_is_taken_over(A, entries):
    """-1, and numbers beyond the pool, among a parent's entries: the child's are the same, and not what stood there before."""
    r = np.random.default_rng(entries)
    c = cache(r, 4, 1, 64, 32, [200, 70, 40, 0], max_pages=entries)
    pages = upload(A, c)
    for n in (-1, c.n_pages, 2**31 - 1, -2**31):
        pages.table[0, 3] = n
        A.pages_fork(params(A, c), pages, ints([0, 0, -1, 0]))
        assert pages.table[1, :7].tolist() == pages.table[3, :7].tolist() == pages.table[0, :7].tolist()
        A.pages_fork(params(A, c), pages, ints([0, -1, -1, -1]))
        pages.table[1:, 3] = int(pages.table[0, 0])               # what stands behind a head's rows has no meaning
