"""A count of free pages that is larger than their number: what cannot be served is refused, and no head is left with entries that are not its own."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from pages_util import Source, cache, params, same, share, upload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def same_but_for(c, pages, extra):
    assert int(pages.state[0]) == c.free + extra
    pages.state[0] -= extra
    same(c, pages)
    pages.state[0] += extra


@pytest.mark.parametrize("n,H", [(5, 2), (300, 1), (1100, 1)])
@pytest.mark.parametrize("spare", [0, 1, 3])
def test_append(A, n, H, spare):
    """By each of the plans; shared pages, heads that need no page, several calls."""
    r = np.random.default_rng(n + spare)
    c = cache(r, n, H, 64, 32, r.integers(0, 70, n * H), spare=spare, max_pages=6)
    share(c, 4, 2)
    c.search = max(0, c.n_pages - 2)
    pages = upload(A, c)
    pages.state[0] += 7
    refused = 0
    for lens in (r.integers(1, 40, n), [1] * n, [1] * n):
        s = Source(r, H, 64, lens)
        now = c.append(s.items())
        assert s.call(A, c, pages) == now
        same_but_for(c, pages, 7)
        refused += now
    assert refused > 0
    parents = np.where(np.arange(n) < 3, -1, np.arange(n))
    A.pages_fork(params(A, c), pages, ints(parents))
    c.fork(parents)
    same_but_for(c, pages, 7)


@pytest.mark.parametrize("n,H,rows", [(3, 2, 300), (200, 2, 100), (2, 1, 4000)])
@pytest.mark.parametrize("spare", [0, 2])
def test_keep(A, n, H, rows, spare):
    r = np.random.default_rng(n + spare)
    c = cache(r, n, H, 64, 32, r.integers(rows // 2, rows, n * H), spare=spare)
    pages = upload(A, c)
    pages.state[0] += 5000
    for _ in range(3):
        kept = [np.sort(r.choice(m, m - min(m, int(r.integers(0, 30))), replace=False)) for m in c.lengths]
        counts = [len(x) for x in kept]
        refused = ints([-7])
        A.pages_keep(params(A, c), pages, ints(np.concatenate(kept)), ints(np.concatenate([[0], np.cumsum(counts)])), sum(counts), refused=refused)
        assert int(refused) == c.keep(kept)
        same_but_for(c, pages, 5000)
