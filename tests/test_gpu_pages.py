"""The cache in 4 bits and in pages on the GPU against its oracle: bytes, pages and counts exactly, attention within what arithmetic in
32 bits allows (pages_util.attend_error)."""
import math

import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from pages_util import Source, attend_error, bf16, cache, params, same, share, upload, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def cu(counts):
    return ints(np.concatenate([[0], np.cumsum(counts)]))


# ---- append ----------------------------------------------------------------------------------------------------------------------

def test_every_value_of_bf16_is_rounded_as_the_format_says(A):
    """All finite bit patterns in blocks of neighbours (a block's largest decides its scale), blocks with one large value, and blocks
    with an infinity or NaN."""
    bits = np.arange(1 << 16, dtype=np.uint32)
    finite = bits[(bits & 0x7f80) != 0x7f80]
    r = np.random.default_rng(0)
    x = np.concatenate([finite, r.permutation(finite), r.permutation(bits), (r.integers(0x3e00, 0x4200, 1 << 15) | r.integers(0, 2, 1 << 15) << 15)])
    x = torch.from_numpy(x.astype(np.uint16).view(np.int16)).view(torch.bfloat16)
    x = x[:x.numel() // 128 * 128].view(-1, 128)
    c = O.Cache(1, 1, 128, 2 * len(x) // 64 + 3, 2 * len(x) // 64 + 3, 64)
    pages = upload(A, c)
    L = len(x)
    flipped = x.flip(0)
    A.pages_append(params(A, c), pages, x.cuda(), flipped.cuda(), [L])
    c.append([[(values(x), values(flipped))]])
    same(c, pages)


@pytest.mark.parametrize("layout", ["head", "token", "strided"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("P", [32, 256])
def test_append_layouts(A, d, P, layout):
    r = np.random.default_rng(d + P)
    c = cache(r, 3, 2, d, P, [0, 31, 32, 40, P, 2 * P - 1], spare=12, max_pages=6)
    pages = upload(A, c)
    for kept in (None, [5, 0, 70, 33, 1, 12]):
        s = Source(r, 2, d, [70, 45, 33], kept, layout)
        assert s.call(A, c, pages) == c.append(s.items())
        same(c, pages)


@pytest.mark.parametrize("H,n,lens", [(1, 1, [1]), (4, 5, [1] * 5), (3, 7, [2, 1, 3, 1, 1, 5, 4]), (2, 1, [300]), (5, 300, [1] * 300), (1, 1100, [1] * 1100)])
def test_append_sizes(A, H, n, lens):
    """One row to many heads (more than one workgroup plans at a time), and many to few."""
    r = np.random.default_rng(n)
    c = cache(r, n, H, 64, 32, r.integers(0, 100, n * H), spare=2 * n * H + 20, max_pages=14)
    pages = upload(A, c)
    s = Source(r, H, 64, lens)
    assert s.call(A, c, pages) == c.append(s.items()) == 0
    same(c, pages)


def test_append_to_the_first_sequences_and_of_nothing(A):
    """Fewer items than sequences; budgets of zero, of some heads, of an item, of all."""
    r = np.random.default_rng(21)
    c = cache(r, 5, 2, 64, 32, [3, 64, 31, 0, 20, 90, 32, 1, 64, 7], spare=30, max_pages=9)
    pages = upload(A, c)
    for lens, kept in (([40, 3], None), ([40, 33, 20], [0, 7, 0, 0, 20, 0]), ([5, 9], [0])):
        s = Source(r, 2, 64, lens, kept)
        assert s.call(A, c, pages) == c.append(s.items()) == 0
        same(c, pages)


def test_append_to_given_sequences(A):
    """In any order; a sequence that is none, and one named twice: the first item that does."""
    r = np.random.default_rng(1)
    c = cache(r, 6, 2, 64, 32, [3, 64, 31, 0, 20, 90, 32, 1], spare=30, max_pages=9)
    pages = upload(A, c)
    for seqs in ([5, 0, 3], [2, 2, 2], [-1, 6, 4], [1, 2**31 - 1, 1], [-2**31, 0, 0]):
        s = Source(r, 2, 64, [40, 3, 17])
        assert s.call(A, c, pages, seqs) == c.append(s.items(), seqs) == 0
        same(c, pages)


def test_append_to_a_few_of_many_sequences(A):
    """More sequences than the small plan keeps owners of, and more items than it has threads: the general one, with sequences named
    twice."""
    r = np.random.default_rng(20)
    c = cache(r, 5000, 1, 64, 32, r.integers(0, 70, 5000), spare=2600)
    c.fork(np.where(np.arange(5000) % 7 == 3, np.arange(5000) - 1, np.arange(5000)))
    pages = upload(A, c)
    for seqs in ([4999, 17, 4999, -1], r.integers(-3, 5003, 1300)):
        s = Source(r, 1, 64, r.integers(1, 4, len(seqs)))
        assert s.call(A, c, pages, seqs) == c.append(s.items(), seqs) == 0
        same(c, pages)


def test_more_items_than_sequences(A):
    r = np.random.default_rng(2)
    c = cache(r, 2, 1, 64, 32, [3, 64], spare=9, max_pages=9)
    pages = upload(A, c)
    s = Source(r, 1, 64, [4, 5, 6, 7])
    assert s.call(A, c, pages, [1, -1, 0, 1]) == c.append(s.items(), [1, -1, 0, 1])
    same(c, pages)


def test_append_to_shared_pages(A):
    """Forks of one sequence grow in one call, all, some, by more than a page; whole shared pages stay shared."""
    r = np.random.default_rng(3)
    for P in (32, 64):
        c = cache(r, 4, 2, 128, P, [75, 64], spare=30, max_pages=9)
        c.fork([0, -1, -1, -1])
        for x in (1, 3):
            share(c, x, 0)
        pages = upload(A, c)
        for lens, seqs in (([1, 1], [0, 1]), ([70, 3], [3, 1]), ([1, 1, 1, 1], [0, 1, 2, 3])):
            s = Source(r, 2, 128, lens)
            assert s.call(A, c, pages, seqs) == c.append(s.items(), seqs) == 0
            same(c, pages)


@pytest.mark.parametrize("spare", [0, 1, 2, 3, 5, 6, 40])
def test_append_when_pages_run_out(A, spare):
    r = np.random.default_rng(4)
    c = cache(r, 5, 2, 64, 32, [31, 32, 33, 64, 1, 0, 60, 96, 5, 90], spare=spare, max_pages=5)
    share(c, 4, 2)
    pages = upload(A, c)
    for lens in ([1] * 5, [2, 40, 1, 1, 1], [100, 1, 1, 70, 3], [1] * 5):
        s = Source(r, 2, 64, lens)
        assert s.call(A, c, pages) == c.append(s.items())
        same(c, pages)


def test_append_beyond_a_table_row(A):
    r = np.random.default_rng(5)
    c = cache(r, 3, 2, 64, 32, [60, 10, 64, 64, 0, 5], spare=30, max_pages=2)
    pages = upload(A, c)
    for lens in ([4, 1, 3], [5, 1, 60], [1, 1, 64], [1, 1, 1]):
        s = Source(r, 2, 64, lens)
        assert s.call(A, c, pages) == c.append(s.items())
        same(c, pages)


@pytest.mark.parametrize("d,lens", [(64, [30000, 1, 121222]), (128, [37000, 40001]), (256, [6, 21000, 18000])])
@pytest.mark.parametrize("kept", [False, True])
def test_append_of_many_rows_is_that_of_fewer_at_a_time(A, d, lens, kept):
    """137 MB and more of K and V in one call, and item by item, below the size from which rows pass the caches by."""
    g = torch.Generator(device="cuda").manual_seed(d)
    H, P, ends = 4, 64, np.cumsum([0] + lens)
    k, v = (torch.randn(int(ends[-1]) * H * d, device="cuda", generator=g).bfloat16() for _ in range(2))
    p = A.Params(H, H, d, 0)
    pages = [A.Pages.empty(p, len(lens), sum(-(-n // P) for n in lens) * H, -(-max(lens) // P), P) for _ in range(2)]
    for c in pages:
        c.pool.zero_()
    r = np.random.default_rng(d)
    rows = [[np.sort(r.choice(n, n - n // 9, replace=False)) if kept else np.arange(n) for _ in range(H)] for n in lens]

    def call(c, items):
        part = slice(int(ends[items[0]]) * H * d, int(ends[items[-1] + 1]) * H * d)
        counts = [len(x) for i in items for x in rows[i]]
        more = dict(indices=ints(np.concatenate([x for i in items for x in rows[i]])), cu_budgets=cu(counts), total_rows=sum(counts)) if kept else {}
        A.pages_append(p, c, k[part], v[part], [lens[i] for i in items], seqs=ints(items), **more)
    call(pages[0], list(range(len(lens))))
    for i in range(len(lens)):
        call(pages[1], [i])
    for name in ("pool", "table", "lengths", "refs", "state"):
        assert torch.equal(getattr(pages[0], name), getattr(pages[1], name)), name
    assert pages[0].lengths.tolist() == [len(x) for item in rows for x in item]


def test_append_searches_round_a_large_pool(A):
    """More pages than one round of the search looks at, few of them free, and the search begins near the end."""
    r = np.random.default_rng(6)
    c = cache(r, 2, 1, 64, 32, [32 * 9000, 40], spare=300, max_pages=9400)
    c.search = c.n_pages - 2
    pages = upload(A, c)
    for lens in ([7, 1000], [32 * 200, 5], [3, 3]):
        s = Source(r, 1, 64, lens)
        assert s.call(A, c, pages) == c.append(s.items()) == 0
        same(c, pages)


def test_a_state_that_promises_too_many_pages_writes_nowhere(A):
    """The count of free pages is wrong: rows without a page are lost, nothing else is touched."""
    r = np.random.default_rng(7)
    c = cache(r, 2, 1, 64, 32, [32, 32], spare=0, max_pages=5)
    pages = upload(A, c)
    pages.state[0] = 3
    before = [t.clone() for t in (pages.pool, pages.refs)]
    s = Source(r, 1, 64, [1, 40])
    s.call(A, c, pages)
    assert torch.equal(pages.pool, before[0]) and torch.equal(pages.refs, before[1])
    q = bf16(r.standard_normal((2, 2, 64))).cuda()
    assert torch.isfinite(A.pages_attend(params(A, c), pages, q).float()).all()


# ---- read ------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,P", [(64, 32), (128, 64), (256, 128), (64, 256)])
def test_read(A, d, P):
    r = np.random.default_rng(d)
    c = cache(r, 3, 2, d, P, [0, 1, 300, 70, 64, 33])
    c.pool[:, P * d:] = r.integers(0, 256, (c.n_pages, P * d // 16))           # every scale there is
    pages = upload(A, c)
    for first, counts in ((None, c.lengths), ([0, 0, 290, 3, 64, 40], [3, 1, 40, 20, 0, 5]), ([5, 0, -2, 0, 2**31 - 1, 0], [0, 0, 5, 0, 9, 1])):
        n = int(np.sum(counts))
        k, v = A.pages_read(params(A, c), pages, cu(counts), n, first=None if first is None else ints(first))
        want = c.read([0] * 6 if first is None else first, counts)
        for got, ref in zip((k, v), want):
            ref = np.where(np.abs(ref) >= 2.0 ** 128, np.copysign(math.inf, ref), ref)     # (scales that append does not write)
            got = values(got)
            small = np.abs(ref) < 2.0 ** -126                                             # numbers below the normal ones may be zero
            assert np.array_equal(got[~small], ref[~small], equal_nan=True)
            assert (np.abs(got[small]) <= 2.0 ** -126).all()


@pytest.mark.parametrize("d,rows", [(64, 33000), (128, 17001), (256, 8200)])
def test_read_of_many_rows(A, d, rows):
    r = np.random.default_rng(d)
    lens = [rows // 2, 0, rows - rows // 2 - 777, 777]
    c = cache(r, 2, 2, d, 64, lens)
    k, v = A.pages_read(params(A, c), upload(A, c), cu(lens), rows)
    for got, want in zip((k, v), c.read([0] * 4, lens)):
        assert np.array_equal(values(got), want)


def test_what_is_read_can_be_decoded_and_scored(A):
    """The way back: bf16 rows as compact packs them, for decode_attend and for accumulate."""
    r = np.random.default_rng(8)
    c = cache(r, 2, 2, 128, 64, [90] * 4)
    p, pages = params(A, c, 4), upload(A, c)
    k, v = A.pages_read(p, pages, cu(c.lengths), 360)
    q = bf16(r.standard_normal((2, 8, 128)) * 2.0 ** -7).cuda()
    a = A.decode_attend(p, q, k, v, cu(c.lengths), 2, 360)
    b = A.pages_attend(p, pages, q)
    attend_error(c, values(q), 128 ** -0.5, values(a))
    attend_error(c, values(q), 128 ** -0.5, values(b))
    weights = A.accumulate(p, q.view(-1), k.view(-1), [90, 90], [1, 1])
    assert math.isclose(float(weights.sum()), 16, rel_tol=1e-4)


# ---- fork ------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("seed", range(6))
def test_fork(A, seed):
    r = np.random.default_rng(seed)
    n, H, P = int(r.integers(1, 40)), int(r.integers(1, 4)), int(r.choice([32, 64]))
    c = cache(r, n, H, 64, P, r.integers(0, 400, n * H), spare=5)
    pages = upload(A, c)
    for _ in range(4):
        parents = r.integers(-1, n, n) if r.random() < 0.8 else None
        if parents is not None:
            parents = np.where(r.random(n) < 0.3, np.arange(n), parents)
        drop = r.integers(-2, 90, n) if r.random() < 0.6 else None
        A.pages_fork(params(A, c), pages, None if parents is None else ints(parents), drop=None if drop is None else ints(drop))
        c.fork(parents, drop)
        same(c, pages)


@pytest.mark.parametrize("n,H,entries", [(1, 1, 40), (32, 4, 8), (25, 3, 14), (64, 2, 16), (43, 3, 16), (9, 1, 228)])
def test_fork_of_tables_of(A, n, H, entries):
    r = np.random.default_rng(entries)
    c = cache(r, n, H, 64, 32, r.integers(0, entries * 32 + 1, n * H), max_pages=entries)
    pages = upload(A, c)
    for parents in (r.integers(-1, n, n), r.permutation(n), np.zeros(n, dtype=np.int64)):
        drop = r.integers(0, 50, n)
        A.pages_fork(params(A, c), pages, ints(parents), drop=ints(drop))
        c.fork(parents, drop)
        same(c, pages)


def test_fork_of_nobody_changes_nothing_and_of_none_empties(A):
    r = np.random.default_rng(9)
    c = cache(r, 3, 2, 64, 32, [70, 1, 33, 0, 64, 32])
    pages = upload(A, c)
    A.pages_fork(params(A, c), pages)
    same(c, pages)
    A.pages_fork(params(A, c), pages, ints([0, 1, 2]))
    same(c, pages)
    A.pages_fork(params(A, c), pages, ints([3, -1, 2**31 - 1]), drop=ints([2**31 - 1, -2**31, 0]))
    c.fork([3, -1, 2**31 - 1])
    same(c, pages)
    assert not c.lengths.any() and c.free == c.n_pages


# ---- keep ------------------------------------------------------------------------------------------------------------------------

def keep(A, c, pages, kept, **more):
    refused = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    counts = [len(x) for x in kept]
    n = sum(counts)
    index = ints(np.concatenate([np.asarray(x, dtype=np.int64) for x in kept])) if n else None
    A.pages_keep(params(A, c), pages, index, cu(counts), n, refused=refused, **more)
    assert int(refused) == c.keep(kept)
    same(c, pages)


@pytest.mark.parametrize("d,P", [(64, 32), (128, 64), (256, 32), (128, 256)])
def test_keep(A, d, P):
    r = np.random.default_rng(d + P)
    c = cache(r, 3, 2, d, P, [0, 1, 700, 333, 512, 64], spare=40)
    pages = upload(A, c)
    for share_kept in (0.9, 0.5, 1.0, 0.1, 0.0):
        kept = []
        for n in c.lengths:
            b = int(n * share_kept)
            first = min(b, int(r.integers(0, n + 1)))                        # a beginning that stays
            rest = np.sort(r.choice(np.arange(first, n), b - first, replace=False))
            kept.append(np.concatenate([np.arange(first), rest]))
        keep(A, c, pages, kept)


@pytest.mark.parametrize("spare", [0, 1, 2, 4, 7])
def test_keep_when_pages_run_out(A, spare):
    r = np.random.default_rng(10)
    c = cache(r, 3, 2, 64, 32, [100, 64, 40, 33, 200, 10], spare=spare)
    pages = upload(A, c)
    for _ in range(3):
        keep(A, c, pages, [np.sort(r.choice(n, max(0, n - int(r.integers(0, 30))), replace=False)) for n in c.lengths])


def test_keep_of_shared_pages_leaves_the_others_theirs(A):
    r = np.random.default_rng(11)
    c = cache(r, 4, 2, 64, 32, [100, 77], spare=40)
    c.fork([0, -1, -1, -1])
    for x in (1, 2, 3):
        share(c, x, 0)
    pages = upload(A, c)
    keep(A, c, pages, [np.sort(r.choice(n, 50 + x // 2, replace=False)) for x, n in enumerate(c.lengths)])
    keep(A, c, pages, [np.arange(int(n) - (g % 3)) for g, n in enumerate(c.lengths)])


def test_keep_many_heads(A):
    r = np.random.default_rng(12)
    c = cache(r, 700, 2, 64, 32, r.integers(0, 70, 1400), spare=2100)
    pages = upload(A, c)
    keep(A, c, pages, [np.sort(r.choice(n, int(r.integers(0, n + 1)), replace=False)) for n in c.lengths])


@pytest.mark.parametrize("n,spare", [(64, 300), (64, 2500), (65, 300)])
def test_keep_plans(A, n, spare):
    """256 heads and more; a beginning of whole pages, of one page, of all but the last rows, and none."""
    r = np.random.default_rng(n + spare)
    c = cache(r, n, 4, 64, 32, r.integers(0, 300, n * 4), spare=spare)
    pages = upload(A, c)
    for _ in range(2):
        kept = []
        for g, m in enumerate(c.lengths):
            first = [min(m, 32), min(m, 128), max(m - 5, 0), 0][g % 4]
            rest = np.arange(first, m) if g % 4 == 2 else np.sort(r.choice(np.arange(first, m), (m - first) // 2, replace=False))
            kept.append(np.concatenate([np.arange(first), rest[:len(rest) - g % 2]]))
        keep(A, c, pages, kept)


def test_keep_of_long_heads(A):
    r = np.random.default_rng(14)
    c = cache(r, 2, 2, 64, 32, [3000, 2049, 2500, 64], spare=300)
    pages = upload(A, c)
    first = [1024, 0, 2400, 32]
    keep(A, c, pages, [np.concatenate([np.arange(f), np.sort(r.choice(np.arange(f, n), (n - f) // 2, replace=False))]) for f, n in zip(first, c.lengths)])


def test_keep_cuts_indices(A):
    """Outside a head's rows they are the nearest of its rows, in the pool and nowhere else."""
    r = np.random.default_rng(13)
    c = cache(r, 1, 1, 64, 32, [50], spare=4)
    pages = upload(A, c)
    keep(A, c, pages, [[-5, 3, 49, 50, 2**31 - 1]])


# ---- attend ----------------------------------------------------------------------------------------------------------------------

def attend(A, c, G, rng, scale=None, q_scale=2.0 ** -6, check=True, **more):
    q = bf16(rng.standard_normal((c.n_seqs, c.H * G, c.d)) * q_scale).cuda()
    lse = torch.full(q.shape[:2], 77.0, device="cuda")
    out = torch.full_like(q, 77.0)
    p = params(A, c, G, **({} if scale is None else {"softmax_scale": scale}))
    A.pages_attend(p, upload(A, c), q, out=out, lse=lse, **more)
    if check:
        attend_error(c, values(q), c.d ** -0.5 if scale is None else float(np.float32(scale)), values(out), values(lse))
    return q, out, lse


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("P", [32, 64, 128, 256])
@pytest.mark.parametrize("G", [1, 7, 16])
def test_attend(A, d, P, G):
    r = np.random.default_rng(d + P + G)
    attend(A, cache(r, 4, 3, d, P, [0, 1, 2, 31, 32, 33, 63, 64, 65, 257, 700, 1500]), G, r)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("G", [1, 8, 9, 16])
def test_attend_short_tables(A, d, G):
    """A workgroup per head: few heads, and more of them with longer tables."""
    r = np.random.default_rng(d + G)
    attend(A, cache(r, 4, 3, d, 32, [0, 1, 2, 31, 32, 33, 63, 64, 65, 257, 400, 512], max_pages=16), G, r)
    attend(A, cache(r, 50, 3, d, 128, np.where(r.random(150) < 0.8, r.integers(0, 60, 150), r.integers(0, 2049, 150)), max_pages=16), G, r)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("G", [1, 7, 16])
@pytest.mark.parametrize("P", [32, 128])
def test_attend_heads_in_parts(A, d, G, P):
    """Tables that long heads would fit in: heads are shared out among workgroups, whatever they are long."""
    r = np.random.default_rng(d + G + P)
    attend(A, cache(r, 4, 3, d, P, [0, 1, 2, 31, 32, 33, 63, 64, 65, 257, 700, 2900], max_pages=4000 // P), G, r)


@pytest.mark.parametrize("lengths", [[1], [0], [5], [129], [4096], [20000], [0, 0, 0, 0, 0, 0, 0, 9], [3000, 1, 1, 1, 1, 1, 1, 1]])
def test_attend_few(A, lengths):
    r = np.random.default_rng(sum(lengths))
    for most in (None, 400):
        attend(A, cache(r, 1, len(lengths), 128, 64, lengths, max_pages=most), 4, r)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_attend_many_heads(A, d):
    """More heads than a workgroup has threads, most of them empty or short: several to a workgroup."""
    r = np.random.default_rng(d)
    lengths = np.where(r.random(900) < 0.7, 0, r.integers(1, 90, 900))
    lengths[[0, 400, 899]] = 800, 1200, 0
    attend(A, cache(r, 300, 3, d, 32, lengths), 2, r)


@pytest.mark.parametrize("d,G", [(64, 4), (64, 16), (128, 7), (128, 12), (256, 2), (256, 9)])
def test_attend_in_a_large_pool(A, d, G):
    """A pool that the memory-side cache does not hold: rows are streamed."""
    r = np.random.default_rng(d + G)
    c = cache(r, 3, 2, d, 64, [0, 1, 33, 700, 2900, 1025], max_pages=64)
    pages = upload(A, c)
    n = (300 << 20) // c.page_bytes
    pool = torch.zeros(n * c.page_bytes, dtype=torch.uint8, device="cuda")
    pool[:pages.pool.numel()] = pages.pool
    pages.pool, pages.refs = pool, torch.cat((pages.refs, torch.zeros(n - c.n_pages, dtype=torch.int32, device="cuda")))
    q = bf16(r.standard_normal((3, 2 * G, d)) * 2.0 ** -6).cuda()
    lse = torch.empty((3, 2 * G), device="cuda")
    out = A.pages_attend(params(A, c, G), pages, q, lse=lse)
    attend_error(c, values(q), d ** -0.5, values(out), values(lse))


@pytest.mark.parametrize("d,H,lengths", [(64, 1, [300_000]), (128, 2, [100_000, 5]), (256, 1, [60_001])])
def test_attend_one_long_head(A, d, H, lengths):
    """As many parts of a head as there are workgroups."""
    r = np.random.default_rng(d)
    attend(A, cache(r, 1, H, d, 256, lengths), 1, r)


@pytest.mark.parametrize("q_scale,scale", [(2.0 ** -2, None), (8.0, None), (64.0, None), (2.0 ** -6, 1.0), (2.0 ** -6, 1e-6)])
def test_attend_where_the_reference_moves(A, q_scale, scale):
    """Logits over many octaves, rising along a head, so that the running reference moves often."""
    r = np.random.default_rng(14)
    c = cache(r, 2, 2, 128, 64, [1000, 999, 650, 3])
    c.pool[c.table[0, :16], 64 * 128:64 * 128 + 64 * 4] = (np.arange(16) // 2 + 118)[:, None]
    attend(A, c, 4, r, scale, q_scale)


def test_attend_equal_keys(A):
    """All weights equal: the mean of V, and a log-sum-exp that is known."""
    r = np.random.default_rng(15)
    c = cache(r, 1, 2, 128, 64, [777, 64])
    c.pool[:, :64 * 64] = 0
    _, out, lse = attend(A, c, 4, r)
    assert np.allclose(values(lse)[0, :4], math.log(777), rtol=1e-6)


def test_attend_infinities_and_nan(A):
    """A block that stands for NaN reaches the queries of its head and no others; noise behind the last row reaches nobody (cache()
    puts it there); queries with an infinity or NaN."""
    r = np.random.default_rng(16)
    P, d = 32, 128
    for section in (P * d, P * d + P * d // 32):                              # K's scales, V's
        c = cache(r, 3, 2, d, P, [40, 64, 33, 5, 70, 32])
        c.pool[c.table[0, 1], section + 7 * 4 + 2] = 255                      # row 39 of head 0
        c.pool[c.table[0, 1], section + 8 * 4:section + P * 4] = 255          # behind its last
        c.pool[c.table[3, 0], section + 5 * 4:section + P * 4] = 255          # behind head 3's last
        q = bf16(r.standard_normal((3, 8, d)) * 2.0 ** -6)
        q[2, 5, 3] = math.nan
        q[1, 1, 3] = math.inf
        pages, lse = upload(A, c), torch.empty((3, 8), device="cuda")
        out = A.pages_attend(params(A, c, 4), pages, q.cuda(), lse=lse)
        got, ls = values(out), values(lse)
        if section == P * d:
            assert np.isnan(got[0, :4]).all() and np.isnan(ls[0, :4]).all()
        else:
            assert np.isnan(got[0, :4, 64:96]).all() and np.isfinite(np.delete(got[0, :4], range(64, 96), axis=1)).all()
            assert np.isfinite(ls[0, :4]).all()
        assert np.isnan(got[2, 5]).all() and np.isnan(ls[2, 5])
        fine = np.ones((3, 8), dtype=bool)
        fine[0, :4] = fine[2, 5] = fine[1, 1] = False
        assert np.isfinite(got[fine]).all() and np.isfinite(ls[fine]).all()


def test_attend_logits_of_minus_infinity(A):
    """Products that overflow: a query all of whose logits are -infinity gives zeros, one with some of them the others."""
    r = np.random.default_rng(17)
    c = cache(r, 2, 1, 64, 32, [70, 40])
    c.pool[:, :32 * 32] = 0x66                                                # 4 in every channel
    c.pool[:, 32 * 64:32 * 64 + 64] = 127
    c.pool[c.table[0, :3], 32 * 64:32 * 64 + 64] = 200
    c.pool[c.table[0, 1], 32 * 64 + 20:32 * 64 + 30] = 127
    q = np.full((2, 2, 64), -2.0 ** 60)
    q[1] = 1
    qt = bf16(q).cuda()
    lse = torch.empty((2, 2), device="cuda")
    out = values(A.pages_attend(params(A, c, 2), upload(A, c), qt, lse=lse))
    k, v = c.rows(0)
    least = (k == 4).all(1)
    assert least.sum() == 5
    assert np.allclose(out[0, 0], v[least].mean(0), rtol=2.0 ** -7) and np.isfinite(values(lse)[0]).all()
    c.pool[c.table[0, :3], 32 * 64:32 * 64 + 64] = 200
    out = values(A.pages_attend(params(A, c, 2), upload(A, c), qt, lse=lse))
    assert not out[0].any() and (values(lse)[0] == -math.inf).all() and np.isfinite(out[1]).all()


def test_attend_pages_that_are_none(A):
    """Entries outside the pool, and lengths beyond a table row: no rows, and no access."""
    r = np.random.default_rng(18)
    c = cache(r, 2, 2, 64, 32, [90, 64, 40, 33])
    q = bf16(r.standard_normal((2, 4, 64)) * 2.0 ** -6).cuda()
    p = params(A, c)
    pages = upload(A, c)
    whole = A.pages_attend(p, pages, q)
    pages.table[0, 1] = -1
    pages.table[3, 0] = c.n_pages
    pages.table[3, 1] = 2**31 - 1
    out = A.pages_attend(p, pages, q)
    assert torch.equal(out[0, 2:], whole[0, 2:]) and torch.equal(out[1, :2], whole[1, :2]) and not out[1, 2:].any()
    k, v = c.rows(0)
    there = np.r_[0:32, 64:90]                                                # the same without that page
    z = k[there] @ values(q)[0, :2].T * 0.125
    w = np.exp(z - z.max(0))
    assert np.allclose(values(out)[0, :2], (w.T @ v[there]) / w.sum(0)[:, None], rtol=2.0 ** -7, atol=2.0 ** -9 * np.abs(v).max())
    pages.lengths[:] = ints([-5, 2**31 - 1, -2**31, 10**6])
    out = A.pages_attend(p, pages, q)
    assert not out[0, :2].any() and not out[1, :2].any()


def test_attend_parts_join_by_their_log_sum_exp(A):
    """A cache in two caches, joined by the caller, is the cache in one."""
    r = np.random.default_rng(19)
    c = cache(r, 1, 2, 128, 32, [320, 320])
    a, b = cache(r, 1, 2, 128, 32, [0]), cache(r, 1, 2, 128, 32, [0])
    for part, at in ((a, slice(0, 4)), (b, slice(4, 10))):
        part.pool, part.n_pages, part.refs = c.pool, c.n_pages, c.refs
        part.table = np.ascontiguousarray(np.pad(c.table[:, at], ((0, 0), (0, 6))))
        part.lengths = np.full(2, 32 * (at.stop - at.start), dtype=np.int32)
    q = bf16(r.standard_normal((1, 8, 128)) * 2.0 ** -6).cuda()
    outs, lses = [], []
    for part in (a, b):
        lse = torch.empty((1, 8), device="cuda")
        outs.append(values(A.pages_attend(params(A, part, 4), upload(A, part), q, lse=lse)))
        lses.append(values(lse))
    m = np.logaddexp(*lses)
    joined = sum(o * np.exp(s - m)[..., None] for o, s in zip(outs, lses))
    ref, ref_lse = c.attend(values(q), 128 ** -0.5)
    k, v = c.rows(0)
    assert np.allclose(m, ref_lse, rtol=1e-5, atol=1e-5)
    assert (np.abs(joined - ref) <= 2.0 ** -8 * sum(np.abs(o) * np.exp(s - m)[..., None] for o, s in zip(outs, lses)) + 2.0 ** -13 * np.abs(v).max()).all()
