"""The cache in pages as a program uses it: together, in graphs, on streams, in pools beyond 32 bits."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as O
from pages_util import Source, attend_error, bf16, cache, params, same, upload, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def cu(counts):
    return ints(np.concatenate([[0], np.cumsum(counts)]))


@pytest.mark.parametrize("d", [64, 128])
def test_a_generation(A, d):
    """A prompt is evicted and appended, forked into a beam, grows and is reordered, loses rejected rows, is cut to a budget, and goes
    on: every step on both sides."""
    r = np.random.default_rng(d)
    H, G, L, W, P = 2, 4, 600, 16, 32
    p = A.Params(H * G, H, d, W)
    src = Source(r, H, d, [L])
    k, v = src.lay(src.k), src.lay(src.v)
    q = bf16(r.standard_normal((1, H * G, W, d))).cuda()
    out = A.evict(p, q.view(-1), k, v, torch.rand(H, device="cuda"), [L], 0.4, 0.125, 1.0)
    counts = np.diff(out["cu_budgets"].cpu().numpy())
    index = out["indices"].cpu().numpy()
    src.index = [index[:counts[0]], index[counts[0]:]]

    pages = A.Pages.empty(p, 4, 200, 40, P)
    c = O.Cache(4, H, d, 200, 40, P, pages.pool.cpu().numpy().reshape(200, -1))
    refused = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.pages_append(p, pages, k, v, [L], indices=out["indices"], cu_budgets=out["cu_budgets"], total_rows=out["total_rows"],
                   seqs=ints([2]), refused=refused)
    assert c.append(src.items(), [2]) == int(refused) == 0
    same(c, pages)
    A.pages_fork(p, pages, ints([2, 2, 2, 2]))
    c.fork([2, 2, 2, 2])
    same(c, pages)
    for step in range(12):
        new = Source(r, H, d, [1] * 4)
        assert new.call(A, c, pages) == c.append(new.items()) == 0
        same(c, pages)
        qs = bf16(r.standard_normal((4, H * G, d)) * 0.5).cuda()
        lse = torch.empty((4, H * G), device="cuda")
        o = A.pages_attend(p, pages, qs, lse=lse)
        attend_error(c, values(qs), d ** -0.5, values(o), values(lse))
        if step % 3 == 1:
            parents = r.integers(0, 4, 4)
            A.pages_fork(p, pages, ints(parents))
            c.fork(parents)
        if step == 5:
            A.pages_fork(p, pages, drop=ints([3, 0, 1, 40]))
            c.fork(None, [3, 0, 1, 40])
        if step == 8:
            kept = [np.concatenate([np.arange(n // 3), np.sort(r.choice(np.arange(n // 3, n), n // 3, replace=False))]) for n in c.lengths]
            A.pages_keep(p, pages, ints(np.concatenate(kept)), cu([len(x) for x in kept]), sum(len(x) for x in kept), refused=refused)
            assert c.keep(kept) == int(refused) == 0
        same(c, pages)
    back = A.pages_read(p, pages, cu(c.lengths), int(c.lengths.sum()))
    for got, ref in zip(back, c.read([0] * 8, c.lengths)):
        assert np.array_equal(values(got), ref)
    A.pages_fork(p, pages, ints([-1] * 4))
    c.fork([-1] * 4)
    same(c, pages)
    assert c.free == 200


def test_a_captured_step_is_replayed(A):
    """append, attend and fork in a graph, filled by seqs, rows, queries and parents; eager calls with the same workspaces, and
    synchronizations, between the replays."""
    r = np.random.default_rng(1)
    n, H, d, P = 5, 2, 128, 32
    c = cache(r, n, H, d, P, [40, 31, 64, 100, 3, 0, 32], spare=120, max_pages=20)
    other = cache(r, n, H, d, P, [700, 3], spare=9)
    p, pages, pages2 = params(A, c, 4), upload(A, c), upload(A, other)
    k, v = (torch.zeros((n, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    seqs, parents, cus = ints([0] * n), ints(range(n)), ints(range(n + 1))
    q = torch.zeros((n, H * 4, d), dtype=torch.bfloat16, device="cuda")
    out, lse, refused = torch.zeros_like(q), torch.zeros((n, H * 4), device="cuda"), ints([0])
    size = max(A.pages_append_workspace_bytes(p, pages, n, n * H), A.pages_attend_workspace_bytes(p, pages),
               A.pages_attend_workspace_bytes(p, pages2), A.pages_fork_workspace_bytes(p, pages))
    ws = torch.randint(0, 255, (size,), dtype=torch.uint8, device="cuda")

    def step():
        A.pages_append(p, pages, k, v, [1] * n, seqs=seqs, cu_seqlens=cus, refused=refused, workspace=ws)
        A.pages_attend(p, pages, q, out=out, lse=lse, workspace=ws)
        A.pages_fork(p, pages, parents, workspace=ws)

    begin = [t.clone() for t in (pages.pool, pages.table, pages.lengths, pages.refs, pages.state)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t, b in zip((pages.pool, pages.table, pages.lengths, pages.refs, pages.state), begin):
        t.copy_(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(6):
        new = Source(r, H, d, [1] * n)
        to = r.permutation(n) if turn % 2 else r.integers(-1, n, n)
        pa = r.integers(-1, n, n) if turn == 3 else np.where(r.random(n) < 0.3, r.integers(0, n, n), np.arange(n))
        k.copy_(new.lay(new.k).view_as(k)), v.copy_(new.lay(new.v).view_as(v)), seqs.copy_(ints(to)), parents.copy_(ints(pa))
        q.copy_(bf16(r.standard_normal(q.shape) * 2.0 ** -6))
        graph.replay()
        torch.cuda.synchronize()
        assert c.append(new.items(), to) == int(refused)
        attend_error(c, values(q), d ** -0.5, values(out), values(lse))
        c.fork(pa)
        same(c, pages)
        eager = A.pages_attend(params(A, other, 4), pages2, q, workspace=ws)       # the same workspace, other contents
        attend_error(other, values(q), d ** -0.5, values(eager))


@pytest.mark.parametrize("n,most", [(3, 40), (40, 90)])
def test_captured_cuts_are_replayed(A, n, most):
    """keep and read in a graph, with small and large tables, filled by indices and budgets; a fork eagerly between the replays."""
    r = np.random.default_rng(n)
    H, d, P = 2, 64, 32
    c = cache(r, n, H, d, P, r.integers(900, 1200, n * H), spare=n * H * 120, max_pages=most)
    p, pages = params(A, c), upload(A, c)
    total = int(c.lengths.sum())
    idx, cus, refused = ints(np.zeros(total)), ints(np.zeros(n * H + 1)), ints([0])
    k, v = (torch.zeros((total, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.randint(0, 255, (max(A.pages_keep_workspace_bytes(p, pages, total), A.pages_fork_workspace_bytes(p, pages)),), dtype=torch.uint8, device="cuda")

    def step():
        A.pages_keep(p, pages, idx, cus, total, refused=refused, workspace=ws)
        A.pages_read(p, pages, cus, total, k_out=k, v_out=v)

    def fill(kept):
        idx[:sum(len(x) for x in kept)] = ints(np.concatenate(kept))
        cus.copy_(cu([len(x) for x in kept]))

    fill([np.arange(int(m)) for m in c.lengths])          # (a head that keeps all of its rows stays as it is)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    same(c, pages)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        kept = [np.sort(r.choice(m, m - int(r.integers(0, 60)), replace=False)) for m in c.lengths]
        fill(kept)
        graph.replay()
        torch.cuda.synchronize()
        assert c.keep(kept) == int(refused) == 0
        same(c, pages)
        counts = [len(x) for x in kept]
        for got, ref in zip((k, v), c.read([0] * (n * H), counts) if turn == 0 else (None, None)):
            assert ref is None or np.array_equal(values(got[:sum(counts)]), ref)
        parents = r.integers(0, n, n)
        A.pages_fork(p, pages, ints(parents), workspace=ws)
        c.fork(parents)
        same(c, pages)


def test_on_another_stream(A):
    r = np.random.default_rng(2)
    c = cache(r, 3, 2, 64, 32, [40, 31, 64], spare=50, max_pages=9)
    pages = upload(A, c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(5):
            new = Source(r, 2, 64, [3, 1, 2])
            assert new.call(A, c, pages) == c.append(new.items()) == 0
        q = bf16(r.standard_normal((3, 4, 64)) * 2.0 ** -6).cuda()
        out = A.pages_attend(params(A, c), pages, q)
    s.synchronize()
    same(c, pages)
    attend_error(c, values(q), 0.125, values(out))


def test_two_steps_at_once_on_one_cache(A):
    """Reading calls may run beside each other, each with a workspace of its own: bit for bit what they give alone."""
    r = np.random.default_rng(3)
    c = cache(r, 6, 2, 128, 64, r.integers(1, 3000, 12))
    p, pages = params(A, c, 4), upload(A, c)
    qs = [bf16(r.standard_normal((6, 8, 128)) * 2.0 ** -6).cuda() for _ in range(4)]
    alone = [A.pages_attend(p, pages, q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    outs = [torch.empty_like(q) for q in qs]
    spaces = [torch.empty(A.pages_attend_workspace_bytes(p, pages), dtype=torch.uint8, device="cuda") for _ in qs]
    for _ in range(5):
        for s, q, o, w in zip(streams, qs, outs, spaces):
            with torch.cuda.stream(s):
                A.pages_attend(p, pages, q, out=o, workspace=w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


def test_equal_inputs_give_equal_bits_wherever_the_pages_lie(A):
    r = np.random.default_rng(4)
    c = cache(r, 4, 2, 128, 64, r.integers(1, 2000, 8), spare=40)
    q = bf16(r.standard_normal((4, 8, 128)) * 2.0 ** -6).cuda()
    first = A.pages_attend(params(A, c, 4), upload(A, c), q)
    perm = r.permutation(c.n_pages)
    moved = cache(r, 4, 2, 128, 64, c.lengths, spare=40)
    moved.pool[perm] = c.pool
    moved.table = perm[np.clip(c.table, 0, c.n_pages - 1)].astype(np.int32)
    assert torch.equal(A.pages_attend(params(A, moved, 4), upload(A, moved), q), first)


def test_a_pool_beyond_32_bits(A):
    """Pages whose bytes begin beyond 2^32, in a pool of 5 GB: every operator."""
    H, d, P = 1, 256, 256
    n_pages = 75000
    r = np.random.default_rng(5)
    p = A.Params(4, H, d, 0)
    pages = A.Pages.empty(p, 3, n_pages, 6, P)
    used = 66000                                   # all pages below belong to somebody else
    pages.refs[:used] = 1
    pages.state[:] = ints([n_pages - used, 70000])
    src = Source(r, H, d, [700, 300])
    refused = ints([9])
    A.pages_append(p, pages, src.lay(src.k), src.lay(src.v), src.lens, refused=refused)
    assert int(refused) == 0 and pages.table[0, :3].tolist() == [70000, 70001, 70002] and pages.table[1, :2].tolist() == [70003, 70004]
    A.pages_fork(p, pages, ints([0, 1, 0]))
    one = Source(r, H, d, [1])
    A.pages_append(p, pages, one.lay(one.k), one.lay(one.v), [1], seqs=ints([2]), refused=refused)
    kept = [np.sort(r.choice(n, n - 50, replace=False)) for n in (700, 300, 701)]
    # the same on the host, in a small pool
    c = O.Cache(3, H, d, 40, 6, P)
    c.append(src.items())
    c.fork([0, 1, 0])
    c.append(one.items(), [2])
    q = bf16(r.standard_normal((3, 4, d))).cuda()
    attend_error(c, values(q), d ** -0.5, values(A.pages_attend(p, pages, q)))
    A.pages_keep(p, pages, ints(np.concatenate(kept)), cu([len(x) for x in kept]), sum(len(x) for x in kept), refused=refused)
    assert c.keep(kept) == int(refused) == 0
    back = A.pages_read(p, pages, cu(c.lengths), int(c.lengths.sum()))
    for got, ref in zip(back, c.read([0] * 3, c.lengths)):
        assert np.array_equal(values(got), ref)
    attend_error(c, values(q), d ** -0.5, values(A.pages_attend(p, pages, q)))
    assert int(pages.state[0]) == n_pages - used - int((c.refs > 0).sum())
