"""Captured cuts whose rows are compared in every replay, and caches that are parts of one pool: the layers of a model, each with slices of
one table and one list of lengths."""
import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("n,most", [(3, 40), (30, 90)])
def test_every_replay_of_a_captured_cut_reads_its_rows(A, n, most):
    r = np.random.default_rng(n)
    H, d, P = 2, 64, 32
    c = cache(r, n, H, d, P, r.integers(200, 400, n * H), spare=n * H * 40, max_pages=most)
    p, pages = params(A, c), upload(A, c)
    total = int(c.lengths.sum())
    idx, cus, refused = ints(np.zeros(total)), ints(np.zeros(n * H + 1)), ints([0])
    k, v = (torch.zeros((total, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(max(A.pages_keep_workspace_bytes(p, pages, total), A.pages_fork_workspace_bytes(p, pages)), dtype=torch.uint8, device="cuda")

    def step():
        A.pages_keep(p, pages, idx, cus, total, refused=refused, workspace=ws)
        A.pages_read(p, pages, cus, total, k_out=k, v_out=v)

    def fill(kept):
        idx[:sum(len(x) for x in kept)] = ints(np.concatenate(kept))
        cus.copy_(cu([len(x) for x in kept]))

    fill([np.arange(int(m)) for m in c.lengths])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        kept = [np.sort(r.choice(m, m - int(r.integers(0, 40)), replace=False)) for m in c.lengths]
        counts = [len(x) for x in kept]
        fill(kept)
        k.fill_(7)
        v.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert c.keep(kept) == int(refused) == 0
        same(c, pages)
        for got, ref in zip((k, v), c.read([0] * (n * H), counts)):
            assert np.array_equal(values(got[:sum(counts)]), ref), turn
            assert not values(got[sum(counts):]).any(), turn                   # rows that no head has
        parents = r.integers(0, n, n)
        A.pages_fork(p, pages, ints(parents), workspace=ws)
        c.fork(parents)
        same(c, pages)


@pytest.mark.parametrize("d,most", [(64, 12), (128, 900)])
def test_layers_of_one_pool(A, d, most):
    """Every call on the sequences of one layer, all layers in turn: the others keep what they have, and pages go from one to another."""
    r = np.random.default_rng(d)
    layers, n, H, P = 3, 2, 2, 32
    c = cache(r, layers * n, H, d, P, r.integers(0, 200, layers * n * H), spare=90, max_pages=most)
    p, whole = params(A, c, 4), upload(A, c)
    heads = n * H
    layer = [A.Pages(whole.pool, whole.table[a * heads:(a + 1) * heads], whole.lengths[a * heads:(a + 1) * heads], whole.refs, whole.state, P)
             for a in range(layers)]
    for turn in range(3):
        for a, pages in enumerate(layer):
            mine = np.arange(a * n, (a + 1) * n)
            s = Source(r, H, d, r.integers(1, 40, n))
            assert s.call(A, c, pages) == c.append(s.items(), mine) == 0
            same(c, whole)
            q = bf16(r.standard_normal((layers * n, H * 4, d)) * 2.0 ** -6)
            got_lse = torch.empty((n, H * 4), device="cuda")
            out = values(A.pages_attend(p, pages, q[mine].cuda(), lse=got_lse))
            every, every_lse = c.attend(values(q), d ** -0.5)
            every[mine], every_lse[mine] = out, values(got_lse)                # (the others: the oracle's own)
            attend_error(c, values(q), d ** -0.5, every, every_lse)
            parents, drop = np.arange(layers * n), np.zeros(layers * n, dtype=np.int64)
            parents[mine] = mine[0] + r.integers(0, n, n)
            drop[mine] = r.integers(0, 20, n)
            A.pages_fork(p, pages, ints(parents[mine] - mine[0]), drop=ints(drop[mine]))
            c.fork(parents, drop)
            same(c, whole)
            kept = [np.arange(int(m)) for m in c.lengths]
            for g in range(a * heads, (a + 1) * heads):
                kept[g] = np.sort(r.choice(c.lengths[g], int(c.lengths[g]) * 3 // 4, replace=False))
            own = kept[a * heads:(a + 1) * heads]
            counts, refused = [len(x) for x in own], ints([-7])
            A.pages_keep(p, pages, ints(np.concatenate(own)), cu(counts), sum(counts), refused=refused)
            assert c.keep(kept) == int(refused) == 0
            same(c, whole)
            rows = np.zeros(layers * heads, dtype=np.int64)
            rows[a * heads:(a + 1) * heads] = counts
            for got, ref in zip(A.pages_read(p, pages, cu(counts), sum(counts)), c.read([0] * (layers * heads), rows)):
                assert np.array_equal(values(got), ref)
