"""What the entry points around the cache in pages refuse, and what they say a call needs. No kernel runs here."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def i32(values):
    return None if values is None else (C.c_int32 * max(1, len(values)))(*values)


PTR = C.c_void_p(4096)          # never read: every call here is refused first
ODD = C.c_void_p(4104)
HUGE = 1 << 40


def cache(A, size=None, page_rows=64, n_pages=100, max_pages=10, pool=PTR, table=PTR, lengths=PTR, refs=PTR, state=PTR):
    G = A.binding._CPages
    return G(C.sizeof(G) if size is None else size, page_rows, n_pages, max_pages, pool, table, lengths, refs, state)


def append(A, p, g, n=4, k=PTR, v=PTR, idx=None, cu_b=None, rows=0, cu=PTR, lens=(5, 7), items=None, seqs=None, ws=PTR, size=HUGE):
    return A.binding._lib.audiokv_pages_append(C.byref(p.c()), g and C.byref(g), n, k, v, idx, cu_b, C.c_int64(rows), cu, i32(lens),
                                               len(lens or []) if items is None else items, seqs, None, ws, C.c_size_t(size), None)


def attend(A, p, g, n=4, q=PTR, out=PTR, ws=PTR, size=HUGE):
    return A.binding._lib.audiokv_pages_attend(C.byref(p.c()), g and C.byref(g), n, q, out, None, ws, C.c_size_t(size), None)


def fork(A, p, g, n=4, parents=PTR, drop=None, ws=PTR, size=HUGE):
    return A.binding._lib.audiokv_pages_fork(C.byref(p.c()), g and C.byref(g), n, parents, drop, ws, C.c_size_t(size), None)


def keep(A, p, g, n=4, idx=PTR, cu=PTR, rows=10, ws=PTR, size=HUGE):
    return A.binding._lib.audiokv_pages_keep(C.byref(p.c()), g and C.byref(g), n, idx, cu, C.c_int64(rows), None, ws, C.c_size_t(size), None)


def read(A, p, g, n=4, cu=PTR, rows=10, k=PTR, v=PTR):
    return A.binding._lib.audiokv_pages_read(C.byref(p.c()), g and C.byref(g), n, None, cu, C.c_int64(rows), k, v, None)


CALLS = [append, attend, fork, keep, read]


@pytest.mark.parametrize("call", CALLS)
def test_caches_that_are_refused(A, call):
    p = A.Params(8, 2, 64, 0)
    for bad in (dict(size=8), dict(page_rows=16), dict(page_rows=48), dict(page_rows=512), dict(page_rows=0), dict(page_rows=-64),
                dict(n_pages=0), dict(max_pages=0), dict(n_pages=-1), dict(pool=None), dict(pool=ODD), dict(table=None), dict(lengths=None),
                dict(refs=None), dict(state=None)):
        assert call(A, p, cache(A, **bad)) == -1, bad
    assert call(A, p, None) == -1
    assert call(A, p, cache(A), n=-1) == -1
    assert call(A, A.Params(8, 3, 64, 0), cache(A)) == -1
    assert call(A, A.Params(8, 2, 80, 0), cache(A)) == -2
    assert call(A, p, cache(A), n=2**20) == -2                                    # 2^21 heads
    assert call(A, p, cache(A, max_pages=2**29), n=4) == -2                       # more entries than 32 bits count
    assert call(A, p, cache(A, max_pages=2**27, page_rows=256), n=1) == -2        # more units of 32 rows
    assert call(A, p, cache(A, max_pages=2**25), n=1) == -2                       # more rows of a head


@pytest.mark.parametrize("call", CALLS)
def test_no_sequences(A, call):
    assert call(A, A.Params(8, 2, 64, 0), None, n=0) == 0


def test_append_refusals(A):
    p = A.Params(8, 2, 64, 0)
    for bad in (dict(k=None), dict(v=None), dict(cu=None), dict(k=ODD), dict(v=ODD), dict(lens=None, items=2), dict(lens=(5, 0)),
                dict(lens=(5, -1)), dict(items=-1), dict(idx=PTR), dict(cu_b=PTR, rows=5), dict(cu_b=PTR, rows=-1), dict(lens=(1,) * 5),       # five items, four sequences
                dict(idx=PTR, cu_b=PTR, rows=-1), dict(idx=PTR, cu_b=PTR, rows=25), dict(ws=None), dict(ws=ODD)):
        assert append(A, p, cache(A), **bad) == -1, bad
    assert append(A, p, cache(A), size=64) == -3
    assert append(A, p, cache(A), lens=(1,) * 5, seqs=PTR, size=64) == -3
    assert append(A, p, cache(A), idx=PTR, cu_b=PTR, rows=24, size=64) == -3
    assert append(A, p, cache(A), cu_b=PTR, rows=0, size=64) == -3                # budgets of zero: no indices
    assert append(A, p, cache(A), lens=(2**30, 2**30)) == -2
    assert append(A, A.Params(8, 2, 64, 0, kv_stride_head=640, kv_stride_tok=64), cache(A)) == -1     # two items, no item stride
    assert append(A, p, cache(A), lens=(), k=None, v=None, cu=None, ws=None) == 0
    assert append(A, A.Params(8, 2, 64, 500), cache(A), size=64) == -3                                # the window plays no part


def test_attend_refusals(A):
    p = A.Params(8, 2, 64, 0)
    for bad in (dict(q=None), dict(out=None), dict(q=ODD), dict(out=ODD), dict(ws=None), dict(ws=ODD)):
        assert attend(A, p, cache(A), **bad) == -1, bad
    assert attend(A, p, cache(A), size=64) == -3
    assert attend(A, A.Params(34, 2, 64, 0), cache(A)) == -2                      # 17 query heads a KV head
    with pytest.raises(A.AudioKVError):
        A.binding._size_of("audiokv_pages_attend_workspace_bytes", A.Params(34, 2, 64, 0), C.byref(cache(A)), 4)


def test_fork_keep_and_read_refusals(A):
    p = A.Params(8, 2, 64, 0)
    for bad in (dict(ws=None), dict(ws=ODD)):
        assert fork(A, p, cache(A), **bad) == -1 and keep(A, p, cache(A), **bad) == -1
    assert fork(A, p, cache(A), size=64) == -3 and keep(A, p, cache(A), size=64) == -3
    assert fork(A, p, cache(A), parents=None) == 0                                # nobody changes: nothing is enqueued
    for bad in (dict(idx=None), dict(cu=None), dict(rows=-1), dict(rows=2**31)):
        assert keep(A, p, cache(A), **bad) == -1, bad
    assert keep(A, p, cache(A), idx=None, rows=0, size=64) == -3                  # (of none: allowed)
    for bad in (dict(cu=None), dict(k=None), dict(v=None), dict(k=ODD), dict(v=ODD), dict(rows=-1), dict(rows=2**31)):
        assert read(A, p, cache(A), **bad) == -1, bad
    assert read(A, p, cache(A), cu=None, rows=0, k=None, v=None) == 0


def test_sizes(A):
    p = A.Params(28, 4, 128, 0)
    assert [A.page_bytes(p, n) for n in (32, 64, 128, 256)] == [4352, 8704, 17408, 34816]
    for bad in (0, 16, 33, 512):
        with pytest.raises(A.AudioKVError):
            A.page_bytes(p, bad)
    size = A.binding._size_of
    g = cache(A)
    assert size("audiokv_pages_append_workspace_bytes", p, C.byref(g), 4, 0, 0) == 0
    assert size("audiokv_pages_attend_workspace_bytes", p, C.byref(g), 0) == 0
    # sizes look at no pointer
    bare = cache(A, pool=None, table=None, lengths=None, refs=None, state=None)
    for name, more in (("append", (4, 2, 100)), ("attend", (4,)), ("fork", (4,)), ("keep", (4, 100))):
        name = f"audiokv_pages_{name}_workspace_bytes"
        assert size(name, p, C.byref(bare), *more) == size(name, p, C.byref(g), *more) > 0
    # a small cache asks for no large one's workspace
    assert size("audiokv_pages_attend_workspace_bytes", p, C.byref(cache(A, max_pages=1)), 1) < 2**20
