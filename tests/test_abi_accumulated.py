"""What the entry points around accumulated weights refuse, and what they say a call needs. No kernel runs here."""
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


def accumulate(A, p, lens, queries, q=PTR, k=PTR, cu=PTR, cu_q=PTR, weights=PTR, pitch=0, ws=PTR, size=1 << 40, n=None):
    cp = p.c()
    return A.binding._lib.audiokv_accumulate(C.byref(cp), q, k, None, cu, i32(lens), cu_q, i32(queries),
                                             len(lens or []) if n is None else n, weights, C.c_int64(pitch), ws, C.c_size_t(size), None)


def test_accumulate_refusals(A):
    p = A.Params(8, 2, 64, 0)
    assert accumulate(A, A.Params(8, 3, 64, 0), [10], [5]) == -1
    assert accumulate(A, A.Params(8, 2, 80, 0), [10], [5]) == -2
    assert accumulate(A, p, [10], [11]) == -1                     # more queries than tokens
    assert accumulate(A, p, [10], [-1]) == -1
    assert accumulate(A, p, [0], [0]) == -1                       # no tokens
    assert accumulate(A, p, None, None, n=1) == -1
    assert accumulate(A, p, [10], None) == -1
    assert accumulate(A, p, [10], [5], n=-1) == -1
    assert accumulate(A, p, [10], [5], q=None) == -1
    assert accumulate(A, p, [10], [5], k=ODD) == -1
    assert accumulate(A, p, [10], [5], weights=None) == -1
    assert accumulate(A, p, [10, 20], [5, 5], pitch=19) == -1
    assert b"pitch" in A.binding._lib.audiokv_last_error()
    assert accumulate(A, p, [10], [5], size=8) == -3
    assert accumulate(A, p, [2**30], [2**30]) == -2               # 2^31 weights
    assert accumulate(A, A.Params(8, 1, 64, 0), [2**30 - 1] * 1, [2**30 - 1]) == -2
    assert accumulate(A, A.Params(8, 2, 64, 0, kv_stride_head=640, kv_stride_tok=64), [10, 10], [5, 5]) == -1   # two items, no item stride


def test_accumulate_of_nothing(A):
    p = A.Params(8, 2, 64, 0)
    assert accumulate(A, p, [], [], q=None, k=None, cu=None, cu_q=None, weights=None, ws=None, size=0) == 0
    assert accumulate(A, p, [10, 7], [0, 0]) == 0                 # no query: nothing is enqueued
    assert A.accumulate_workspace_bytes(p, [], []) == 0
    with pytest.raises(ValueError):
        A.accumulate_workspace_bytes(p, [10], [])


def test_accumulate_workspace(A):
    p = A.Params(28, 4, 128, 0)
    small, large = A.accumulate_workspace_bytes(p, [700], [700]), A.accumulate_workspace_bytes(p, [32768], [32768])
    assert 28 * 700 * 8 <= small < large < 2**30


def slots(A, capacity=16, k=PTR, v=PTR, lengths=PTR, weights=PTR, positions=PTR, size=None):
    S = A.binding._CSlots
    return S(C.sizeof(S) if size is None else size, capacity, k, v, lengths, weights, positions)


def shared(A, p, items=1, rows=100, n=4, most=4, s=None, own=0, q=PTR, kp=PTR, vp=PTR, cu=PTR, cu_s=PTR, kn=None, vn=None, pos=None,
           out=PTR, ws=PTR, size=1 << 40):
    cp = p.c()
    return A.binding._lib.audiokv_decode_shared(C.byref(cp), q, kp, vp, cu, items, C.c_int64(rows), cu_s, n, most, s and C.byref(s), own,
                                                kn, vn, pos, out, ws, C.c_size_t(size), None)


def test_decode_shared_refusals(A):
    p = A.Params(8, 2, 64, 0)
    last = A.binding._lib.audiokv_last_error
    assert shared(A, A.Params(8, 3, 64, 0)) == -1
    assert shared(A, A.Params(66, 2, 64, 0)) == -2                # 33 query heads a KV head
    for bad in (dict(items=-1), dict(n=-1), dict(rows=-1), dict(rows=2**31), dict(most=0), dict(q=None), dict(kp=None), dict(vp=None),
                dict(cu=None), dict(cu_s=None), dict(out=None), dict(ws=None), dict(q=ODD), dict(kp=ODD), dict(out=ODD), dict(ws=ODD),
                dict(kn=PTR), dict(vn=PTR), dict(kn=PTR, vn=PTR)):     # a new row without slots
        assert shared(A, p, **bad) == -1, bad
    assert shared(A, p, size=64) == -3
    for bad in (dict(size=8), dict(k=None), dict(v=None), dict(lengths=None), dict(k=ODD), dict(capacity=0), dict(capacity=7)):
        assert shared(A, p, s=slots(A, **bad), own=8) == -1, bad
    assert shared(A, p, s=slots(A), own=-1) == -1
    assert shared(A, p, s=slots(A), own=8, kn=PTR, vn=PTR) == -1 and b"pos_new" in last()
    assert shared(A, p, s=slots(A), own=8, kn=ODD, vn=PTR, pos=PTR) == -1
    assert shared(A, p, s=slots(A), own=0, kn=PTR, vn=PTR, pos=PTR) == -1
    strided = A.Params(8, 2, 64, 0, kv_stride_head=16 * 64, kv_stride_tok=64)
    assert shared(A, strided, s=slots(A), own=8) == -1 and b"kv_stride_item" in last()
    assert shared(A, p, n=2**24, most=1) == -2                    # more heads than a launch holds
    # without prompts their pointers do not matter; then the workspace is looked at last
    assert shared(A, p, items=0, rows=0, most=0, kp=None, vp=None, cu=None, cu_s=None, s=slots(A), own=8, size=64) == -3


def test_decode_shared_of_prompts_without_rows(A):
    # a compacted cache without rows has no address; its table and the sequences still have
    p = A.Params(8, 2, 64, 0)
    assert shared(A, p, rows=0, kp=None, vp=None, size=64) == -3
    assert shared(A, p, rows=0, kp=None, vp=None, cu=None) == -1
    assert shared(A, p, rows=0, kp=None, vp=None, cu_s=None) == -1


def test_decode_shared_of_nothing(A):
    p = A.Params(8, 2, 64, 0)
    assert shared(A, p, items=0, n=0, q=None, kp=None, vp=None, cu=None, cu_s=None, out=None, ws=None, size=0) == 0
    assert A.decode_shared_workspace_bytes(p, 0, 0, 0, 0, 0) == 0


def test_decode_shared_workspace_never_shrinks(A):
    rows = sorted({max(0, (m << s) + e) for s in range(7, 22) for m in (1, 3, 64, 65, 511, 512, 513) for e in (-1, 0, 1)}
                  | set(range(0, 2_000_000, 9973)))
    for p, n, most in ((A.Params(28, 4, 128, 0), 40, 20), (A.Params(8, 2, 256, 0), 3, 1), (A.Params(32, 1, 64, 0), 300, 300)):
        sizes = [A.decode_shared_workspace_bytes(p, 2, r, n, most, 0) for r in rows]
        assert sizes == sorted(sizes)
        sizes = [A.decode_shared_workspace_bytes(p, 0, 0, n, 0, r) for r in range(0, 9000, 31)]
        assert sizes == sorted(sizes)


def evict(A, p, s, n=2, budget=4, budgets=None, recent=2, own=16, ws=PTR, size=1 << 40):
    cp = p.c()
    return A.binding._lib.audiokv_evict_accumulated(C.byref(cp), s and C.byref(s), n, budget, budgets, recent, own, ws, C.c_size_t(size), None)


def test_evict_accumulated_refusals(A):
    p = A.Params(8, 2, 64, 0)
    assert evict(A, A.Params(8, 3, 64, 0), slots(A)) == -1
    assert evict(A, p, None) == -1
    for bad in (dict(size=8), dict(k=None), dict(v=ODD), dict(lengths=None), dict(capacity=15), dict(weights=None), dict(positions=None)):
        assert evict(A, p, slots(A, **bad)) == -1, bad
    for bad in (dict(n=-1), dict(budget=-1), dict(recent=-1), dict(own=-1)):
        assert evict(A, p, slots(A), **bad) == -1, bad
    assert evict(A, p, slots(A), n=2**20) == -2
    big = slots(A, capacity=4096)
    assert evict(A, p, big, own=4096, budget=2000, size=64) == -3
    assert evict(A, p, big, own=4096, budget=2000, ws=None) == -1


def test_evict_accumulated_of_nothing(A):
    p = A.Params(8, 2, 64, 0)
    assert evict(A, p, None, n=0) == 0
    assert evict(A, p, slots(A), budget=16) == 0                  # nobody can have too many: nothing is enqueued
    assert A.evict_accumulated_workspace_bytes(p, 2, 16, 16) == 0
    assert A.evict_accumulated_workspace_bytes(p, 2, 5000, 2000) > 0
    assert A.evict_accumulated_workspace_bytes(p, 2, 5000, 4900) == 0     # few moves: the ranking workgroup makes them
