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
