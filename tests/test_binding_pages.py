"""What the binding of the cache in pages refuses before the library is called, and what it lets through. CPU only: tensors without
memory stand for the device's, and the library's functions note that they were reached."""
import pytest
import torch

from test_binding_accumulated import A, BF16, F32, I32, dev       # noqa: F401 (A: a fixture)

U8 = torch.uint8


def pages(A, **change):
    """Three sequences of two KV heads of 64 channels, four pages at most each, in a pool of ten."""
    return A.Pages(**{**dict(pool=dev(10 * 64 * 68, dtype=U8), table=dev(6, 4, dtype=I32), lengths=dev(6, dtype=I32), refs=dev(10, dtype=I32),
                             state=dev(2, dtype=I32), page_rows=64), **change})


def params(A, **more):
    return A.Params(4, 2, 64, 0, **more)


def append(A, g=None, p=None, **change):
    given = dict(k=dev(80 * 2 * 64), v=dev(80 * 2 * 64), seqlens=[50, 30], cu_seqlens=dev(3, dtype=I32), seqs=dev(2, dtype=I32),
                 indices=dev(40, dtype=I32), cu_budgets=dev(5, dtype=I32), total_rows=40, refused=dev(1, dtype=I32),
                 workspace=dev(1 << 16, dtype=U8))
    given.update(change)
    A.pages_append(p or params(A), g or pages(A), **given)


def attend(A, g=None, p=None, **change):
    A.pages_attend(p or params(A), g or pages(A), **{**dict(q=dev(3, 4, 64), out=dev(3, 4, 64), lse=dev(3, 4, dtype=F32), workspace=dev(1 << 16, dtype=U8)), **change})


def fork(A, g=None, p=None, **change):
    A.pages_fork(p or params(A), g or pages(A), **{**dict(parents=dev(3, dtype=I32), drop=dev(3, dtype=I32), workspace=dev(1 << 16, dtype=U8)), **change})


def keep(A, g=None, p=None, **change):
    A.pages_keep(p or params(A), g or pages(A), **{**dict(indices=dev(40, dtype=I32), cu_budgets=dev(7, dtype=I32), total_rows=40,
                                                          refused=dev(1, dtype=I32), workspace=dev(1 << 16, dtype=U8)), **change})


def read(A, g=None, p=None, **change):
    A.pages_read(p or params(A), g or pages(A), **{**dict(cu_rows=dev(7, dtype=I32), total_rows=40, first=dev(6, dtype=I32), k_out=dev(40, 64),
                                                          v_out=dev(40, 64)), **change})


CALLS = {"append": append, "attend": attend, "fork": fork, "keep": keep, "read": read}


def refused(name, A, *args, **change):
    del A.reached[:]
    with pytest.raises(ValueError):
        CALLS[name](A, *args, **change)
    assert "audiokv_pages_" + name not in A.reached, change


@pytest.mark.parametrize("name", sorted(CALLS))
def test_what_fits_is_taken(A, name):
    CALLS[name](A)
    CALLS[name](A, pages(A, pool=dev(10 * 64 * 68 + 5, dtype=U8)))
    assert A.reached.count("audiokv_pages_" + name) == 2


@pytest.mark.parametrize("name", sorted(CALLS))
def test_caches_that_are_refused(A, name):
    for bad in (dict(pool=dev(10 * 64 * 68 - 1, dtype=U8)), dict(pool=dev(10 * 64 * 68, dtype=torch.int8)), dict(page_rows=128),
                dict(pool=dev(20 * 64 * 68, dtype=U8)[::2]), dict(table=dev(5, 4, dtype=I32)), dict(table=dev(24, dtype=I32)),
                dict(table=dev(4, 6, dtype=I32).T), dict(table=dev(6, 4, dtype=torch.int64)), dict(lengths=dev(5, dtype=I32)),
                dict(lengths=dev(7, dtype=I32), table=dev(7, 4, dtype=I32)), dict(lengths=dev(12, dtype=I32)[::2]), dict(lengths=dev(6, dtype=F32)),
                dict(refs=dev(11, dtype=I32)), dict(refs=dev(10, dtype=torch.int64)), dict(refs=dev(20, dtype=I32)[::2]),
                dict(state=dev(1, dtype=I32)), dict(state=dev(3, dtype=I32)), dict(state=dev(4, dtype=I32)[::2]),
                dict(state=dev(2, dtype=torch.int64))):
        refused(name, A, pages(A, **bad))
    for where in ("cuda:1", "cpu"):
        for field, shape, dtype in (("pool", (10 * 64 * 68,), U8), ("table", (6, 4), I32), ("lengths", (6,), I32), ("refs", (10,), I32), ("state", (2,), I32)):
            refused(name, A, pages(A, **{field: dev(*shape, dtype=dtype, device=where)}))


SIZES = {"append": dict(seqs=(2, I32), indices=(40, I32), refused=(1, I32), cu_budgets=(5, I32), cu_seqlens=(3, I32), k=(80 * 128, BF16), v=(80 * 128, BF16)),
         "attend": dict(out=(3 * 4 * 64, BF16), lse=(12, F32)), "fork": dict(parents=(3, I32), drop=(3, I32)),
         "keep": dict(indices=(40, I32), cu_budgets=(7, I32), refused=(1, I32)),
         "read": dict(cu_rows=(7, I32), first=(6, I32), k_out=(40 * 64, BF16), v_out=(40 * 64, BF16))}


@pytest.mark.parametrize("name", sorted(SIZES))
def test_tensors_that_are_too_small_or_of_another_kind(A, name):
    for field, (n, dtype) in SIZES[name].items():
        CALLS[name](A, **{field: dev(n + 1, dtype=dtype)})
        refused(name, A, **{field: dev(n - 1, dtype=dtype)})
        refused(name, A, **{field: dev(n, dtype=torch.float64)})
        refused(name, A, **{field: dev(2 * n + 2, dtype=dtype)[::2]})
        for where in ("cuda:1", "cpu"):
            refused(name, A, **{field: dev(n, dtype=dtype, device=where)})
    if name != "read":
        refused(name, A, workspace=dev(1 << 16, dtype=U8, device="cuda:1"))
        refused(name, A, workspace=dev(1 << 17, dtype=U8)[::2])


def test_queries_must_be_those_of_all_sequences(A):
    for q in (dev(2, 4, 64), dev(4, 4, 64), dev(3, 2, 64), dev(3, 4, 64, dtype=F32), dev(3, 4, 128)[..., ::2], dev(3, 4, 64, device="cuda:1")):
        refused("attend", A, q=q)


def test_rows_that_strides_lead_out_of_are_refused(A):
    slab = params(A, kv_stride_item=2 * 52 * 64, kv_stride_head=52 * 64, kv_stride_tok=64)
    end = (2 * 52 + 52 + 29) * 64 + 64                        # of item 1's last row
    append(A, None, slab, k=dev(end), v=dev(end + 8)[8:])
    refused("append", A, None, slab, k=dev(end - 1), v=dev(end))
    refused("append", A, None, slab, k=dev(end), v=dev(end)[8:])


def test_without_indices_all_rows_are_meant(A):
    """total_rows is what the lengths say then, for the workspace, too."""
    seen = []
    A.binding._lib.__dict__["audiokv_pages_append"] = lambda *args: seen.append(args[7]) or 0
    append(A, indices=None, cu_budgets=None, total_rows=7)
    append(A)
    assert seen == [160, 40]


def test_a_cache_is_made_empty():
    import paper_2604_06694_amd as A
    g = A.Pages.empty(A.Params(28, 4, 128, 0), 3, 20, 5, 32, device="cpu")
    assert g.pool.numel() == 20 * 4352 and g.table.shape == (12, 5) and g.state.tolist() == [20, 0] and g.n_seqs(A.Params(28, 4, 128, 0)) == 3
    assert not g.lengths.any() and not g.refs.any()
