"""What the binding of accumulate, decode_shared and evict_accumulated refuses before the library is called, and what it lets
through. CPU only: tensors without memory stand for the device's, and the library's functions note that they were reached."""
import warnings

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Library:
    """Stands for the loaded library: every entry point succeeds and is listed in `reached`."""

    def __init__(self):
        self.reached = []

    def __getattr__(self, name):
        def call(*args):
            self.reached.append(name)
            return 0
        return call


@pytest.fixture
def A(monkeypatch):
    import paper_2604_06694_amd as A
    library = Library()
    monkeypatch.setattr(A.binding, "_lib", library)
    monkeypatch.setattr(A.binding, "_raw_device", lambda: 0)
    monkeypatch.setattr(A.binding, "_SIZE_CACHE", {})         # (sizes that this library answers are not the real one's)
    monkeypatch.setattr(A.binding, "_stream", lambda: 0)
    A.reached = library.reached
    with FakeTensorMode(), warnings.catch_warnings():
        warnings.simplefilter("ignore")                       # (that tensors here have no address)
        yield A
    del A.reached


def dev(*shape, dtype=BF16, device="cuda:0"):
    return torch.empty(shape, dtype=dtype, device=device)


def refused(call, A, **change):
    del A.reached[:]
    with pytest.raises(ValueError):
        call(A, **change)
    assert not any(name in ("audiokv_accumulate", "audiokv_decode_shared", "audiokv_evict_accumulated") for name in A.reached), change


# ---- accumulate: two items of 50 and 30 tokens, 20 and 30 queries, 4 query heads on 2 KV heads of 64 channels ----

def accumulate(A, **change):
    given = dict(p=A.Params(4, 2, 64, 0), q=dev(50 * 4 * 64), k=dev(80 * 2 * 64), weights=dev(160, dtype=F32), lse=dev(200, dtype=F32),
                 cu_seqlens=dev(3, dtype=I32), cu_queries=dev(3, dtype=I32), workspace=dev(1 << 16, dtype=torch.uint8), pitch=0)
    given.update(change)
    p, q, k = (given.pop(x) for x in ("p", "q", "k"))
    return A.accumulate(p, q, k, [50, 30], [20, 30], **given)


def test_accumulate_takes_what_fits(A):
    accumulate(A)
    accumulate(A, cu_seqlens=dev(9, dtype=I32), k=dev(81 * 2 * 64), lse=None, weights=None)
    assert A.reached == ["audiokv_accumulate"] * 2


def test_accumulate_refuses_keys_that_end_too_early(A):
    refused(accumulate, A, k=dev(80 * 2 * 64 - 1))
    slab = dict(kv_stride_item=2 * 52 * 64, kv_stride_head=52 * 64, kv_stride_tok=64)
    end = (2 * 52 + 52 + 29) * 64 + 64                        # of item 1's last row, behind which the slab may end
    accumulate(A, p=A.Params(4, 2, 64, 0, **slab), k=dev(end))
    refused(accumulate, A, p=A.Params(4, 2, 64, 0, **slab), k=dev(end - 1))
    accumulate(A, p=A.Params(4, 2, 64, 0, **slab), k=dev(end + 64)[64:80])         # a view: what it is a view of counts
    refused(accumulate, A, p=A.Params(4, 2, 64, 0, **slab), k=dev(end + 63)[64:80])
    # an earlier item may reach further than the last one
    long = dict(kv_stride_item=8, kv_stride_head=64, kv_stride_tok=128)
    accumulate(A, p=A.Params(4, 2, 64, 0, **long), k=dev(49 * 128 + 128))
    refused(accumulate, A, p=A.Params(4, 2, 64, 0, **long), k=dev(49 * 128 + 127))


@pytest.mark.parametrize("name", ["cu_seqlens", "cu_queries"])
def test_accumulate_refuses_tables_that_are_none(A, name):
    for bad in (dev(2, dtype=I32), dev(3, dtype=torch.int64), dev(3, dtype=F32), torch.empty(3, dtype=I32), dev(6, dtype=I32)[::2]):
        refused(accumulate, A, **{name: bad})


# ---- decode_shared: two sequences with 10 own slots a head, on one prompt of 11 rows; the same geometry ----

SLAB = dict(kv_stride_item=2 * 12 * 64, kv_stride_head=12 * 64, kv_stride_tok=64)
SLAB_END = (2 * 12 + 12 + 9) * 64 + 64                        # of the last slot


def slots(A, **change):
    return A.Slots(**{**dict(k=dev(2 * 2 * 10 * 64), v=dev(2 * 2 * 10 * 64), lengths=dev(4, dtype=I32), capacity=10,
                             weights=dev(4, 10, dtype=F32), positions=dev(4, 10, dtype=I32)), **change})


def decode_shared(A, **change):
    given = dict(p=A.Params(4, 2, 64, 0), q=dev(2, 4, 64), k_prompt=dev(11, 64), v_prompt=dev(11, 64), cu_budgets=dev(3, dtype=I32), total_rows=11,
                 cu_seqs=dev(2, dtype=I32), max_seqs=2, slots=slots(A), max_own=8, k_new=dev(2, 2, 64), v_new=dev(2, 2, 64),
                 pos_new=dev(2, dtype=I32), out=dev(2, 4, 64), workspace=dev(1 << 16, dtype=torch.uint8))
    given.update(change)
    return A.decode_shared(**given)


def evict(A, p=None, s=None, budgets=None, workspace=None):
    A.evict_accumulated(p or A.Params(4, 2, 64, 0), s or slots(A), 2, 4, 2, 8, budgets=budgets, workspace=workspace)


def test_slots_that_fit(A):
    decode_shared(A)
    evict(A)
    strided = A.Params(4, 2, 64, 0, **SLAB)
    for s in (slots(A, k=dev(SLAB_END), v=dev(SLAB_END)), slots(A, k=dev(SLAB_END + 8)[8:16], v=dev(2, 2, 12, 64)[:, :, :10])):
        decode_shared(A, p=strided, slots=s)
        evict(A, p=strided, s=s)
    assert A.reached.count("audiokv_decode_shared") == A.reached.count("audiokv_evict_accumulated") == 3


def test_slots_that_strides_lead_out_of_are_refused(A):
    strided = A.Params(4, 2, 64, 0, **SLAB)
    for change in (dict(k=dev(SLAB_END - 1)), dict(v=dev(SLAB_END - 1)), dict(k=dev(SLAB_END)[8:]), dict(capacity=11)):
        s = slots(A, **{**dict(k=dev(SLAB_END), v=dev(SLAB_END), weights=dev(4, 11, dtype=F32), positions=dev(4, 11, dtype=I32)), **change})
        refused(decode_shared, A, p=strided, slots=s)
        refused(evict, A, p=strided, s=s)


@pytest.mark.parametrize("where", ["cuda:1", "cpu"])
def test_tensors_of_another_device_are_refused(A, where):
    def there(*shape, dtype=BF16):
        return dev(*shape, dtype=dtype, device=where)
    for change in (dict(q=there(50 * 4 * 64)), dict(k=there(80 * 2 * 64)), dict(weights=there(160, dtype=F32)), dict(lse=there(200, dtype=F32)),
                   dict(cu_seqlens=there(3, dtype=I32)), dict(cu_queries=there(3, dtype=I32)), dict(workspace=there(1 << 16, dtype=torch.uint8))):
        refused(accumulate, A, **change)
    own = (dict(k=there(2 * 2 * 10 * 64)), dict(v=there(2 * 2 * 10 * 64)), dict(lengths=there(4, dtype=I32)),
           dict(weights=there(4, 10, dtype=F32)), dict(positions=there(4, 10, dtype=I32)))
    for change in (dict(q=there(2, 4, 64)), dict(k_prompt=there(11, 64)), dict(v_prompt=there(11, 64)), dict(cu_budgets=there(3, dtype=I32)),
                   dict(cu_seqs=there(2, dtype=I32)), dict(k_new=there(2, 2, 64)), dict(v_new=there(2, 2, 64)), dict(pos_new=there(2, dtype=I32)),
                   dict(out=there(2, 4, 64)), dict(workspace=there(1 << 16, dtype=torch.uint8)), *(dict(slots=slots(A, **x)) for x in own)):
        refused(decode_shared, A, **change)
    for change in (dict(budgets=there(4, dtype=I32)), dict(workspace=there(1 << 16, dtype=torch.uint8)), *(dict(s=slots(A, **x)) for x in own)):
        refused(evict, A, **change)
    with pytest.raises(ValueError):                           # everything elsewhere: the stream is the current device's
        evict(A, s=slots(A, k=there(2 * 2 * 10 * 64), v=there(2 * 2 * 10 * 64), lengths=there(4, dtype=I32),
                         weights=there(4, 10, dtype=F32), positions=there(4, 10, dtype=I32)))


def test_prompts_of_no_item_are_refused(A):
    """cu_seqs of one entry says that no sequence takes part; a call without items would let all of them."""
    refused(decode_shared, A, cu_seqs=dev(1, dtype=I32))
    refused(decode_shared, A, cu_seqs=dev(0, dtype=I32))
    decode_shared(A, k_prompt=None, v_prompt=None, cu_budgets=None, cu_seqs=None, total_rows=0)      # without prompts all of them do


def test_params_are_plain_values(A):
    """Calls leave nothing in them, setting a field runs no code of ours, and what the library is given is always the fields' values."""
    p = A.Params(4, 2, 64, 0)
    decode_shared(A, p=p)
    evict(A, p=p)
    assert A.Params(**vars(p)) == p and "__setattr__" not in vars(A.Params)
    given = []
    A.binding._lib.__dict__["audiokv_evict_accumulated"] = lambda params, *rest: given.append(bytes(params._obj)) or 0
    for field, value in (("softmax_scale", 0.5), ("kv_layout", 1), ("softmax_scale", 0.25), ("kv_layout", 0), ("softmax_scale", 0.5)):
        setattr(p, field, value)
        evict(A, p=p)
        assert given[-1] == bytes(p.c())
