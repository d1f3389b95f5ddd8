"""Tables of more entries than 32 bits count are refused: the library would be told what is left of their width. CPU only: tensors without
memory stand for the device's."""
import pytest

from test_binding_accumulated import A, I32, dev       # noqa: F401 (A: a fixture)
from test_binding_pages import CALLS, U8, pages, params, refused


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("shape", [(6, 2**32 + 4), (6, 2**31), (2**32 + 6, 1)])
def test_tables_beyond_32_bits(A, name, shape):
    refused(name, A, pages(A, table=dev(*shape, dtype=I32), lengths=dev(shape[0], dtype=I32)))


def test_sizes_of_tables_beyond_32_bits(A):
    g = pages(A, table=dev(6, 2**32 + 4, dtype=I32))
    for size in (A.pages_attend_workspace_bytes, A.pages_fork_workspace_bytes):
        with pytest.raises(ValueError):
            size(params(A), g)
    assert not A.reached
