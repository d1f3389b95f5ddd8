"""What the compiler made of the kernels of accumulate, decode_shared and evict_accumulated: no register of theirs lives in memory.
CPU only."""
import pytest

from test_kernel_code import LIB, code_objects, pytestmark, resources      # noqa: F401 (fixtures)

KERNELS = {"accumulate_rows_kernel<": 6, "accumulate_norm_kernel": 1, "accumulate_cols_kernel<": 6, "accumulate_join_kernel": 1,
           "shared_partial_kernel<": 3, "shared_join_kernel<": 2, "evict_rank_kernel<": 3, "evict_move_kernel": 1}


@pytest.mark.parametrize("part", sorted(KERNELS))
def test_no_vector_register_is_spilled(resources, part):
    found = {name: spills for name, (_, spills, _) in resources.items() if part in name}
    assert len(found) == KERNELS[part] and not any(found.values()), found
