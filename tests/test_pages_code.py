"""What the compiler made of the kernels of the cache in pages: no register or variable of theirs lives in memory, and attend keeps the
waves per SIMD that its grid counts on. CPU only."""
import re

import pytest

from test_accumulated_code import private_bytes                                     # noqa: F401 (fixture)
from test_kernel_code import code_objects, named, pytestmark, resources             # noqa: F401 (fixtures)

KERNELS = {"append_plan_kernel": 1, "append_plan_small_kernel<": 2, "append_rows_kernel<": 6, "read_kernel<": 6, "fork_take_kernel": 1,
           "fork_give_kernel": 1, "fork_small_kernel<": 2, "keep_plan_kernel<": 2, "keep_move_kernel<": 3, "keep_table_kernel": 1,
           "keep_whole_kernel<": 3, "attend_kernel<": 18, "::join_kernel<": 3}


@pytest.mark.parametrize("part", sorted(KERNELS))
def test_no_vector_register_is_spilled(resources, part):
    found = {name: spills for name, (_, spills, _) in resources.items() if part in name}
    assert len(found) == KERNELS[part] and not any(found.values()), found


@pytest.mark.parametrize("part", sorted(KERNELS))
def test_no_variable_lies_in_memory(private_bytes, part):
    """(names are mangled here: the number before a name is its length)"""
    bare = part.strip("<:")
    found = {name: n for name, n in private_bytes.items() if f"{len(bare)}{bare}" in name}
    assert len(found) == KERNELS[part] and not any(found.values()), found


def test_attend_has_as_many_waves_as_its_grid_counts_on(resources):
    for name, (vgprs, _, _) in named(resources, "attend_kernel<").items():
        d = int(re.search(r"attend_kernel<(\d+)", name).group(1))
        assert vgprs <= {64: 128, 128: 168, 256: 256}[d], (name, vgprs)
