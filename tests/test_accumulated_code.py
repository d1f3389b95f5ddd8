"""What the compiler made of the kernels of accumulate, decode_shared and evict_accumulated: no register or variable of theirs lives
in memory. CPU only."""
import re
import subprocess

import pytest

from test_kernel_code import LLVM, code_objects, pytestmark, resources      # noqa: F401 (fixtures)

KERNELS = {"accumulate_rows_kernel<": 6, "accumulate_norm_kernel": 1, "accumulate_cols_kernel<": 6, "accumulate_join_kernel": 1,
           "shared_partial_kernel<": 3, "shared_join_kernel<": 2, "evict_rank_kernel<": 3, "evict_move_kernel": 1}


@pytest.mark.parametrize("part", sorted(KERNELS))
def test_no_vector_register_is_spilled(resources, part):
    found = {name: spills for name, (_, spills, _) in resources.items() if part in name}
    assert len(found) == KERNELS[part] and not any(found.values()), found


@pytest.fixture(scope="module")
def private_bytes(code_objects):
    """Kernel (its mangled name) -> bytes of memory that a lane has to itself."""
    out = {}
    for f in code_objects:
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", f], check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n  - (?=\.)", notes)[1:]:
            value = [re.search(rf"^\s*{key}:\s+(\S+)", kernel, re.M).group(1) for key in (r"\.name", r"\.private_segment_fixed_size")]
            out[value[0]] = int(value[1])
    return out


@pytest.mark.parametrize("part", sorted(KERNELS))
def test_no_variable_lies_in_memory(private_bytes, part):
    found = {name: n for name, n in private_bytes.items() if part.rstrip("<") in name}
    assert len(found) == KERNELS[part] and not any(found.values()), found
