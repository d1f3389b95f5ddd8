"""The largest sizes that accumulate, decode_shared and evict_accumulated can be asked for: right, or refused. CPU only."""
import ctypes as C
import os
import shutil
import subprocess

import pytest


@pytest.fixture(scope="module")
def A():
    import paper_2604_06694_amd as A
    return A


def test_decode_shared_workspace_up_to_the_last_number(A):
    """A logit per query head and own row is the least that a step needs."""
    p = A.Params(8, 2, 64, 0)
    for own in (2**30 - 1, 2**30, 2**31 - 64, 2**31 - 1):
        try:
            assert A.decode_shared_workspace_bytes(p, 0, 0, 1, 0, own) >= 8 * own * 4, own
        except A.AudioKVError as e:
            assert e.code == -2 and own >= 2**30


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_limits_under_asan_and_ubsan():
    from paper_2604_06694_amd.build import build_sanitized
    exe = os.path.join(os.path.dirname(build_sanitized(verbose=False)), "abi_accumulated_limits_check")
    env = dict(os.environ)
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=0:verify_asan_link_order=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "all checks passed" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]


ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run_on_host(check, tmp_path):
    exe = str(tmp_path / check)
    r = subprocess.run(["hipcc", "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++20", "-O1", "-I",
                        os.path.join(ROOT, "paper_2604_06694_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", check + ".cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr


def test_pieces_of_moved_rows(tmp_path):
    """The pieces of 2^25 moved rows at head_dim 256 are more than 32 bits count: moves are counted."""
    run_on_host("row_moves_check", tmp_path)
    with open(os.path.join(ROOT, "paper_2604_06694_amd", "csrc", "evict_accumulated.hip")) as f:
        assert "listed[0] * per" not in f.read()


PTR = C.c_void_p(4096)          # never read


def accumulate(A, lens, queries, q=PTR, workspace=PTR, size=1 << 40, lse=None, k=PTR):
    cp = A.Params(8, 2, 64, 0).c()
    i32 = C.c_int32 * len(lens)
    return A.binding._lib.audiokv_accumulate(C.byref(cp), q, k, lse, PTR, i32(*lens), PTR, i32(*queries), len(lens), PTR, C.c_int64(0),
                                             workspace, C.c_size_t(size), None)


def test_accumulate_of_no_query_needs_neither_queries_nor_workspace(A):
    """An empty tensor of queries has no address, and a workspace of no bytes none either."""
    assert A.accumulate_workspace_bytes(A.Params(8, 2, 64, 0), [10, 7], [0, 0]) == 0
    assert accumulate(A, [10, 7], [0, 0], q=None, workspace=None, size=0) == 0
    assert accumulate(A, [10, 7], [0, 0], k=None) == -1           # the rest is looked at
    assert accumulate(A, [10, 7], [1, 0], q=None) == -1
    assert accumulate(A, [10, 7], [1, 0], workspace=None) == -1


@pytest.mark.parametrize("heads,lens,queries", [((32, 8), [131072] + [500] * 255, None), ((28, 4), [131072] + [300] * 255, [2000] + [300] * 255),
                                                ((28, 4), [32768] * 28, None), ((1, 1), [1], None)])
def test_accumulate_workspace_does_not_grow_with_ragged_items(A, heads, lens, queries):
    """A norm per query, and what 256 workgroups at most find for the two blocks at most that each shares with others: a
    (reference, sum) per row, a sum per key, of blocks of at most 448."""
    queries = queries or lens
    most = heads[0] * sum(queries) * 4 + 2 * 256 * 448 * (8 + 4) + 3 * 256
    assert A.accumulate_workspace_bytes(A.Params(*heads, 128, 0), lens, queries) <= most


def test_slots_of_shared_blocks(tmp_path):
    run_on_host("accumulate_slots_check", tmp_path)


@pytest.mark.parametrize("items,rows,seqs,most", [(64, 64 * 4 * 5000, 512, 512), (500, 500 * 4 * 400, 999, 500), (1, 4 * 13107, 32, 32)])
def test_decode_shared_workspace_follows_the_sequences(A, items, rows, seqs, most):
    """A result per sequence, query head and first chunk, and per sequence of the widest item and later chunk, of which there are
    less than twice as many as wanted: 384 workgroups, in blocks of 128 query rows."""
    blocks = -(-most * 7 // 128)
    results = seqs * 28 + 2 * -(-384 // blocks) * most * 7
    assert A.decode_shared_workspace_bytes(A.Params(28, 4, 128, 0), items, rows, seqs, most, 0) <= results * (128 * 4 + 8) + seqs * 4 * 4 + 4 * 256
