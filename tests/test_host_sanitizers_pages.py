"""The host code behind the cache in pages (validation, sizes, planning) under AddressSanitizer and UndefinedBehaviorSanitizer, driven by
tests/abi_pages_check.cpp. CPU only: nothing is launched."""
import os
import shutil
import subprocess

import pytest


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_host_paths_are_clean_under_asan_and_ubsan():
    from paper_2604_06694_amd.build import build_sanitized
    exe = os.path.join(os.path.dirname(build_sanitized(verbose=False)), "abi_pages_check")
    env = dict(os.environ)
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=0:verify_asan_link_order=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "all checks passed" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-4000:]
