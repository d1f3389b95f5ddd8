"""What the kernels of the cache in pages compute without memory, on the host: scales, sections of a page, shares of the work and where
their results go. CPU only."""
import shutil

import pytest

from test_accumulated_limits import run_on_host


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_scales_pages_and_shares(tmp_path):
    run_on_host("pages_check", tmp_path)
