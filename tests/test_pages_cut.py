"""How attend cuts heads into parts, on the host. CPU only."""
import shutil

import pytest

from test_accumulated_limits import run_on_host


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_shares_that_end_with_heads(tmp_path):
    run_on_host("pages_cut_check", tmp_path)
