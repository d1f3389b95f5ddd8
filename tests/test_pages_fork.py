"""What a thread of fork's second launch does, on the host, in whatever order threads run. CPU only."""
import shutil

import pytest

from test_accumulated_limits import run_on_host


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not available")
def test_fork_gives_back_in_any_order_of_threads(tmp_path):
    run_on_host("pages_fork_check", tmp_path)
