"""How the work of accumulated weights is cut into spans, compiled for the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_spans_cover_every_tile_once(tmp_path):
    exe = str(tmp_path / "accumulate_plan_check")
    r = subprocess.run(["hipcc", "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++20", "-O1", "-I",
                        os.path.join(ROOT, "paper_2604_06694_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "accumulate_plan_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
