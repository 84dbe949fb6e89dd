"""What an attention call with masks launches (ea_host.cpp), driven over sizes by tests/native/attend_plan_main.cpp.  CPU only."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_room_for_tokens_is_not_taken_for_tokens(tmp_path):
    exe = str(tmp_path / "attend_plan")
    cmd = ["g++", "-std=c++17", "-O1", "-o", exe, os.path.join(ROOT, "tests", "native", "attend_plan_main.cpp"),
           os.path.join(ROOT, "paper_2510_00636_amd", "csrc", "ea_host.cpp")]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "attention plans follow from what is cached" in r.stdout
