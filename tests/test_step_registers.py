"""The loads from memory to LDS that are written out leave m0 as they find it.  Read from the objects that the build leaves next to
the package.  CPU only."""
import os
import re
import subprocess

import pytest

import paper_2510_00636_amd as ea

LLVM = "/opt/rocm/llvm/bin"


@pytest.mark.skipif(not os.path.exists(os.path.join(LLVM, "llvm-objdump")), reason="no ROCm toolchain")
def test_loads_to_lds_leave_m0_as_it_was(tmp_path):
    obj = os.path.join(os.path.dirname(os.path.abspath(ea.__file__)), "_build", "ea_attend_tile.hip.o")
    if not os.path.exists(obj):
        import __graft_entry__
        __graft_entry__.build()
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.run([os.path.join(LLVM, "llvm-objcopy"), "--dump-section", ".hip_fatbin=" + fat, obj, os.devnull], check=True, timeout=60)
    subprocess.run([os.path.join(LLVM, "clang-offload-bundler"), "--type=o", "--unbundle", "--input=" + fat,
                    "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--output=" + code], check=True, timeout=60)
    text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", code], check=True, timeout=60,
                          capture_output=True, text=True).stdout
    lines = [x.split("//")[0].strip() for x in text.splitlines()]
    loads = [i for i, x in enumerate(lines) if x.startswith("global_load_lds")]
    assert len(loads) > 50
    for i in loads:
        kept = re.fullmatch(r"s_mov_b32 (s\d+|vcc_lo|vcc_hi|ttmp\d+), m0", lines[i - 3])
        assert kept and lines[i - 2].startswith("s_mov_b32 m0, ") and lines[i - 1] == "s_nop 0", lines[i - 3:i + 2]
        assert lines[i + 1] == "s_mov_b32 m0, " + kept.group(1), lines[i - 3:i + 2]
    assert sum(x.startswith("s_mov_b32 m0,") for x in lines) == 2 * len(loads)      # and nobody else writes it
