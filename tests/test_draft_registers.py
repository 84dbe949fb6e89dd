"""The loads from memory to LDS of the kernel with masks leave m0 as they find it, as those without do.  Read from the object that the
build leaves next to the package.  CPU only."""
import os
import re
import subprocess

import pytest

import paper_2510_00636_amd as ea

LLVM = "/opt/rocm/llvm/bin"


@pytest.mark.skipif(not os.path.exists(os.path.join(LLVM, "llvm-objdump")), reason="no ROCm toolchain")
def test_loads_to_lds_leave_m0_as_it_was(tmp_path):
    obj = os.path.join(os.path.dirname(os.path.abspath(ea.__file__)), "_build", "ea_attend_tile_tree.hip.o")
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


@pytest.mark.skipif(not os.path.exists(os.path.join(LLVM, "llvm-readelf")), reason="no ROCm toolchain")
def test_two_workgroups_of_the_fp32_kernel_are_on_a_cu(tmp_path):
    """Wavefronts over rows at d = 128, without masks: from 169 registers on two wavefronts are on a SIMD, of up to 168 three, which take
    each other's keys out of the L1 cache."""
    obj = os.path.join(os.path.dirname(os.path.abspath(ea.__file__)), "_build", "ea_attend_f32.hip.o")
    if not os.path.exists(obj):
        import __graft_entry__
        __graft_entry__.build()
    fat, code = str(tmp_path / "fat"), str(tmp_path / "code")
    subprocess.run([os.path.join(LLVM, "llvm-objcopy"), "--dump-section", ".hip_fatbin=" + fat, obj, os.devnull], check=True, timeout=60)
    subprocess.run([os.path.join(LLVM, "clang-offload-bundler"), "--type=o", "--unbundle", "--input=" + fat,
                    "--targets=hipv4-amdgcn-amd-amdhsa--gfx950", "--output=" + code], check=True, timeout=60)
    notes = subprocess.run([os.path.join(LLVM, "llvm-readelf"), "--notes", code], check=True, timeout=60, capture_output=True, text=True).stdout
    registers = {}
    for part in notes.split(".agpr_count:")[1:]:
        name = re.search(r"\.name:\s+(\S+)", part).group(1)
        registers[name] = int(re.search(r"\.vgpr_count:\s+(\d+)", part).group(1))
    over_rows = [n for x, n in registers.items() if "k_attend_f32ILi128ELb0E" in x]
    assert over_rows and all(169 <= n <= 256 for n in over_rows), registers
