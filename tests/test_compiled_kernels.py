"""What the compiler made of the kernels, read from the built library's own code: no lane's value is lost where branches meet, and attention's loops keep all they hold in registers."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1902_01064_amd", "libhop.so")
OBJDUMP, READELF = "/opt/rocm/llvm/bin/llvm-objdump", "/opt/rocm/llvm/bin/llvm-readelf"

pytestmark = pytest.mark.skipif(not all(os.path.exists(p) for p in (LIB, OBJDUMP, READELF)), reason="needs the built library and the HIP toolchain")

# instructions that work on scalars, whichever lanes are on
SCALAR = ("v_readlane", "v_writelane", "v_readfirstlane", "v_nop")
WIDENS = re.compile(r"s_or_b64 exec, exec|s_mov_b64 exec, -1|s_or_saveexec_b64|s_xor_b64 exec")
NARROWS_OR_ENDS = re.compile(r"s_\w+ exec|s_\w+_saveexec|v_cmpx|s_c?branch|s_endpgm")


def lost_lanes(code):
    """(kernel, block, instructions) of every block that is jumped to with no lane on (so a branch of some lanes ends there) and that writes vector registers or
    memory before it has the other lanes on again.  A compiler short of registers has put copies and spills there: lanes that had not taken the branch kept none."""
    found = []
    for part in re.split(r"\n(?=(?:[0-9a-f]+ )?<_Z\S+>:)", code)[1:]:
        name = re.search(r"<(\S+)>:", part)[1]
        body = [line.split("//")[0].strip() for line in part.split("\n")[1:]]
        ends = {line.split()[1] for line in body if line.startswith("s_cbranch_execz")}
        block, written = None, []
        for line in body:
            label = re.match(r"<(\S+)>:", line)
            if label:
                block, written = label[1] if label[1] in ends else None, []
            elif block and WIDENS.match(line):
                if written:
                    found.append((name, block, written))
                block = None
            elif block and NARROWS_OR_ENDS.match(line):
                block = None
            elif block and line.startswith(("v_", "scratch_", "global_", "flat_", "buffer_", "ds_")) and not line.startswith(SCALAR):
                written.append(line)
    return found


HEAD = "code\n<_Zkernel>:\n\ts_and_saveexec_b64 s[2:3], vcc // 00\n\ts_cbranch_execz L0 // 04\n\tglobal_load_dword v0, v[2:3], off // 08\n<L0>:\n"


@pytest.mark.parametrize("lines,lost", [
    ("s_or_b64 exec, exec, s[2:3]\nv_mov_b32_e32 v1, v0", 0), ("v_mov_b32_e32 v1, v0\ns_mov_b64 s[4:5], s[6:7]\ns_or_b64 exec, exec, s[2:3]", 1),
    ("scratch_store_dwordx2 off, v[26:27], off offset:60\ns_or_b64 exec, exec, s[2:3]", 1), ("v_accvgpr_write_b32 a112, v186\ns_or_b64 exec, exec, s[4:5]", 1),
    ("v_readlane_b32 s2, v255, 20\nv_writelane_b32 v255, s2, 1\ns_or_b64 exec, exec, s[2:3]", 0), ("v_mov_b32_e32 v1, v0\ns_endpgm", 0),
    ("v_mov_b32_e32 v1, v0\ns_and_saveexec_b64 s[4:5], vcc\ns_or_b64 exec, exec, s[4:5]", 0)])
def test_the_search_finds_what_it_is_for(lines, lost):
    assert len(lost_lanes(HEAD + lines + "\n")) == lost


@pytest.fixture(scope="module")
def objects(tmp_path_factory):
    folder = tmp_path_factory.mktemp("kernels")
    shutil.copy(LIB, folder / "libhop.so")
    subprocess.run([OBJDUMP, "--offloading", "libhop.so"], cwd=folder, check=True, capture_output=True)
    return sorted(str(p) for p in folder.iterdir() if p.name.endswith("gfx950"))


def test_no_lane_loses_a_value_where_branches_meet(objects):
    kernels = 0
    for o in objects:
        code = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", "--no-leading-addr", o], capture_output=True, text=True, check=True).stdout
        kernels += len(re.findall(r"^<_Z\S+>:", code, re.M))
        assert not lost_lanes(code)
    assert kernels > 100


def test_attention_keeps_what_it_holds_in_registers(objects):
    kernels = 0
    for o in objects:
        notes = subprocess.run([READELF, "--notes", o], capture_output=True, text=True, check=True).stdout
        for name, scratch in re.findall(r"\.name:\s*(_Z\S+)\n(?:.*\n)*?\s*\.private_segment_fixed_size:\s*(\d+)", notes):
            if "attention_kernel" in name:
                kernels += 1
                assert int(scratch) == 0, name
    assert kernels >= 4
