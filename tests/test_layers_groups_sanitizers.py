"""The rule for gradients of groups that share memory, host code only, under AddressSanitizer and UBSan (kernel launchers are stubs)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"), reason="needs g++ and the HIP headers")
def test_groups_places_are_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "layers_groups_driver")
    csrc = os.path.join(ROOT, "paper_1902_01064_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
           "-ffp-contract=off", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
           os.path.join(ROOT, "tests", "layers_groups_driver.cpp"), os.path.join(csrc, "hop_layers.cpp"), os.path.join(csrc, "hop_sim.cpp"),
           "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    subprocess.run(cmd, check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0")
    out = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-4000:]
    told = dict(p.split("=") for p in out.stdout.split()[1:])
    assert out.stdout.startswith("ok ") and int(told["good"]) > 500 and int(told["bad"]) > 500 and int(told["launches"]) == int(told["good"]), out.stdout
