"""Registers of the prompt kernels, from what the compiler reports, and the plans of their calls (no GPU)."""
import os
import re
import subprocess

import pytest

import test_sanitizers_cpu as san
from paper_2502_06766_amd import build as hip_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("source,instances", [("prompt.hip", 32), ("coded_prompt.hip", 32)])
def test_no_register_of_the_16_bit_kernels_is_in_memory(source, instances):
    """Scratch memory of prompt_kernel<type, format, d, waves, sums put aside>, as the library is built, where queries have 16 bits (type 1 or 2): none, or the room of the
    sums put aside (d / 2 + 3 numbers a lane, in whole 16 bytes)."""
    run = subprocess.run([hip_build.HIPCC, *hip_build.FLAGS, *hip_build.SOURCE_FLAGS.get(source, []), "--offload-device-only",
                          "-Rpass-analysis=kernel-resource-usage", "-c", os.path.join(hip_build.CSRC, source), "-o", os.devnull],
                         capture_output=True, text=True, check=True)
    found = {}
    for line in run.stderr.splitlines():
        name = re.search(r"Function Name: (\S+)", line)
        if name:
            kernel = re.match(r"_ZN3tka13prompt_kernelILi([12])ELi(n?\d)ELi(\d+)ELi\dELb([01])", name.group(1))
        scratch = re.search(r"ScratchSize \[bytes/lane\]: (\d+)", line)
        if scratch and kernel:
            room = (int(kernel.group(3)) // 2 + 3) * 4 if kernel.group(4) == "1" else 0
            found[kernel.group(0)] = int(scratch.group(1)) - (room + 15) // 16 * 16
    assert len(found) == instances
    assert not any(found.values()), {k: v for k, v in found.items() if v}


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")
def test_plans_of_the_widest_windows_under_ubsan(tmp_path):
    obj, exe = str(tmp_path / "plan.o"), str(tmp_path / "plan")
    host = [x for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all") for x in ("-Xarch_host", f)]
    subprocess.check_call([hip_build.HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", *host, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-c",
                           os.path.join(ROOT, "tests", "sanitize_prompt_plan_driver.hip"), "-o", obj], stderr=subprocess.DEVNULL)
    subprocess.check_call([hip_build.HIPCC, "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", obj, "-o", exe],
                          stderr=subprocess.DEVNULL)
    env = dict(san.ENV, ASAN_OPTIONS=san.ENV["ASAN_OPTIONS"] + ":protect_shadow_gap=0",
               LSAN_OPTIONS="suppressions=" + os.path.join(ROOT, "tests", "sanitize_lsan.supp") + ":print_suppressions=0")
    run = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert run.returncode == 0 and "plan driver: done" in run.stdout, run.stdout + run.stderr
