"""Registers of the prompt kernels, from what the compiler reports (no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2502_06766_amd import build as hip_build


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
