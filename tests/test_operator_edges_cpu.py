"""Edges of the operators beside the top-k decode that need no GPU."""
import os
import subprocess

import numpy as np
import pytest

import operator_bounds as ob
import test_sanitizers_cpu as san
from paper_2502_06766_amd import build as hip_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")
def test_selections_longer_than_any_decode_has_are_refused(tmp_path):
    """k up to the largest max_k reaches the kernel, whose 32-bit count stays within its range; beyond it the call is refused."""
    host = [x for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all") for x in ("-Xarch_host", f)]
    common = [hip_build.HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", *host, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
    objs = []
    for src in (os.path.join(hip_build.CSRC, "api_ops.hip"), os.path.join(ROOT, "tests", "sanitize_mass_driver.hip")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.check_call([*common, "-c", src, "-o", objs[-1]], stderr=subprocess.DEVNULL)
    exe = str(tmp_path / "mass_san")
    subprocess.check_call([hip_build.HIPCC, "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", *objs, "-o", exe],
                          stderr=subprocess.DEVNULL)
    env = dict(san.ENV, ASAN_OPTIONS=san.ENV["ASAN_OPTIONS"] + ":protect_shadow_gap=0",
               LSAN_OPTIONS="suppressions=" + os.path.join(ROOT, "tests", "sanitize_lsan.supp") + ":print_suppressions=0",
               HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, f"{r.stdout[-2000:]}\n{r.stderr[-4000:]}"
    assert "mass driver: all checks passed" in r.stdout


@pytest.mark.parametrize("dtype,enough", [(ob.F16, 2), (ob.BF16, 3)])
def test_the_bound_of_the_weights_tells_their_parts(dtype, enough):
    """Weights in one part fewer than the kernel takes (and, in bf16, in two fewer) exceed the bound that the GPU test holds; those it takes do not."""
    g = np.random.default_rng(0)
    q, k = ob.grid_scores(g, 4, 64)
    w = np.exp2(q[:, None].astype(np.float64) * k * (np.log2(np.e) / 8))
    exact = w / w.sum(1, keepdims=True)
    w32 = w.astype(np.float32)
    for parts in range(1, enough + 1):
        got = ob.in_parts(w32, dtype, parts) / w32.astype(np.float64).sum(1, keepdims=True)
        off = (np.abs(got - exact) / exact).max()
        assert (off <= ob.quotient_bound(dtype, 10)) == (parts == enough), (parts, off, ob.quotient_bound(dtype, 10))
