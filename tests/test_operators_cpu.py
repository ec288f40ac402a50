"""Oracle of the operators beside the decode, pinned against things that are not the oracle, and static checks of their kernels."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import operators_ref as ref
from paper_2502_06766_amd import build as hip_build
from paper_2502_06766_amd import isa_check
from paper_2502_06766_amd import topk_attn as ta

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_attention_is_the_library_softmax():
    g = np.random.default_rng(0)
    q, K, V = g.standard_normal((4, 16)), g.standard_normal((2, 50, 16)), g.standard_normal((2, 50, 16))
    out, lse, mass = ref.attend(q, K, V)
    s = torch.from_numpy(np.einsum("hd,hnd->hn", q, K.repeat(2, 0)) / 4)
    np.testing.assert_allclose(lse, torch.logsumexp(s, 1).numpy(), rtol=1e-13)
    np.testing.assert_allclose(out, torch.einsum("hn,hnd->hd", torch.softmax(s, 1), torch.from_numpy(V.repeat(2, 0))).numpy(), rtol=1e-12)
    np.testing.assert_allclose(mass.sum(1), 2.0)


def test_rotation_keeps_lengths_and_depends_on_the_distance():
    g = np.random.default_rng(1)
    x, y = g.standard_normal((1, 1, 32)), g.standard_normal((1, 1, 32))
    freq = 10000.0 ** (-np.arange(16) / 16)
    for inter in (False, True):
        turn = lambda z, p: ref.rms_rotate(z, None, 0.0, [p], freq, inter)[0, 0]
        np.testing.assert_allclose(np.linalg.norm(turn(x, 77)), np.linalg.norm(x))
        np.testing.assert_allclose(turn(x, 100) @ turn(y, 93), turn(x, 12) @ turn(y, 5), atol=1e-12)
        np.testing.assert_allclose(turn(x, 0), x[0, 0])
    one = ref.rms_rotate(x, np.full(32, 2.0), 0.0, [0], freq[:0], False)
    np.testing.assert_allclose((one ** 2).mean(), 4.0)


def test_page_scores_bound_every_key_and_survivors_are_the_heaviest():
    g = np.random.default_rng(2)
    q, K = g.standard_normal((6, 8)), g.standard_normal((2, 200, 8))
    s = ref.page_scores(q, K)
    raw = np.einsum("hgd,hnd->hgn", q.reshape(2, 3, 8), K).max(1)
    for p in range(4):
        assert (raw[:, 64 * p:64 * p + 64].max(1) <= s[:, p] + 1e-12).all()
    assert all(3 in head and len(head) == 2 for head in ref.pick_blocks(q, K, 2))
    mass = np.array([[5.0, 1.0, 5.0, 0.0, np.nan, 5.0, 9.0, 0.0]], np.float32)
    assert list(ref.survivors(mass, 8, 4, 1)[0]) == [0, 2, 6, 7]
    assert list(ref.survivors(mass, 7, 6, 0)[0]) == [0, 1, 2, 3, 5, 6]


def test_rotary_struct_matches_the_header():
    # uint32 + 2 int32 + float, int64, 3 pointers, 6 int64, 5 pointers
    assert ctypes.sizeof(ta.Rotary) == 16 + 8 + 24 + 48 + 40


def test_block_index_storage():
    base = dict(n_layers=2, n_seqs=3, n_q_heads=40, n_kv_heads=2, head_dim=32, max_tokens=1000, max_k=64)
    up = lambda x: (x + 255) // 256 * 256
    for dtype, e in ((ta.F32, 4), (ta.BF16, 2)):
        heads = dict(base, n_q_heads=4) if dtype == ta.F32 else base
        plain = ta.topk_attn_kv_bytes(ta.make_config(dtype=dtype, **heads))
        cfg = ta.make_config(dtype=dtype, index_kind=ta.INDEX_BOXES, **heads)
        assert ta.topk_attn_kv_bytes(cfg) == plain + up(2 * 3 * 2 * 16 * 2 * 32 * e)
        assert ta.topk_attn_workspace_bytes(cfg) > ta.topk_attn_workspace_bytes(ta.make_config(dtype=dtype, **heads))


def test_null_handles():
    L = ta.lib()
    assert L.topk_attn_decode_dense(None, 0, None, None, None, None, None) == ta.EINVAL
    assert L.topk_attn_decode_blocks(None, 0, None, 1, None, None, None, None, None) == ta.EINVAL
    assert L.topk_attn_add_mass(None, 0, None, None, None, 1, None, None) == ta.EINVAL
    assert L.topk_attn_evict(None, 0, None, 1, 0, None, None) == ta.EINVAL
    assert L.topk_attn_append_rotary(None, 0, 0, None, None) == ta.EINVAL


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")
def test_no_mfma_result_is_read_early_in_the_attention(tmp_path):
    out = str(tmp_path / "dense.s")
    subprocess.check_call([hip_build.HIPCC, *hip_build.FLAGS, "--offload-device-only", "-S", os.path.join(hip_build.CSRC, "dense.hip"), "-o", out],
                          stderr=subprocess.DEVNULL)
    assert open(out).read().count("v_mfma") > 500
    assert not isa_check.check(out)


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")
def test_host_side_of_the_operators_under_asan_and_ubsan(tmp_path):
    """api_ops.hip with sanitized host code, linked with stand-ins for the kernel launchers: refusals, calls that end at a missing device, and the
    launch plans of random shapes, held against the room there is for them."""
    import test_sanitizers_cpu as san
    host = [x for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all") for x in ("-Xarch_host", f)]
    common = [hip_build.HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", *host, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
    objs = []
    for src in (os.path.join(hip_build.CSRC, "api_ops.hip"), os.path.join(ROOT, "tests", "sanitize_ops_driver.hip")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.check_call([*common, "-c", src, "-o", objs[-1]], stderr=subprocess.DEVNULL)
    exe = str(tmp_path / "ops_san")
    subprocess.check_call([hip_build.HIPCC, "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", *objs, "-o", exe],
                          stderr=subprocess.DEVNULL)
    env = dict(san.ENV, ASAN_OPTIONS=san.ENV["ASAN_OPTIONS"] + ":protect_shadow_gap=0",
               LSAN_OPTIONS="suppressions=" + os.path.join(ROOT, "tests", "sanitize_lsan.supp") + ":print_suppressions=0",
               HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, f"sanitizer run failed ({r.returncode}):\n{r.stdout[-2000:]}\n{r.stderr[-4000:]}"
    assert "runtime error" not in r.stderr and "ERROR: AddressSanitizer" not in r.stderr, r.stderr[-4000:]
    assert "ops driver: all checks passed" in r.stdout
