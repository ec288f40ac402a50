"""Oracle of the 8-bit cache and of windowed attention, pinned against things that are not the oracle, the host side of their entries, and
static checks of their kernels."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import coded_cache_ref as ref
from paper_2502_06766_amd import build as hip_build
from paper_2502_06766_amd import isa_check
from paper_2502_06766_amd import topk_attn as ta

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_e4m3_is_the_types_rounding():
    x = np.concatenate([np.linspace(-448, 448, 20011), np.random.default_rng(0).standard_normal(20000) * 2.0 ** np.random.default_rng(1).integers(-12, 6, 20000)])
    x = x[np.abs(x) <= 448].astype(np.float32)
    np.testing.assert_array_equal(ref.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("fmt", [ref.INT8, ref.E4M3])
@pytest.mark.parametrize("size", [1.0, 1e-25, 3e37])
def test_held_rows_are_near_and_whole_blocks_only(fmt, size):
    g = np.random.default_rng(2)
    x = (g.standard_normal((150, 32)) * size).astype(np.float32).astype(np.float64)
    y = ref.held(x, fmt)
    np.testing.assert_array_equal(y[128:], x[128:])
    for p in range(2):
        b, h = x[64 * p:64 * p + 64], y[64 * p:64 * p + 64]
        amax = np.abs(b).max()
        if fmt == ref.INT8:
            s = ref.scale_of(b, fmt)
            assert abs(s / (amax / 127) - 1) <= 2.0 ** -16 and (s * 2.0 ** 200 * 2.0 ** -np.floor(np.log2(s * 2.0 ** 200)) * 2 ** 15).is_integer()
            assert (np.abs(h - b) <= s / 2 * (1 + 1e-12)).all() and np.abs(h).max() <= 127 * s
        else:
            s = ref.scale_of(b, fmt)
            assert amax <= 448 * s and amax > 224 * s and np.log2(s).is_integer()
            assert (np.abs(h - b) <= np.maximum(2.0 ** -4 * np.abs(b), 2.0 ** -10 * s)).all()
    assert (ref.held(np.zeros((64, 4)), fmt) == 0).all() and (ref.held(np.full((64, 4), 2.0 ** -101), fmt) == 0).all()
    z = np.ones((64, 4))
    z[3, 1] = np.inf
    assert np.isnan(ref.held(z, fmt)).all()


def test_masked_attention_is_the_library_softmax():
    g = np.random.default_rng(3)
    q, K, V = g.standard_normal((9, 4, 16)), g.standard_normal((2, 40, 16)), g.standard_normal((2, 40, 16))
    for sinks, window in ((0, 40), (3, 5), (0, 1), (50, 2)):
        out, lse = ref.attend(q, K, V, sinks, window)
        s = torch.from_numpy(np.einsum("mhd,hnd->mhn", q, K.repeat(2, 0)) / 4)
        p, t = torch.arange(31, 40)[:, None], torch.arange(40)
        s = s.masked_fill(~((t <= p) & ((p - t < window) | (t < sinks)))[:, None], -torch.inf)
        np.testing.assert_allclose(lse, torch.logsumexp(s, 2).numpy(), rtol=1e-12)
        np.testing.assert_allclose(out, torch.einsum("mhn,hnd->mhd", torch.softmax(s, 2), torch.from_numpy(V.repeat(2, 0))).numpy(), rtol=1e-11, atol=1e-14)
    K[0, 0], V[0, 35] = np.nan, np.inf                        # not seen by the row of token 34
    out, _ = ref.attend(q, K, V, 0, 10)
    assert np.isfinite(out[3]).all() and not np.isfinite(out[4, :2]).any()


def test_config_struct_matches_the_header():
    # uint32 + 5 int32, int64, 4 int32, 2 (pointer + size_t)
    assert ctypes.sizeof(ta.CodedConfig) == 24 + 8 + 16 + 32


def test_storage_is_a_byte_an_element_and_two_scales_a_block():
    up = lambda x: (x + 255) // 256 * 256
    for dtype, e in ((ta.F32, 4), (ta.BF16, 2)):
        cfg = ta.make_coded_config(3, 2, 8, 4, 128, 1000, dtype)
        streams, blocks = 3 * 2 * 4, 15
        assert ta.topk_attn_coded_kv_bytes(cfg) == 2 * up(streams * blocks * 64 * 128) + up(streams * blocks * 8) + up(streams * 2 * 64 * 128 * e)
        assert ta.topk_attn_coded_workspace_bytes(cfg) > 0
    for bad in (dict(head_dim=96), dict(dtype=5), dict(format=2), dict(n_q_heads=7), dict(max_tokens=0), dict(n_layers=0)):
        cfg = ta.make_coded_config(**{**dict(n_layers=1, n_seqs=1, n_q_heads=8, n_kv_heads=4, head_dim=64, max_tokens=100, dtype=ta.F16), **bad})
        assert ta.topk_attn_coded_kv_bytes(cfg) == ta.topk_attn_coded_workspace_bytes(cfg) == 0


def test_null_handles():
    L = ta.lib()
    assert L.topk_attn_decode_sinks(None, 0, None, 0, 1, None, None, None) == ta.EINVAL
    assert L.topk_attn_prompt(None, 0, 0, None, 1, 0, 1, None, None, None) == ta.EINVAL
    assert L.topk_attn_coded_append(None, 0, 0, None, None, 1, 0, 0, 0, None) == ta.EINVAL
    assert L.topk_attn_coded_read(None, 0, 0, 0, 1, None, None, 0, 0, 0, None) == ta.EINVAL
    assert L.topk_attn_coded_decode(None, 0, None, 0, 1, None, None, None) == ta.EINVAL
    assert L.topk_attn_coded_prompt(None, 0, 0, None, 1, 0, 1, None, None, None) == ta.EINVAL
    assert L.topk_attn_coded_reset(None, 0, 0, None) == ta.EINVAL
    assert L.topk_attn_coded_destroy(None) == ta.EINVAL
    assert L.topk_attn_coded_create(None, None) == ta.EINVAL
    assert L.topk_attn_coded_length(None, 0, 0) == -1


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")
@pytest.mark.parametrize("source,least", [("coded_decode.hip", 500), ("prompt.hip", 500), ("coded_prompt.hip", 1000)])
def test_no_mfma_result_is_read_early(tmp_path, source, least):
    out = str(tmp_path / "kernels.s")
    subprocess.check_call([hip_build.HIPCC, *hip_build.FLAGS, *hip_build.SOURCE_FLAGS.get(source, []), "--offload-device-only", "-S",
                           os.path.join(hip_build.CSRC, source), "-o", out], stderr=subprocess.DEVNULL)
    assert open(out).read().count("v_mfma") > least
    assert not isa_check.check(out)


@pytest.mark.skipif(not os.path.exists(hip_build.HIPCC), reason="hipcc not installed")
def test_host_side_under_asan_and_ubsan(tmp_path):
    """api_coded.hip and api_prompt.hip with sanitized host code, linked with stand-ins for the kernel launchers: refusals, calls that end at a missing device, and the
    launch plans of random shapes, held against the room there is for them."""
    import test_sanitizers_cpu as san
    host = [x for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all") for x in ("-Xarch_host", f)]
    common = [hip_build.HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", *host, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
    objs = []
    for src in (os.path.join(hip_build.CSRC, "api_coded.hip"), os.path.join(hip_build.CSRC, "api_prompt.hip"), os.path.join(ROOT, "tests", "sanitize_coded_driver.hip")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.check_call([*common, "-c", src, "-o", objs[-1]], stderr=subprocess.DEVNULL)
    exe = str(tmp_path / "coded_san")
    subprocess.check_call([hip_build.HIPCC, "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", *objs, "-o", exe],
                          stderr=subprocess.DEVNULL)
    env = dict(san.ENV, ASAN_OPTIONS=san.ENV["ASAN_OPTIONS"] + ":protect_shadow_gap=0",
               LSAN_OPTIONS="suppressions=" + os.path.join(ROOT, "tests", "sanitize_lsan.supp") + ":print_suppressions=0",
               HIP_VISIBLE_DEVICES="", ROCR_VISIBLE_DEVICES="")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, f"sanitizer run failed ({r.returncode}):\n{r.stdout[-2000:]}\n{r.stderr[-4000:]}"
    assert "runtime error" not in r.stderr and "ERROR: AddressSanitizer" not in r.stderr, r.stderr[-4000:]
    assert "coded driver: all checks passed" in r.stdout
