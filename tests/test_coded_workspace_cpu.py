"""Room that the 8-bit cache asks for beside its rows (no GPU)."""
import itertools

import pytest

from paper_2502_06766_amd import topk_attn as ta


@pytest.mark.parametrize("dtype", [ta.F32, ta.F16])
@pytest.mark.parametrize("d", [32, 128, 256])
def test_workspace_is_a_small_part_of_the_cache(dtype, d):
    """Partial sums of many short sequences and of long ones: beside 256 MB (two workgroups of 128 rows on each compute unit, and splits that fill the chip) a quarter of the storage
    (single rows of 64 that are held as they came)."""
    for seqs, heads, tokens in itertools.product((1, 64, 1024, 65535), (1, 8, 64), (1, 64, 1000, 65536, 1 << 20, 1 << 30)):
        cfg = ta.make_coded_config(1, seqs, 4 * heads, heads, d, tokens, dtype)
        kv, ws = ta.topk_attn_coded_kv_bytes(cfg), ta.topk_attn_coded_workspace_bytes(cfg)
        if seqs * heads > 1 << 22:
            assert kv == ws == 0
        else:
            assert 0 < ws <= kv / 4 + (256 << 20), (seqs, heads, tokens, kv, ws)
