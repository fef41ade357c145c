"""How easyspec_attn_weights cuts contexts, as its workspace shows it: a maximum and a sum, 8 bytes, per layer, query row and chunk."""
import pytest

import paper_2502_02493_amd as es


def chunks(heads, hd, n, lens, dtype="bf16"):
    """Chunks of all contexts, of sequences with as many tokens each."""
    Hq, H = heads
    layout = es.easyspec_kv_layout(1, len(lens), H, max(lens), hd, es.EASYSPEC_DTYPE_BF16 if dtype == "bf16" else es.EASYSPEC_DTYPE_F32)
    got = es.easyspec_attn_weights_workspace_bytes(layout, [n] * len(lens), lens, Hq)
    per_chunk = 8 * n * Hq
    assert got % per_chunk == 0
    return got // per_chunk


@pytest.mark.parametrize("heads,hd,n,lens,want", [
    ((8, 1), 128, 4, [32768], 256),          # 32 rows, 64 or 128 slots to a workgroup: one to a CU
    ((16, 8), 128, 12, [4096], 32),
    ((32, 8), 128, 6, [8192], 32),
    ((28, 4), 128, 4, [24576], 64),
    ((32, 8), 128, 6, [16384], 32),          # 256 slots with two to a CU: not more than two rounds
    ((32, 8), 128, 6, [20480], 64),          # 320: two to a CU
    ((32, 8), 128, 5, [2048] * 16, 64),
    ((32, 8), 128, 6, [4096, 8192, 16384, 32768], 4 + 8 + 16 + 32),      # chunks of 1024
    ((32, 8), 64, 6, [32768], 64),
    ((32, 8), 128, 4, [32768], 32),          # one row tile, more than two, or fp32: one to a CU whatever the length
    ((32, 8), 128, 9, [32768], 32),
])
def test_two_workgroups_to_a_cu_only_for_long_chunks_of_two_row_tiles(heads, hd, n, lens, want):
    assert chunks(heads, hd, n, lens) == want


def test_fp32_has_one_workgroup_to_a_cu():
    assert chunks((32, 8), 128, 6, [32768], "fp32") == 32
