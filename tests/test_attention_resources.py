"""Compile-time resource checks of the attention and paged-cache kernels (no GPU needed):
what their comments count on in registers, LDS and waves a SIMD."""

import pytest

from test_kernel_resources import _resources


@pytest.mark.parametrize("kernel,scratch,waves", [
    # the loops of the rows kernel of 128 channels need all 256 registers; what spills is
    # outside them
    ("attention_rows_kernelINS0_8Bf16TileILi128E", 60, 2),
    ("attention_rows_kernelINS0_8Bf16TileILi64E", 0, 2),
    ("attention_rows_kernelINS0_7F32TileILi128E", 0, 2),
    ("attention_rows_kernelINS0_7F32TileILi64E", 0, 3),
    ("attention_keys_kernelINS0_8Bf16TileILi128E", 0, 1),
    ("attention_keys_kernelINS0_8Bf16TileILi64E", 0, 1),
    ("attention_keys_kernelINS0_7F32TileILi128E", 0, 1),
    ("attention_keys_kernelINS0_7F32TileILi64E", 0, 1),
])
def test_dense_attention(kernel, scratch, waves, tmp_path):
    r = _resources("attention.hip", kernel, tmp_path)
    assert r["ScratchSize"] <= scratch, r
    assert r["Occupancy"] >= waves, r
    assert r["LDS Size"] <= 160 * 1024, r


@pytest.mark.parametrize("kernel", ["paged_attention_kernelILi128ELb0", "paged_attention_kernelILi128ELb1",
                                    "paged_attention_kernelILi64ELb0", "paged_attention_kernelILi64ELb1"])
def test_paged_attention_runs_two_workgroups_a_cu(kernel, tmp_path):
    r = _resources("paged.hip", kernel, tmp_path)
    assert r["ScratchSize"] == 0, r
    assert r["Occupancy"] >= 2, r
    assert r["LDS Size"] <= 80 * 1024, r


def test_rows_in_and_out(tmp_path):
    for kernel in ("paged_append_kernel", "paged_read_kernel"):
        assert _resources("paged.hip", kernel, tmp_path)["ScratchSize"] == 0
