"""Compile-time resource checks of the kernels that weigh, choose, move and sample (no GPU
needed): what their comments count on in registers, LDS and waves a SIMD."""

import pytest

from test_kernel_resources import _resources


@pytest.mark.parametrize("source,kernel,scratch,waves,lds", [
    ("weights.hip", "weights_rows_kernelINS0_8RowsBf16ILi128EEELi2E", 0, 2, 80),
    ("weights.hip", "weights_rows_kernelINS0_8RowsBf16ILi128EEELi1E", 0, 2, 80),
    ("weights.hip", "weights_rows_kernelINS0_8RowsBf16ILi64EEELi2E", 0, 2, 80),
    ("weights.hip", "weights_rows_kernelINS0_8RowsBf16ILi64EEELi1E", 0, 2, 80),
    ("weights.hip", "weights_rows_kernelINS0_7RowsF32ILi64E", 0, 2, 80),
    # (fp32 keys and rows of 128 channels need more registers than there are)
    ("weights.hip", "weights_rows_kernelINS0_7RowsF32ILi128E", 128, 2, 80),
    ("weights.hip", "weights_few_kernelINS0_8RowsBf16ILi128E", 0, 2, 0),
    ("weights.hip", "weights_few_kernelINS0_8RowsBf16ILi64E", 0, 2, 0),
    ("weights.hip", "weights_few_kernelINS0_7RowsF32ILi128E", 0, 2, 0),
    ("weights.hip", "weights_few_kernelINS0_7RowsF32ILi64E", 0, 2, 0),
    ("weights.hip", "paged_weights_kernelILi128ELb0E", 0, 2, 80),
    ("weights.hip", "paged_weights_kernelILi128ELb1E", 0, 2, 80),
    ("weights.hip", "paged_weights_kernelILi64ELb0E", 0, 2, 80),
    ("weights.hip", "paged_weights_kernelILi64ELb1E", 0, 2, 80),
    ("evict.hip", "evict_select_kernelILi4E", 0, 4, 32),
    ("evict.hip", "evict_select_kernelILi16E", 0, 4, 32),
    ("evict.hip", "evict_rows_kernel", 0, 4, 8),
    ("evict.hip", "paged_evict_kernelILi128E", 0, 4, 8),
    ("evict.hip", "paged_evict_kernelILi64E", 0, 4, 8),
    ("sample.hip", "sample_kernelIt", 0, 4, 160),
    ("sample.hip", "sample_kernelIf", 0, 4, 160),
])
def test_resources(source, kernel, scratch, waves, lds, tmp_path):
    r = _resources(source, kernel, tmp_path)
    assert r["ScratchSize"] <= scratch, r
    assert r["Occupancy"] >= waves, r
    assert r["LDS Size"] <= lds * 1024, r
