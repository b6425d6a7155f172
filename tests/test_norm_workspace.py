"""Workspace of the norm's backward pass (CPU only): a row of fp32 for each workgroup, one a
compute unit at most."""
import pytest

import paper_2604_01622_amd as ec


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d", [1, 63, 64, 1001, 2048, 4097, 8192, 16384])
def test_size(d, dtype):
    def size(rows):
        return ec.lib().ec_rms_norm_workspace_size(dtype, rows, d)

    align = 256
    assert 0 < size(1) <= d * 4 + align
    for rows in (255, 256, 257, 5000, 1 << 20, (1 << 31) - 1):
        assert 4 * d <= size(rows) <= 256 * d * 4 + align
    assert 256 * d * 4 <= size((1 << 31) - 1)
