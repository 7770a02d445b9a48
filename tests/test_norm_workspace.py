"""The norm's workspace is what its documentation says: 4 bytes a column and thread block, of at most 1184 blocks and no more than rows,
by rows, n and the size of the type."""
import pytest

from paper_2412_11810_b200 import binding as sb


@pytest.mark.parametrize("n", [1, 64, 512, 1000, 1024, 1536, 2048, 4096, 8192, 16384, 20000])
def test_blocks_of_the_backward_pass(n):
    for rows in (1, 2, 100, 1184, 5000, 32768, 1 << 22):
        sizes = {}
        for dtype in (0, 1, 2):
            for weight_dtype in {0, dtype}:
                size = sb.snn_rms_norm_workspace(sb.snn_rms_norm_args(rows, n, dtype, weight_dtype, 1e-6))
                assert 4 * n <= size <= (4 * n * min(rows, 148 * 8) + 255) // 256 * 256
                sizes.setdefault(dtype, set()).add(size)
        assert all(len(s) == 1 for s in sizes.values()) and sizes[1] == sizes[2]
