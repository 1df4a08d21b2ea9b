"""What the compiler gave the kernels of the operators in 8 bits (no GPU)."""
import os

import pytest

import paper_2601_07396_amd as pkg
from test_kernel_resources import _kernels


@pytest.mark.parametrize("kernel,least", [("matmul8_shared_kernel", 21), ("matmul8_tile_kernel", 36), ("matmul8_finish_kernel", 1), ("rms_norm8_rows_kernel", 48),
                                          ("rms_norm8_long_kernel", 4), ("quantize_rows_kernel", 2), ("quantize_blocks_kernel", 2)])
def test_no_scratch(kernel, least):
    """Rows, sums and operands stay in registers."""
    if not os.path.exists(pkg.lib_path()):
        pytest.skip("the library is not built")
    found = {n: k[".private_segment_fixed_size"] for n, k in _kernels(pkg.lib_path()).items() if kernel in n}
    assert len(found) >= least
    assert {n: size for n, size in found.items() if size} == {}
