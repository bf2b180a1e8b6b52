"""Among how many CTAs the backward pass of the layer norm deals its rows out, which shows in its workspace: two sums a column for each."""
import ctypes as C

import pytest

from paper_2510_11400_b200 import api, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.lib()


@pytest.mark.parametrize("dtype,most", [(api.FH_F32, 14336), (api.FH_BF16, 12288)])
def test_as_many_as_fit_the_device_at_once(lib, dtype, most):
    """Long rows hold their sums in shared memory, columns rounded up to 512 vectors of 16 bytes (2048 and 4096 columns): two CTAs to an SM
    up to 14336 columns, 112 KB, one beyond."""
    for cols in (4097, 8193, 10241, 12288, most - 1, most, most + 1, 13000, 14336, 14337, 20000, 28672):
        wide = 2048 if dtype == api.FH_F32 else 4096
        if cols <= 1024 * (wide // 512):
            continue
        parts = 296 if -(-cols // wide) * wide <= 14336 else 148
        assert (parts == 296) == (cols <= most)
        assert lib.fh_layer_norm_work_bytes(C.byref(api.norm_desc(10 ** 6, cols, dtype))) == parts * 2 * cols * 4, cols
        assert lib.fh_layer_norm_work_bytes(C.byref(api.norm_desc(100, cols, dtype))) == 100 * 2 * cols * 4, cols
