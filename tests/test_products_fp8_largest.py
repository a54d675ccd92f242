"""The largest sizes that the header allows for cap_product_fp8 are not refused: without a GPU the call comes to its launch,
which fails there, and says so.  (Not run where there is a GPU: the pointers are none.)"""
import pytest
import torch

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the launch would run")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n", [1, 8, 30, 64, 128])
@pytest.mark.parametrize("kdim", [128, 8192])
@pytest.mark.parametrize("max_rows", [1, 2 ** 20, 2 ** 28, 2 ** 29 + 7, 2 ** 30 - 64, 2 ** 30 - 1])
def test_largest_rows_are_launched(max_rows, kdim, n, dtype):
    from paper_2607_05116_amd import capi
    if max_rows == 1 and n == 1:
        x_rows, row_src = 1, None
    else:
        x_rows, row_src = 5, 0x7000
    st = capi._lib.cap_product_fp8(dtype, 8, n, kdim, max_rows, 0x1000, 0x2000, x_rows, row_src, 0x3000, 0x4000, 0x5000, 0x6000, 0x10000,
                                   1 << 40, None)
    assert st == capi.CAP_ERR_HIP
