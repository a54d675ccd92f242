"""cap_product_fp8 over hundreds of millions of rows, each taken from one of a few: every row has its source's result."""
import numpy as np
import pytest
import torch

import scores_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,out", [(1, torch.float32), (8, torch.bfloat16), (30, torch.bfloat16)])
def test_rows_by_the_hundred_million(n, out):
    from paper_2607_05116_amd import capi
    rows, sources, k = 2 ** 28 + 3, 5, 128
    g = torch.Generator(device="cuda").manual_seed(n)
    code = lambda *s: torch.randint(0x20, 0x48, s, generator=g, device="cuda", dtype=torch.uint8)
    x, w = code(sources, k), code(2, n, k)
    sx, sw = torch.rand((sources, 1), generator=g, device="cuda"), torch.rand((2, 1, 1), generator=g, device="cuda")
    cut = rows // 3
    offsets = torch.tensor([0, cut, rows], dtype=torch.int32, device="cuda")
    row_src = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(sources)
    y = torch.full((rows + 1, n), 7.0, dtype=out, device="cuda")
    ws = torch.empty(capi.cap_workspace_size(capi.CAP_OP_PRODUCT_FP8, None, n, k, rows), dtype=torch.uint8, device="cuda")
    dt = capi.CAP_DTYPE_F32 if out == torch.float32 else capi.CAP_DTYPE_BF16
    capi.cap_product_fp8(dt, 2, n, k, rows, x, sx, sources, row_src, offsets, w, sw, y, ws)
    torch.cuda.synchronize()
    assert (y[rows] == 7.0).all()
    values = ref.code_values()
    vx, vw = values[x.cpu().numpy()] * sx.cpu().numpy().astype(np.float64), values[w.cpu().numpy()]
    for e, (lo, hi) in enumerate(((0, cut), (cut, rows))):
        first = -lo % sources                           # the first row of source 0
        table = y[lo + first:lo + first + sources]
        want = vx @ vw[e].T * float(sw[e])
        # all terms are positive: 128 additions of 2^-24 each and the scales', the 8-bit instructions' 2^-13 of the largest
        # of eight products for each of the other seven, and the result's rounding
        assert np.all(np.abs(table.double().cpu().numpy() - want) <= (132 * 2.0 ** -24 if out == torch.float32 else 7 * 2.0 ** -13 + 2.0 ** -8) * want)
        for at in range(lo, hi, 2 ** 24):
            part = slice(at, min(at + 2 ** 24, hi))
            assert torch.equal(y[part], table[row_src[part].long()]), (e, at)
