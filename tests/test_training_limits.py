"""The largest sizes that the router's losses take: accepted and refused on the host, before anything is launched."""
import pytest

from paper_2607_05116_amd import capi

BIG = 1 << 50


def _balance(T, S, nbytes):
    return capi._lib.cap_balance_loss(T, 1, 1, 0x1000, 0x2000, None, None, 0x4000, S, 0.1, 0.1, 0x5000, 0x6000, 0x7000, 0x8000,
                                      0x10000, nbytes, None)


def _grad(T, S):
    return capi._lib.cap_router_grad(T, 1, 1, 0x1000, 0x2000, None, None, None, None, 0x4000, S, 0x5000, 0x7000, 0.1, 0.1, None,
                                     5, 0xB000, None)


@pytest.mark.parametrize("T,S,ok", [(2 ** 31 - 4096, 3, True), (2 ** 31 - 4095, 3, False), (2 ** 31 - 1, 3, False),
                                    (64, 2 ** 30, True), (64, 2 ** 30 + 1, False), (64, 2 ** 31 - 1, False)])
def test_sizes(T, S, ok):
    # (an accepted size is refused for its workspace or type, which are looked at later)
    assert _balance(T, S, 0) == (capi.CAP_ERR_WORKSPACE if ok else capi.CAP_ERR_INVALID_ARG)
    assert _grad(T, S) == (capi.CAP_ERR_UNSUPPORTED if ok else capi.CAP_ERR_INVALID_ARG)
    if not ok:
        assert _balance(T, S, BIG) == capi.CAP_ERR_INVALID_ARG
    size = capi.cap_workspace_size(capi.CAP_OP_BALANCE_LOSS, capi.Topology(E=1, T=T), max_rows=S)
    assert (size > 0) == ok


@pytest.mark.parametrize("batch,rows,cols", [(65535, 16, 16), (65535, 64, 100), (4096, 128, 128), (64, 16, 65536), (1, 1, 65536)])
def test_workspace_of_small_matrices(batch, rows, cols):
    """Not more than 400 MB beside 64 bytes a value: the padding of small matrices is not paid for a whole batch."""
    got = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=cols, inter=rows, max_rows=batch)
    assert 0 < got <= (400 << 20) + 64 * batch * rows * cols
