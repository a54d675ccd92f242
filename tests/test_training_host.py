"""Argument checks of the training operators (cap_balance_loss, cap_router_grad, cap_orthogonalise,
cap_muon_update): every refusal is decided on the host, before anything is launched."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def capi():
    from paper_2607_05116_amd import capi as c
    return c


BIG = 1 << 40


def _balance(capi, **over):
    a = dict(T=64, k=2, E=16, logits=0x1000, idx=0x2000, keep=0x3000, mask=None, offs=0x4000, n_seq=3, bc=0.01, zc=0.001,
             counts=0x5000, probs=0x6000, tokens=0x7000, loss=0x8000, ws=0x10000, nbytes=BIG)
    a.update(over)
    return capi._lib.cap_balance_loss(*a.values(), None)


@pytest.mark.parametrize("over", [dict(T=-1), dict(k=0), dict(k=9), dict(k=3, E=2), dict(E=0), dict(E=257), dict(n_seq=0),
                                  dict(T=2 ** 31 // 4, k=4), dict(n_seq=2 ** 27, E=256), dict(offs=None),
                                  dict(logits=None), dict(idx=None), dict(counts=None), dict(probs=None),
                                  dict(tokens=None), dict(loss=None), dict(bc=float("nan")), dict(zc=float("inf")),
                                  dict(logits=0x1002), dict(idx=0x2001), dict(offs=0x4002), dict(counts=0x5001),
                                  dict(probs=0x6002), dict(tokens=0x7002), dict(loss=0x8001)])
def test_balance_loss_refuses(capi, over):
    if "T" in over and over["T"] > 0:
        over = dict(over, k=8)
    assert _balance(capi, **over) == capi.CAP_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(ws=None), dict(ws=0x10010), dict(nbytes=0)])
def test_balance_loss_refuses_workspace(capi, over):
    assert _balance(capi, **over) == capi.CAP_ERR_WORKSPACE
    topo = capi.Topology(E=16, T=64)
    need = capi.cap_workspace_size(capi.CAP_OP_BALANCE_LOSS, topo, max_rows=3)
    assert need > 0 and _balance(capi, nbytes=need - 1) == capi.CAP_ERR_WORKSPACE


def _grad(capi, **over):
    a = dict(T=64, k=2, E=16, logits=0x1000, idx=0x2000, keep=0x3000, w=0x9000, d_w=0xA000, mask=None, offs=0x4000,
             n_seq=3, counts=0x5000, tokens=0x7000, bc=0.01, zc=0.001, d_loss=None, dtype=0, out=0xB000)
    a.update(over)
    return capi._lib.cap_router_grad(*a.values(), None)


@pytest.mark.parametrize("over", [dict(T=-1), dict(k=0), dict(k=9), dict(E=257), dict(n_seq=0), dict(offs=None),
                                  dict(logits=None), dict(out=None), dict(idx=None), dict(w=None), dict(counts=None),
                                  dict(tokens=None), dict(bc=float("inf")), dict(zc=float("nan")), dict(out=0xB002),
                                  dict(out=0xB001, dtype=1), dict(d_loss=0x3), dict(w=0x9002), dict(d_w=0xA001)])
def test_router_grad_refuses(capi, over):
    assert _grad(capi, **over) == capi.CAP_ERR_INVALID_ARG


def test_router_grad_other(capi):
    assert _grad(capi, dtype=2) == capi.CAP_ERR_UNSUPPORTED
    assert _grad(capi, T=0, logits=None, out=None) == capi.CAP_OK           # no token: nothing to do


def _orth(capi, **over):
    a = dict(dtype=0, batch=2, rows=8, cols=16, g=0x1000, steps=5, coef=None, eps=1e-7, out=0x2000, ws=0x10000, nbytes=BIG)
    a.update(over)
    return capi._lib.cap_orthogonalise(*a.values(), None)


def _muon(capi, **over):
    a = dict(dtype=0, batch=2, rows=8, cols=16, g=0x1000, mom=0x3000, mu=0.95, nesterov=1, steps=5, coef=None, eps=1e-7,
             out=0x2000, ws=0x10000, nbytes=BIG)
    a.update(over)
    return capi._lib.cap_muon_update(*a.values(), None)


@pytest.mark.parametrize("call", [_orth, _muon])
def test_orthogonalise_refuses(capi, call):
    bad = (ctypes.c_float * 15)(*([1.0] * 14 + [float("nan")]))
    for over in (dict(batch=-1), dict(rows=-1), dict(cols=-1), dict(steps=0), dict(steps=17), dict(eps=-1.0),
                 dict(eps=float("nan")), dict(eps=float("inf")), dict(coef=bad), dict(g=None), dict(out=None),
                 dict(g=0x1002), dict(dtype=1, g=0x1001), dict(out=0x2001)):
        assert call(capi, **over) == capi.CAP_ERR_INVALID_ARG, over
    for over in (dict(dtype=2), dict(rows=65537), dict(cols=65537), dict(batch=65536)):
        assert call(capi, **over) == capi.CAP_ERR_UNSUPPORTED, over
    need = capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=16, inter=8, max_rows=2)
    for over in (dict(ws=None), dict(ws=0x10080), dict(nbytes=need - 1)):
        assert call(capi, **over) == capi.CAP_ERR_WORKSPACE, over
    for over in (dict(batch=0), dict(rows=0), dict(cols=0)):                # nothing to do
        assert call(capi, **over) == capi.CAP_OK, over


def test_muon_refuses(capi):
    for over in (dict(mu=-0.1), dict(mu=1.0), dict(mu=float("nan")), dict(mom=None), dict(mom=0x3002)):
        assert _muon(capi, **over) == capi.CAP_ERR_INVALID_ARG, over


def test_binding_checks_coefficients(capi):
    with pytest.raises(ValueError):
        capi._coefficients([(1.0, 2.0, 3.0)], 2)
    assert capi._coefficients(None, 5) is None
    assert list(capi._coefficients([(1, 2, 3), (4, 5, 6)], 2)) == [1, 2, 3, 4, 5, 6]


def test_workspace_sizes(capi):
    topo = capi.Topology(E=16, T=64)
    size = lambda **k: capi.cap_workspace_size(capi.CAP_OP_BALANCE_LOSS, topo, **k)   # noqa: E731
    assert size(max_rows=0) == 0 and size(max_rows=1) > 0
    orth = lambda r, c, b: capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=c, inter=r, max_rows=b)  # noqa: E731
    assert orth(0, 4, 1) == 0 and orth(4, 0, 1) == 0 and orth(4, 4, 0) == 0
    assert orth(100, 700, 2) == orth(700, 100, 2) > 0
