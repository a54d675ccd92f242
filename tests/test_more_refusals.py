"""Argument checks of cap_route_scores, cap_route_scores_grad, cap_quantise_fp8, cap_product_fp8 and cap_expert_ffn_fp8:
every refusal is decided on the host, before anything is launched."""
import pytest


@pytest.fixture(scope="module")
def capi():
    from paper_2607_05116_amd import capi as c
    return c


BIG = 1 << 40


def _options(capi, **over):
    return capi.ScoreOptions(**{**dict(kind=1, n_groups=8, topk_groups=4, group_top=2, normalise=1, scale=2.5, bias=0x100), **over})


def _route(capi, options={}, topo={}, **over):
    t = capi.Topology(**{**dict(E=64, R=8, ranks_per_node=8, T=64, tokens_per_rank=8, k=6, expert_rank=0x1000, expert_local=0x2000,
                                inter_node_cost=5.0), **topo})
    a = {**dict(topo=t, logits=0x3000, options=_options(capi, **options), p=0.1, idx=0x4000, w=0x5000, keep=0x6000, mask=0x7000), **over}
    return capi._lib.cap_route_scores(*a.values(), None)


@pytest.mark.parametrize("over", [dict(options=dict(n_groups=0)), dict(options=dict(n_groups=7)), dict(options=dict(topk_groups=0)),
                                  dict(options=dict(topk_groups=9)), dict(options=dict(n_groups=32, topk_groups=2)),
                                  dict(options=dict(group_top=0)), dict(options=dict(group_top=3)), dict(options=dict(scale=0.0)),
                                  dict(options=dict(scale=float("nan"))), dict(options=dict(scale=float("inf"))),
                                  dict(options=dict(bias=0x101)), dict(options=dict(n_groups=128, topk_groups=128), topo=dict(E=128)),
                                  dict(topo=dict(k=9)), dict(topo=dict(E=60)), dict(topo=dict(T=63)), dict(topo=dict(expert_rank=None)),
                                  dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(logits=None), dict(logits=0x3002), dict(idx=None),
                                  dict(w=None), dict(w=0x5001), dict(keep=None), dict(mask=None), dict(mask=0x7004)])
def test_route_refuses(capi, over):
    assert _route(capi, **over) == capi.CAP_ERR_INVALID_ARG


def test_route_refuses_other(capi):
    assert _route(capi, options=dict(kind=2)) == capi.CAP_ERR_UNSUPPORTED
    t = capi.Topology(E=64, R=8, ranks_per_node=8, T=64, tokens_per_rank=8, k=6, expert_rank=1, expert_local=1, inter_node_cost=5.0)
    assert capi._lib.cap_route_scores(t, 0x3000, None, 0.1, 0x4000, 0x5000, 0x6000, 0x7000, None) == capi.CAP_ERR_INVALID_ARG


def _grad(capi, options={}, **over):
    a = dict(T=64, k=6, E=64, logits=0x1000, idx=0x2000, keep=0x3000, w=0x4000, d_w=0x5000, options=_options(capi, **options),
             d_add=None, dtype=0, out=0x6000)
    a.update(over)
    return capi._lib.cap_route_scores_grad(*a.values(), None)


@pytest.mark.parametrize("over", [dict(T=-1), dict(k=0), dict(k=9), dict(E=5), dict(E=257), dict(T=2 ** 31 // 6 + 1), dict(logits=None),
                                  dict(idx=None), dict(w=None), dict(d_w=None), dict(out=None), dict(logits=0x1001), dict(idx=0x2002),
                                  dict(w=0x4001), dict(d_w=0x5002), dict(d_add=0x7001), dict(out=0x6002), dict(out=0x6001, dtype=1),
                                  dict(options=dict(scale=-1.0)), dict(options=dict(kind=0, normalise=0), logits=None)])
def test_grad_refuses(capi, over):
    assert _grad(capi, **over) == capi.CAP_ERR_INVALID_ARG


def test_grad_other(capi):
    assert _grad(capi, dtype=2) == capi.CAP_ERR_UNSUPPORTED
    assert _grad(capi, options=dict(kind=7)) == capi.CAP_ERR_UNSUPPORTED
    assert _grad(capi, T=0, logits=None, idx=None, out=None) == capi.CAP_OK


def _quantise(capi, **over):
    a = dict(dtype=1, batch=2, rows=100, cols=256, block_rows=1, x=0x1000, q=0x2000, scale=0x3000)
    a.update(over)
    return capi._lib.cap_quantise_fp8(*a.values(), None)


@pytest.mark.parametrize("over", [dict(batch=-1), dict(rows=-1), dict(cols=-128), dict(block_rows=0), dict(block_rows=64), dict(x=None),
                                  dict(q=None), dict(scale=None), dict(x=0x1008), dict(q=0x2004), dict(scale=0x3002)])
def test_quantise_refuses(capi, over):
    assert _quantise(capi, **over) == capi.CAP_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(dtype=2), dict(cols=200), dict(cols=64), dict(batch=2 ** 12, rows=2 ** 17, cols=256),
                                  dict(batch=2 ** 31 - 1, rows=2 ** 31 - 1, cols=2 ** 30), dict(block_rows=128, batch=2 ** 24, rows=1, cols=128),
                                  dict(block_rows=128, batch=2 ** 23, rows=1, cols=256)])
def test_quantise_unsupported(capi, over):
    assert _quantise(capi, **over) == capi.CAP_ERR_UNSUPPORTED


@pytest.mark.parametrize("over", [dict(batch=0), dict(rows=0), dict(cols=0), dict(rows=0, x=None, q=None, scale=None)])
def test_quantise_nothing(capi, over):
    assert _quantise(capi, **over) == capi.CAP_OK


def _product(capi, **over):
    a = dict(dtype=1, E_loc=4, n=100, kdim=256, max_rows=50, x=0x1000, x_scale=0x2000, x_rows=50, row_src=None, offsets=0x3000, w=0x4000,
             w_scale=0x5000, y=0x6000, ws=0x10000, ws_bytes=BIG)
    a.update(over)
    return capi._lib.cap_product_fp8(*a.values(), None)


@pytest.mark.parametrize("over", [dict(E_loc=0), dict(E_loc=257), dict(n=0), dict(kdim=0), dict(max_rows=-1), dict(x=None), dict(x=0x1008),
                                  dict(x_scale=None), dict(x_scale=0x2002), dict(x_rows=0), dict(x_rows=49), dict(row_src=0x7001),
                                  dict(row_src=0x7000, x_rows=0), dict(offsets=None), dict(offsets=0x3001), dict(w=None), dict(w=0x4008),
                                  dict(w_scale=None), dict(w_scale=0x5001), dict(y=None), dict(y=0x6001), dict(y=0x6002, dtype=0)])
def test_product_refuses(capi, over):
    assert _product(capi, **over) == capi.CAP_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(dtype=2), dict(kdim=192), dict(kdim=64), dict(kdim=2 ** 15 + 128), dict(n=2 ** 25, kdim=128),
                                  dict(x_rows=2 ** 25, kdim=128), dict(max_rows=2 ** 30, x_rows=1, row_src=0x7000, n=2 ** 20, kdim=128)])
def test_product_unsupported(capi, over):
    assert _product(capi, **over) == capi.CAP_ERR_UNSUPPORTED


def test_product_nothing(capi):
    assert _product(capi, max_rows=0, x=None, x_scale=None, x_rows=0, w=None, w_scale=None, y=None, ws=None) == capi.CAP_OK


def test_product_workspace(capi):
    need = capi.cap_workspace_size(capi.CAP_OP_PRODUCT_FP8, None, d=100, inter=256, max_rows=50)
    if need:
        assert _product(capi, ws_bytes=need - 1) == _product(capi, ws=None) == _product(capi, ws=0x10010) == capi.CAP_ERR_WORKSPACE
    for bad in (dict(d=0, inter=256, max_rows=5), dict(d=5, inter=100, max_rows=5), dict(d=5, inter=256, max_rows=-1)):
        assert capi.cap_workspace_size(capi.CAP_OP_PRODUCT_FP8, None, **bad) == 0


def _ffn(capi, **over):
    a = dict(E_loc=4, d=256, inter=128, max_rows=50, x=0x1000, x_scale=0x2000, x_rows=50, row_src=None, offsets=0x3000, w1=0x4000, s1=0x4100,
             w3=0x5000, s3=0x5100, w2=0x6000, s2=0x6100, y=0x7000, ws=0x10000, ws_bytes=BIG)
    a.update(over)
    return capi._lib.cap_expert_ffn_fp8(*a.values(), None)


@pytest.mark.parametrize("over", [dict(E_loc=0), dict(E_loc=257), dict(d=0), dict(inter=-1), dict(max_rows=-1), dict(x=None), dict(x=0x1004),
                                  dict(x_scale=None), dict(x_rows=49), dict(row_src=0x8002), dict(offsets=None), dict(w1=None), dict(s1=None),
                                  dict(w3=None), dict(s3=None), dict(w2=None), dict(s2=None), dict(y=None), dict(w1=0x4008), dict(w3=0x5008),
                                  dict(w2=0x6004), dict(y=0x7008), dict(s1=0x4101), dict(s3=0x5102), dict(s2=0x6103)])
def test_ffn_refuses(capi, over):
    assert _ffn(capi, **over) == capi.CAP_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(d=200), dict(inter=192), dict(d=2 ** 15 + 128), dict(inter=2 ** 15 + 128),
                                  dict(x_rows=2 ** 24), dict(max_rows=2 ** 25, x_rows=10, row_src=0x8000)])
def test_ffn_unsupported(capi, over):
    assert _ffn(capi, **over) == capi.CAP_ERR_UNSUPPORTED


def test_ffn_workspace(capi):
    need = capi.cap_workspace_size(capi.CAP_OP_EXPERT_FFN_FP8, None, d=256, inter=128, max_rows=50)
    assert need >= 50 * 128 + 50 * 4
    for over in (dict(ws=None), dict(ws=0x10080), dict(ws_bytes=need - 1)):
        assert _ffn(capi, **over) == capi.CAP_ERR_WORKSPACE
    assert _ffn(capi, max_rows=0, x=None, x_scale=None, x_rows=0, ws=None, w1=None, y=None) == capi.CAP_OK


@pytest.mark.parametrize("T", [2 ** 29, 2 ** 31 - 8])
def test_more_tokens_than_a_launch_has_threads_for(capi, T):
    assert _route(capi, topo=dict(T=T, tokens_per_rank=T // 8, k=1)) == capi.CAP_ERR_UNSUPPORTED
    assert _grad(capi, T=T, k=1) == capi.CAP_ERR_UNSUPPORTED


@pytest.mark.parametrize("max_rows", [2 ** 30, 2 ** 31 - 1])
@pytest.mark.parametrize("n", [1, 8])
def test_more_rows_than_row_numbers_hold(capi, max_rows, n):
    assert _product(capi, max_rows=max_rows, x_rows=1, row_src=0x7000, n=n, kdim=128) == capi.CAP_ERR_UNSUPPORTED
    assert capi.cap_workspace_size(capi.CAP_OP_PRODUCT_FP8, None, n, 128, max_rows) == 0
