"""A layer that routes by scores carries out its other options or refuses them (host only: no call goes through)."""
import dataclasses

import pytest
import torch

from paper_2607_05116_amd import capi
from test_scores_layer_refusals import CFG, _layer


@pytest.fixture
def calls(monkeypatch):
    made = []
    for name in ("cap_route_scores", "cap_route_prune", "cap_route_prune_naive", "cap_router_route_prune", "cap_route_layout",
                 "cap_dispatch_layout", "cap_coactivation"):
        monkeypatch.setattr(capi, name, lambda *a, _n=name, **k: made.append((_n, a)))
    return made


def test_expert_level_pruning_by_scores_is_refused(calls):
    layer = _layer()
    layer.naive = True
    layer.route()
    layer.set_scores()
    for call in (layer.route, layer.front, lambda: layer.router_route(torch.zeros(16, 256), torch.zeros(64, 16))):
        with pytest.raises(ValueError):
            call()
    assert [n for n, _ in calls] == ["cap_route_prune_naive"]
    layer.naive = False
    layer.route()
    layer.set_scores(None)
    layer.naive = True
    layer.route()
    assert [n for n, _ in calls] == ["cap_route_prune_naive", "cap_route_scores", "cap_route_prune_naive"]


def test_the_fused_front_end_by_scores_is_refused(calls):
    layer = _layer()
    layer.route_layout()
    layer.set_scores()
    with pytest.raises(ValueError):
        layer.route_layout()
    layer.front()
    assert [n for n, _ in calls] == ["cap_route_layout", "cap_route_scores", "cap_dispatch_layout", "cap_coactivation"]


def test_the_router_product_by_scores(calls):
    layer, w_gate = _layer(), torch.zeros(CFG.E, CFG.d)
    layer.router_route(w_gate)
    layer.set_scores()
    with pytest.raises(ValueError):
        layer.router_route(w_gate)
    logits = torch.zeros(CFG.T, CFG.E)
    layer.router_route(w_gate, logits)
    assert [n for n, _ in calls] == ["cap_router_route_prune", "cap_router_route_prune", "cap_route_scores"]
    assert calls[2][1][1] is logits and calls[1][1][-2] is logits


@pytest.mark.gpu
def test_the_router_product_and_scores_against_both_calls():
    from paper_2607_05116_amd.layer import DeviceLayer
    from workloads import generator as gen
    cfg = dataclasses.replace(CFG, E=32)               # the router's product takes 17 experts at least
    layer = DeviceLayer(cfg, gen.logits(cfg), gen.activations(cfg), *gen.sequential_placement(cfg), 0.1)
    g = torch.Generator(device="cuda").manual_seed(1)
    w_gate = (torch.randn((cfg.E, cfg.d), generator=g, device="cuda") / 16).to(torch.bfloat16)
    logits = torch.empty((cfg.T, cfg.E), device="cuda")
    layer.router_route(w_gate, logits)
    layer.logits.copy_(logits)
    layer.set_scores("sigmoid", n_groups=4, topk_groups=2, group_top=2, scale=2.5)
    layer.route()
    want = [t.clone() for t in (layer.idx, layer.w, layer.keep, layer.mask)]
    for t in (layer.idx, layer.w, layer.keep, layer.mask):
        t.zero_()
    layer.router_route(w_gate, logits)
    assert all(torch.equal(a, b) for a, b in zip(want, (layer.idx, layer.w, layer.keep, layer.mask)))
