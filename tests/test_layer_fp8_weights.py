"""When a layer's weights are in 8 bits: complete for every stream after set_fp8 and set_rank_weights, and never first made
in a captured graph."""
import numpy as np
import pytest
import torch

from paper_2607_05116_amd import capi
from test_scores_layer_refusals import CFG, _layer


def test_no_first_quantisation_in_a_capture(monkeypatch):
    made = []
    for name in ("cap_quantise_fp8", "cap_expert_ffn_fp8"):
        monkeypatch.setattr(capi, name, lambda *a, _n=name, **k: made.append(_n))
    layer = _layer()
    layer.set_fp8()
    layer.weights[0] = tuple(torch.zeros(4, 128, 256) for _ in range(2)) + (torch.zeros(4, 256, 128),)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    for call in (lambda: layer.ffn_fp8(0), lambda: layer.quantise_weights(0)):
        with pytest.raises(RuntimeError):
            call()
    assert not made and 0 not in layer.weights_fp8
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    layer.quantise_weights(0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    layer.quantise_weights(0)                           # into the buffers that are there
    layer.ffn_fp8(0)
    assert made == ["cap_quantise_fp8"] * 6 + ["cap_expert_ffn_fp8"]


def _on_gpu():
    from paper_2607_05116_amd.layer import DeviceLayer
    from workloads import generator as gen
    er, el = gen.sequential_placement(CFG)
    layer = DeviceLayer(CFG, gen.logits(CFG), gen.activations(CFG), er, el, 0.1)
    ws = [gen.expert_weights(CFG, e) for e in range(CFG.E) if er[e] == 0]
    return layer, [np.stack([w[i] for w in ws]) for i in range(3)]


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["weights first", "8 bits first", "by the first step", "again"])
def test_complete_for_other_streams(order):
    """The stream that quantises is busy: a copy made on another one right after holds the codes all the same."""
    layer, w = _on_gpu()
    busy, other = torch.cuda.Stream(), torch.cuda.Stream()
    if order == "weights first":
        layer.set_rank_weights(0, *w)
    elif order == "again":
        layer.set_rank_weights(0, *(v[::-1].copy() for v in w))
        layer.set_fp8()
    else:
        layer.set_fp8()
    if order == "by the first step":
        from paper_2607_05116_amd.layer import to_device_rows
        layer.weights[0] = tuple(to_device_rows(v, "bf16", "cuda") for v in w)
        layer.front()
        layer.row_source(0)
        layer.quantise_x()
    torch.cuda.synchronize()
    with torch.cuda.stream(busy):
        torch.cuda._sleep(50_000_000)
        if order == "weights first":
            layer.set_fp8()
        elif order == "by the first step":
            layer.ffn_fp8(0, busy)
        else:
            layer.set_rank_weights(0, *w)
    with torch.cuda.stream(other):
        got = [t.view(torch.uint8).clone() for t in layer.weights_fp8[0]]
    torch.cuda.synchronize()
    want = []
    for t in layer.weights[0]:
        q = torch.empty(t.shape, dtype=torch.float8_e4m3fn, device="cuda")
        s = torch.empty((t.shape[0], t.shape[1] // 128, t.shape[2] // 128), device="cuda")
        capi.cap_quantise_fp8(capi.CAP_DTYPE_BF16, *t.shape, 128, t, q, s)
        want += [q.view(torch.uint8), s.view(torch.uint8)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_a_graph_without_an_eager_step_before():
    layer, w = _on_gpu()
    layer.set_rank_weights(0, *w)
    layer.set_scores("sigmoid", n_groups=4, topk_groups=2, group_top=2)
    layer.set_fp8()
    codes = [t.data_ptr() for t in layer.weights_fp8[0]]
    graph = layer.capture_step(0, warmup=0)
    layer.step(0)                                       # before the first replay
    torch.cuda.synchronize()
    want = layer.y.clone()
    assert torch.isfinite(want).all() and want.abs().max() > 0
    for _ in range(3):
        layer.y.zero_()
        layer.Y.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.y, want)
    # new weights reach the captured step, in the same buffers
    layer.set_rank_weights(0, *(v[::-1].copy() for v in w))
    assert codes == [t.data_ptr() for t in layer.weights_fp8[0]]
    graph.replay()
    torch.cuda.synchronize()
    replayed = layer.y.clone()
    layer.step(0)
    torch.cuda.synchronize()
    assert torch.equal(layer.y, replayed) and not torch.equal(replayed, want)
