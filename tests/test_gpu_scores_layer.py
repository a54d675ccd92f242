"""Routing by scores and the experts in 8-bit floating point as a layer and its training use them together
(paper_2607_05116_amd.layer, .training), in graphs and on several streams."""
import numpy as np
import pytest
import torch

import scores_reference as ref
from workloads import generator as gen

pytestmark = pytest.mark.gpu

CODES = ref.code_values()
CFG = gen.Config("scores", T=512, d=256, E=32, k=4, inter=128, R=4, ranks_per_node=2, n_clusters=4, zipf_s=1.1, dtype="bf16",
                 trace_tokens=512)
OPT = dict(kind="sigmoid", n_groups=8, topk_groups=3, group_top=2, normalise=True, scale=2.5)
P = 0.1


@pytest.fixture(scope="module")
def capi():
    from paper_2607_05116_amd import capi as c
    return c


def _layer(cfg=CFG, fp8=True, masked=False):
    from paper_2607_05116_amd.layer import DeviceLayer
    er, el = gen.sequential_placement(cfg)
    layer = DeviceLayer(cfg, gen.logits(cfg), gen.activations(cfg), er, el, P)
    for rank in range(cfg.R):
        ws = [gen.expert_weights(cfg, e) for e in range(cfg.E) if er[e] == rank]
        layer.set_rank_weights(rank, *(np.stack([w[i] for w in ws]) for i in range(3)))
    bias = torch.linspace(-0.2, 0.2, cfg.E, device="cuda")
    mask = (torch.arange(cfg.T, device="cuda") % 11 != 0) if masked else None
    layer.set_scores(bias=bias, token_mask=mask, **OPT)
    layer.set_fp8(fp8)
    return layer, np.asarray(er), bias.cpu().numpy(), None if mask is None else mask.cpu().numpy()


def _values(q, scale, block_rows):
    v = CODES[q.view(torch.uint8).cpu().numpy()]
    return v * scale.cpu().numpy().astype(np.float64).repeat(block_rows, -2)[..., :v.shape[-2], :].repeat(128, -1)


@pytest.mark.parametrize("masked", [False, True])
def test_layer_against_64_bits(masked):
    layer, er, bias, mask = _layer(masked=masked)
    cfg = CFG
    layer.front()
    for rank in range(cfg.R):
        layer.row_source(rank)
        layer.quantise_x()
        layer.ffn_fp8(rank)
        layer.dest_reduce(rank)
    layer.src_reduce(1)
    torch.cuda.synchronize()
    idx, w, keep, dev_mask, close = ref.route(gen.logits(cfg), cfg.k, er, cfg.R, cfg.ranks_per_node, P, 5.0, bias=bias, token_mask=mask, **OPT)
    assert not close.any()
    assert np.array_equal(layer.host("idx"), idx) and np.array_equal(layer.host("keep"), keep)
    assert np.array_equal(layer.host("mask").view(np.uint64), dev_mask)
    assert int(layer.host("expert_counts").sum()) == int(keep.sum())
    x = _values(layer.x8, layer.x8_scale, 1)
    want_x = gen.bf16_bits_to_f32(gen.activations(cfg)).astype(np.float64)
    q, s = ref.quantise(want_x, 1)
    assert np.array_equal(x, q * s.repeat(128, 1))
    y = np.zeros((cfg.tokens_per_rank, cfg.d))
    experts = {}
    for e in range(cfg.E):
        q8 = layer.weights_fp8[int(er[e])]
        at = e % cfg.E_loc
        experts[e] = [_values(q8[2 * i][at], q8[2 * i + 1][at], 128) for i in range(3)]
    t0 = cfg.tokens_per_rank
    for t in range(t0, 2 * t0):
        for s_ in range(cfg.k):
            if not keep[t, s_]:
                continue
            w1, w3, w2 = experts[int(idx[t, s_])]
            g = w1 @ x[t]
            h, hs = ref.quantise((g / (1 + np.exp(-g)) * (w3 @ x[t]))[None], 1)
            y[t - t0] += w[t, s_] * (w2 @ (h * hs.repeat(128, 1))[0])
    got = gen.bf16_bits_to_f32(layer.host("y")).astype(np.float64)
    # three roundings to bf16 (the expert's row, the rank's sum, the token's sum), each 2^-8 of a value at most; codes
    # of H that round to a neighbour are few
    assert np.linalg.norm(got - y) <= 3 * 2.0 ** -8 * np.linalg.norm(y)
    if masked:
        assert (got[~mask[t0:2 * t0]] == 0).all()


def test_step_graph_replays_the_eager_step():
    layer, *_ = _layer()
    layer.step(0)
    torch.cuda.synchronize()
    eager = {n: layer.host(n) for n in ("idx", "w", "keep", "y", "slot_pos")}
    g = layer.capture_step(0)
    other = torch.randn(256, 256, device="cuda")
    for i in range(4):
        layer.y.zero_()
        layer.w.zero_()
        layer.Y.fill_(3.0)
        other = other @ other / 16
        g.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(layer.host(n), v) for n, v in eager.items()), i
    side = torch.cuda.Stream()
    layer.y.zero_()
    layer.step(0, side=side)
    torch.cuda.synchronize()
    assert all(np.array_equal(layer.host(n), v) for n, v in eager.items())


def test_back_to_the_other_path():
    """Scores and 8 bits off again: the layer's own path, bit for bit."""
    layer, er, *_ = _layer()
    layer.step(0)
    layer.set_scores(None)
    layer.set_fp8(False)
    layer.step(0)
    from paper_2607_05116_amd.layer import DeviceLayer
    plain = DeviceLayer(CFG, gen.logits(CFG), gen.activations(CFG), *gen.sequential_placement(CFG), P)
    plain.weights = layer.weights
    plain.step(0)
    torch.cuda.synchronize()
    n = int(plain.host("recv_offsets")[1])
    for name in ("idx", "w", "keep", "mask", "slot_pos"):
        assert np.array_equal(layer.host(name), plain.host(name))
    assert np.array_equal(layer.host("parts")[:n], plain.host("parts")[:n])


def test_new_weights_are_quantised_again():
    layer, *_ = _layer()
    layer.step(0)
    before = layer.weights_fp8[0][0].view(torch.uint8).clone()
    w1, w3, w2 = (v.view(torch.int16).cpu().numpy().view(np.uint16) for v in layer.weights[0])
    layer.set_rank_weights(0, w1[::-1].copy(), w3, w2)
    torch.cuda.synchronize()
    assert torch.equal(layer.weights_fp8[0][0].view(torch.uint8), before.flip(0))


@pytest.mark.parametrize("rows,E", [(24, 8), (700, 3), (9000, 4)])
def test_feed_forwards_on_two_streams(capi, rows, E):
    """Two calls at once, each with its own buffers, and the same calls one after the other; then both in one graph."""
    d, inter = 384, 256
    g = torch.Generator(device="cuda").manual_seed(3)

    def problem(seed):
        r = lambda *s: torch.randint(0x20, 0x48, s, generator=g, device="cuda", dtype=torch.uint8)
        f = lambda *s: torch.rand(s, generator=g, device="cuda") / 8
        offs = torch.linspace(0, rows, E + 1, device="cuda").to(torch.int32)
        need = capi.cap_workspace_size(capi.CAP_OP_EXPERT_FFN_FP8, None, d, inter, rows)
        return [E, d, inter, rows, r(rows, d), f(rows, d // 128), rows, None, offs, r(E, inter, d), f(E, 2, 3), r(E, inter, d), f(E, 2, 3),
                r(E, d, inter), f(E, 3, 2), torch.zeros((rows, d), dtype=torch.bfloat16, device="cuda"),
                torch.empty(need, dtype=torch.uint8, device="cuda")]
    a, b = problem(1), problem(2)
    for p in (a, b):
        capi.cap_expert_ffn_fp8(*p)
    torch.cuda.synchronize()
    want = [p[15].clone() for p in (a, b)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for p in (a, b):
            p[15].zero_()
        torch.cuda.synchronize()
        for p, s in zip((a, b), streams):
            capi.cap_expert_ffn_fp8(*p, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(a[15], want[0]) and torch.equal(b[15], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for p in (a, b):
            capi.cap_expert_ffn_fp8(*p)
    for _ in range(3):
        for p in (a, b):
            p[15].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a[15], want[0]) and torch.equal(b[15], want[1])


# ------------------------------------------------------------------ training
T, D, E, K, SEQS = 1024, 256, 32, 4, 4
OFFSETS = [16, 100, 100, 700, T - 8]


def _trainer(**kw):
    from paper_2607_05116_amd.training import RouterTrainer, Scores
    g = torch.Generator("cuda").manual_seed(5)
    e = torch.arange(E, dtype=torch.int32)
    w = torch.randn((E, D), generator=g, device="cuda") / 16
    return RouterTrainer(T, D, E, K, 4, 4, e // 8, e % 8, w, p=P, n_seq=SEQS, scores=Scores(**kw), lr=1e-2)


def _batch(seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.randn((T, D), generator=g, device="cuda").to(torch.bfloat16)


@pytest.mark.parametrize("kind,normalise", [("sigmoid", True), ("sigmoid", False), ("softmax", False)])
def test_training_step_by_scores(kind, normalise):
    from tests import training_reference as R
    t = _trainer(kind=kind, n_groups=4, topk_groups=2, group_top=2, normalise=normalise, scale=2.0, bias_speed=0.05)
    t.bias.copy_(torch.linspace(-0.1, 0.1, E))
    bias0 = t.bias.cpu().numpy()
    x, offs = _batch(1), torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
    mask = (torch.arange(T, device="cuda") % 13 != 0)
    d_gates = torch.randn((T, K), generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    t.step(x, d_gates, offs, mask)
    torch.cuda.synchronize()
    logits, idx, keep, gates = (v.cpu().numpy() for v in (t.logits, t.idx, t.keep, t.gates))
    m = mask.cpu().numpy()
    r = ref.route(logits, K, np.arange(E) // 8, 4, 4, P, 5.0, kind=kind, n_groups=4, topk_groups=2, group_top=2, normalise=normalise,
                  scale=2.0, bias=bias0, token_mask=m)
    assert np.array_equal(idx, r[0]) and np.array_equal(keep[~r[4]], r[2][~r[4]])
    want = R.balance64(logits, idx, keep, m, OFFSETS, t.balance_coef, t.z_coef)
    assert np.array_equal(t.counts.cpu().numpy(), want["counts"])
    counted = m & (np.arange(T) >= OFFSETS[0]) & (np.arange(T) < OFFSETS[-1])
    losses = R.grad64(logits, idx, keep, gates, np.zeros((T, K)), m, OFFSETS, t.balance_coef, t.z_coef)
    d = losses + ref.grad(logits.astype(np.float64), idx, keep * counted[:, None], d_gates.cpu().numpy().astype(np.float64), kind, normalise, 2.0)
    got = t.d_logits.double().cpu().numpy()
    assert (got[~counted] == 0).all()
    # rounded to bf16 once; the terms' fp32 arithmetic is far below that
    assert np.linalg.norm(got - d) <= 2.0 ** -8 * np.linalg.norm(d)
    loads = want["counts"].sum(0)
    assert np.allclose(t.bias.cpu().numpy() - bias0, 0.05 * np.sign(loads.mean() - loads), atol=1e-6)


def test_training_step_in_a_graph():
    runs = []
    for graphed in (False, True):
        t = _trainer(kind="sigmoid", n_groups=4, topk_groups=2, group_top=2, bias_speed=0.01)
        x, offs = _batch(2).clone(), torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
        d_gates = 0.1 * torch.randn((T, K), generator=torch.Generator("cuda").manual_seed(8), device="cuda")
        if graphed:
            w, wb, mo = t.w.clone(), t.w_bf16.clone(), t.opt.momentum.clone()
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                t.step(x, d_gates, offs)
            torch.cuda.current_stream().wait_stream(s)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                t.step(x, d_gates, offs)
            t.w.copy_(w)
            t.w_bf16.copy_(wb)
            t.opt.momentum.copy_(mo)
            t.bias.zero_()
        out = []
        for i in range(4):
            x.copy_(_batch(10 + i))
            g.replay() if graphed else t.step(x, d_gates, offs)
            torch.cuda.synchronize()
            out += [t.w.cpu(), t.bias.cpu(), t.d_logits.cpu(), t.loss.cpu()]
        runs.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_a_given_stream_takes_all_of_a_step_by_scores():
    # the stream is busy when the calls are made: whatever ran on another would read what is not written yet
    a, b = (_trainer(kind="sigmoid", n_groups=4, topk_groups=2, scale=2.0) for _ in range(2))
    offs, x = torch.tensor(OFFSETS, dtype=torch.int32, device="cuda"), _batch(4)
    d_gates = torch.randn((T, K), generator=torch.Generator("cuda").manual_seed(9), device="cuda")
    a.step(x, d_gates, offs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    b.forward(x, offs, stream=side)
    b.backward(x, d_gates, offs, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a.d_logits, b.d_logits) and torch.equal(a.d_w, b.d_w)
