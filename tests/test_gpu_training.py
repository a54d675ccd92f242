"""The training step that runs the operators together (paper_2607_05116_amd.training)."""
import numpy as np
import pytest

from tests import training_reference as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2607_05116_amd.training import Muon, RouterTrainer  # noqa: E402

T, D, E, K, RANKS, SEQS = 1024, 256, 32, 4, 4, 4


def _trainer(**kw):
    g = torch.Generator("cuda").manual_seed(5)
    e = torch.arange(E, dtype=torch.int32)
    w = torch.randn((E, D), generator=g, device="cuda") / 16
    return RouterTrainer(T, D, E, K, RANKS, RANKS, e // (E // RANKS), e % (E // RANKS), w, p=0.1, n_seq=SEQS, **kw)


def _batch(seed):
    g = torch.Generator("cuda").manual_seed(seed)
    common = torch.randn((1, D), generator=torch.Generator("cuda").manual_seed(99), device="cuda")
    return (torch.randn((T, D), generator=g, device="cuda") + 1.5 * common).to(torch.bfloat16)


OFFSETS = [0, 100, 100, 700, T]


def test_one_step_against_64_bits():
    t = _trainer(lr=1e-2)
    x, offs = _batch(1), torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
    d_gates = torch.randn((T, K), generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    w0 = t.w.double().cpu().numpy()[0]
    t.step(x, d_gates, offs)
    torch.cuda.synchronize()
    logits, idx, keep, gates = (v.cpu().numpy() for v in (t.logits, t.idx, t.keep, t.gates))
    ref = R.balance64(logits, idx, keep, None, OFFSETS, t.balance_coef, t.z_coef)
    assert np.array_equal(t.counts.cpu().numpy(), ref["counts"])
    assert np.allclose(t.loss.cpu().numpy(), ref["loss"], rtol=1e-5)
    d = R.grad64(logits, idx, keep, gates, d_gates.cpu().numpy(), None, OFFSETS, t.balance_coef, t.z_coef)
    dw = d.T @ x.double().cpu().numpy()
    # two roundings to bf16 (the logits' gradient, its product with x)
    got = t.d_w.double().cpu().numpy()[0]
    assert np.linalg.norm(got - dw) <= 8e-3 * np.linalg.norm(dw)
    # the update from the gradient that the optimizer was given: mu M + G with M = G, that is G (1 + mu)
    want = w0 - t.opt.lr * t.opt.scale * R.orth64(got)
    moved = t.opt.lr * t.opt.scale * np.sqrt(E)
    assert np.linalg.norm(t.w.double().cpu().numpy()[0] - want) <= 1e-2 * moved
    assert torch.equal(t.w_bf16, t.w.to(torch.bfloat16))


def test_training_evens_the_loads():
    t = _trainer(lr=5e-3)
    offs = torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
    t.step(_batch(100), seq_offsets=offs)
    first, peak = t.loss[1].item(), (t.expert_loads().max() * E / t.expert_loads().sum()).item()
    for i in range(40):
        t.step(_batch(101 + i), seq_offsets=offs)
    last, now = t.loss[1].item(), (t.expert_loads().max() * E / t.expert_loads().sum()).item()
    assert first > 1.5 and last < 0.5 * (first + 1.0) and now < 0.7 * peak, (first, last, peak, now)


def test_captured_step_replays_the_eager_one():
    a, b = _trainer(), _trainer()
    offs = torch.tensor(OFFSETS, dtype=torch.int32, device="cuda")
    x = _batch(3)
    mask = (torch.arange(T, device="cuda") % 7 != 0).to(torch.uint8)
    start = b.w.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step(x, None, offs, mask)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step(x, None, offs, mask)
    b.w.copy_(start)
    b.w_bf16.copy_(start)
    b.opt.momentum.zero_()
    for i in range(4):
        x.copy_(_batch(10 + i))
        a.step(x, None, offs, mask)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.w, b.w) and torch.equal(a.loss, b.loss), i


@pytest.mark.parametrize("handle", [False, True])
def test_a_given_stream_takes_all_of_a_step(handle):
    # the stream is busy when the calls are made: whatever ran on another would read what is not written yet
    a, b = _trainer(), _trainer()
    offs, x = torch.tensor(OFFSETS, dtype=torch.int32, device="cuda"), _batch(4)
    a.step(x, None, offs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    b.forward(x, offs, stream=stream)
    b.backward(x, None, offs, stream=stream)
    b.opt.step(b.w, b.d_w, b.w_bf16, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(a.d_w, b.d_w) and torch.equal(a.w, b.w) and torch.equal(a.w_bf16, b.w_bf16)


def test_muon_refuses():
    opt = Muon(2, 8, 16, 1e-3)
    w, g = torch.zeros((2, 8, 16), device="cuda"), torch.zeros((2, 16, 8), device="cuda")
    with pytest.raises(ValueError):
        opt.step(w, g)
    with pytest.raises(ValueError):
        opt.step(w.half(), w)
    with pytest.raises(ValueError):
        opt.step(w, g.transpose(1, 2))
