"""The bias that evens the loads (training.Scores) in replayed graphs of batches of many sequences."""
import pytest
import torch

pytestmark = pytest.mark.gpu

D, K, R = 128, 4, 4


def _trainer(T, E, n_seq):
    from paper_2607_05116_amd.training import RouterTrainer, Scores
    g = torch.Generator("cuda").manual_seed(5)
    e = torch.arange(E, dtype=torch.int32)
    w = torch.randn((E, D), generator=g, device="cuda") / 8
    return RouterTrainer(T, D, E, K, R, R, e // (E // R), e % (E // R), w, p=0.1, n_seq=n_seq, lr=1e-2,
                         scores=Scores("sigmoid", n_groups=4, topk_groups=2, group_top=2, bias_speed=0.01))


@pytest.mark.parametrize("T,E,n_seq", [(4096, 32, 1), (4096, 32, 4), (4096, 32, 4096), (65536, 256, 65536), (65536, 20, 40001)])
def test_bias_in_a_graph(T, E, n_seq):
    """Each step adds 0.01 sign(mean load - load), the mean exact: eager steps and replays, with other work between."""
    g = torch.Generator("cuda").manual_seed(T + n_seq)
    offs = torch.linspace(0, T, n_seq + 1, device="cuda", dtype=torch.float64).to(torch.int32)
    t = _trainer(T, E, n_seq)
    x = torch.randn((T, D), generator=g, device="cuda").to(torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        t.step(x, None, offs)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.step(x, None, offs)
    other = torch.randn((1024, 1024), generator=g, device="cuda")
    for i in range(6):
        x.copy_(torch.randn((T, D), generator=g, device="cuda"))
        before = t.bias.clone()
        other = other @ other / 32
        torch.cuda.synchronize()
        graph.replay() if i % 3 < 2 else t.step(x, None, offs)
        torch.cuda.synchronize()
        loads = t.counts.cpu().long().sum(0)
        want = torch.sign(loads.sum() - loads * E).float()
        # one rounding of a sum of a few hundredths
        assert torch.allclose((t.bias - before).cpu(), 0.01 * want, rtol=0, atol=1e-7), i
        assert torch.equal(t.expert_loads().cpu(), loads)
        # the weights' gradient is a library product: replayed, it is the same as called
        assert torch.equal(t.d_w[0], torch.mm(t.d_logits.t(), x))
