"""What the training classes refuse before anything is launched: tensors that the kernels, which go by pointers and
sizes, would read past or misread (paper_2607_05116_amd.training; on the CPU, where no call goes through)."""
import pytest
import torch

from paper_2607_05116_amd import training
from paper_2607_05116_amd.training import Muon, RouterTrainer

T, D, E, K, SEQS = 64, 128, 32, 4, 3


@pytest.fixture
def trainer(monkeypatch):
    for name in ("cap_router_route_prune", "cap_balance_loss", "cap_router_grad", "cap_muon_update"):
        monkeypatch.setattr(training.capi, name, lambda *a, **k: pytest.fail("a refused call went through"))
    e = torch.arange(E, dtype=torch.int32)
    return RouterTrainer(T, D, E, K, 4, 4, e // 8, e % 8, torch.zeros(E, D), n_seq=SEQS, device="cpu")


def _good():
    return dict(x=torch.zeros(T, D, dtype=torch.bfloat16), seq_offsets=torch.zeros(SEQS + 1, dtype=torch.int32),
                token_mask=torch.ones(T, dtype=torch.uint8), d_gates=torch.zeros(T, K))


BAD = [dict(x=torch.zeros(T, D)), dict(x=torch.zeros(T - 1, D, dtype=torch.bfloat16)),
       dict(x=torch.zeros(T, D + 64, dtype=torch.bfloat16)[:, :D]), dict(x=torch.zeros(T, D, dtype=torch.bfloat16, device="meta")),
       dict(x=None), dict(seq_offsets=torch.zeros(SEQS + 1, dtype=torch.int64)),
       dict(seq_offsets=torch.zeros(SEQS, dtype=torch.int32)), dict(seq_offsets=[0, 1, 2, 3]),
       dict(token_mask=torch.ones(T, dtype=torch.int64)), dict(token_mask=torch.ones(T - 1, dtype=torch.uint8)),
       dict(token_mask=torch.ones(2 * T, dtype=torch.uint8)[::2])]
BAD_BACKWARD = [dict(d_gates=torch.zeros(T, K, dtype=torch.bfloat16)), dict(d_gates=torch.zeros(T, K + 1)),
                dict(d_gates=torch.zeros(K, T).t())]


@pytest.mark.parametrize("bad", range(len(BAD)))
def test_router_trainer_refuses(trainer, bad):
    a = {**_good(), **BAD[bad]}
    for call in (lambda: trainer.forward(a["x"], a["seq_offsets"], a["token_mask"]),
                 lambda: trainer.backward(a["x"], a["d_gates"], a["seq_offsets"], a["token_mask"]),
                 lambda: trainer.step(a["x"], a["d_gates"], a["seq_offsets"], a["token_mask"])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("bad", range(len(BAD_BACKWARD)))
def test_router_trainer_refuses_gradients(trainer, bad):
    a = {**_good(), **BAD_BACKWARD[bad]}
    with pytest.raises(ValueError):
        trainer.backward(a["x"], a["d_gates"], a["seq_offsets"], a["token_mask"])
    with pytest.raises(ValueError):
        trainer.step(a["x"], a["d_gates"], a["seq_offsets"], a["token_mask"])


@pytest.mark.parametrize("d_loss", [torch.zeros((), dtype=torch.float64), torch.zeros(2), 1.0])
def test_router_trainer_refuses_d_loss(trainer, d_loss):
    a = _good()
    with pytest.raises(ValueError):
        trainer.backward(a["x"], a["d_gates"], a["seq_offsets"], a["token_mask"], d_loss)


def test_muon_refuses(monkeypatch):
    monkeypatch.setattr(training.capi, "cap_muon_update", lambda *a, **k: pytest.fail("a refused call went through"))
    opt = Muon(2, 8, 16, 1e-3, device="cpu")
    w, g = torch.zeros(2, 8, 16), torch.zeros(2, 8, 16)
    for a in ((w[:1], g), (w.double(), g), (w, g[:1]), (w, g.half()), (w, g.transpose(1, 2)), (w, None),
              (w, torch.zeros(2, 8, 16, device="meta")), (w, g, torch.zeros(8, 16, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            opt.step(*a)
