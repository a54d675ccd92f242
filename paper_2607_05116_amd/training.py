"""Training the router and the weights of an expert-parallel MoE layer on one GPU.

RouterTrainer owns the device buffers of a router's training step and chains the
C-ABI calls in its order:

  router_route_prune (logits, routing, pruning) -> balance_loss -> router_grad
  -> the gradient of the router's weights -> muon_update -> the weights

Muon is the optimizer for a batch of matrices of one shape (the experts' of a
rank, or the router's): momentum, then the orthogonalised update.

Every step of the method runs in libcap.so's HIP kernels; this module allocates,
passes pointers, and takes the weights' gradient as one library product and the
weights' own update as elementwise torch operations.  All calls are asynchronous on
the current stream, write fixed buffers and read nothing back, so a step can be
captured into a HIP graph.

`python -m paper_2607_05116_amd.training` trains a router on synthetic tokens
until its experts are evenly loaded.
"""
from __future__ import annotations

import contextlib
import math

import torch

from . import capi

_BF16 = torch.bfloat16


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def _on(stream):
    """What follows, torch operations too, on the given stream (None: the current one)."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        # (an ExternalStream of handle 0 is a new stream of torch's pool, not the default one)
        stream = torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


def _check(name: str, t, shape, dtypes, device, optional: bool = True):
    """Refuses what a kernel would misread: it goes by pointers and sizes alone."""
    if t is None and optional:
        return
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: a tensor is taken, got {type(t).__name__}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} is {list(t.shape)}, expected {list(shape)}")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} is {t.dtype}; {' or '.join(str(d) for d in dtypes)} is taken")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class Muon:
    """Momentum and orthogonalised updates of `batch` matrices [rows][cols].

    step(): M <- mu M + G; O = orthogonalised G + mu M; W <- (1 - lr wd) W - lr 0.2 sqrt(max(rows, cols)) O.
    The factor gives every entry of the update a size of about 0.2 lr whatever the shape, since O's singular
    values are about 1.
    """

    def __init__(self, batch: int, rows: int, cols: int, lr: float, mu: float = 0.95, weight_decay: float = 0.0,
                 steps: int = 5, nesterov: bool = True, eps: float = 1e-7, device: str = "cuda"):
        self.shape = (batch, rows, cols)
        self.lr, self.mu, self.weight_decay = float(lr), float(mu), float(weight_decay)
        self.steps, self.nesterov, self.eps = int(steps), bool(nesterov), float(eps)
        self.scale = 0.2 * math.sqrt(max(rows, cols))
        self.momentum = torch.zeros(self.shape, dtype=torch.float32, device=device)
        self.update = torch.empty(self.shape, dtype=_BF16, device=device)
        self.ws = _workspace(capi.cap_workspace_size(capi.CAP_OP_ORTHOGONALISE, None, d=cols, inter=rows,
                                                     max_rows=batch), device)

    def step(self, w: torch.Tensor, g: torch.Tensor, w_bf16: torch.Tensor | None = None, stream=None):
        """w (fp32, updated in place), g (fp32 or bf16): [batch][rows][cols], contiguous; w_bf16: a copy of the
        weights to refresh (what the layer's kernels read).  All of it on `stream` (None: the current one)."""
        if tuple(w.shape) != self.shape:
            raise ValueError(f"weights are {list(w.shape)}, expected {list(self.shape)}")
        if w.dtype != torch.float32 or w.device != self.momentum.device:
            raise ValueError(f"weights are {w.dtype} on {w.device}; fp32 on {self.momentum.device} is taken")
        if w_bf16 is not None and tuple(w_bf16.shape) != self.shape:
            raise ValueError(f"the weights' copy is {list(w_bf16.shape)}, expected {list(self.shape)}")
        _check("the gradient", g, self.shape, (torch.float32, _BF16), self.momentum.device, optional=False)
        dt = capi.CAP_DTYPE_BF16 if g.dtype == _BF16 else capi.CAP_DTYPE_F32
        with _on(stream):
            capi.cap_muon_update(dt, *self.shape, g, self.momentum, self.mu, self.nesterov, self.steps, None, self.eps,
                                 self.update, self.ws)
            if self.weight_decay:
                w.mul_(1.0 - self.lr * self.weight_decay)
            w.add_(self.update, alpha=-self.lr * self.scale)
            if w_bf16 is not None:
                w_bf16.copy_(w)


class RouterTrainer:
    """Buffers and calls of one layer's router training.

    T tokens a step over R virtual ranks (T % R == 0), hidden size d (a multiple of 64), E experts (17 to 256), top k;
    expert_rank / expert_local: the placement that pruning goes by (int32 [E]); p its threshold.  n_seq: sequences
    of a batch (their offsets come with each step).

    Tokens that a mask or the offsets leave out count nowhere, whatever their rows of x hold: with either given, a copy
    of x with zeros in those rows is what the router and the weights' gradient read (a zero gradient times a row that
    is not finite would be NaN in all of the weights).
    """

    def __init__(self, T: int, d: int, E: int, k: int, R: int, ranks_per_node: int, expert_rank, expert_local, w_gate,
                 p: float = 0.0, n_seq: int = 1, balance_coef: float = 1e-2, z_coef: float = 1e-3, lr: float = 1e-3,
                 mu: float = 0.95, device: str = "cuda"):
        self.T, self.d, self.E, self.k, self.n_seq, self.p = T, d, E, k, n_seq, float(p)
        self.balance_coef, self.z_coef = float(balance_coef), float(z_coef)
        dev = self.dev = torch.device(device)
        self.expert_rank = torch.as_tensor(expert_rank, dtype=torch.int32).to(dev)
        self.expert_local = torch.as_tensor(expert_local, dtype=torch.int32).to(dev)
        self.topo = capi.make_topology(E, R, ranks_per_node, T, k, self.expert_rank, self.expert_local)
        self.w = torch.as_tensor(w_gate, dtype=torch.float32).to(dev).reshape(1, E, d).contiguous()
        self.w_bf16 = self.w.to(_BF16)
        i32 = dict(dtype=torch.int32, device=dev)
        self.idx = torch.empty((T, k), **i32)
        self.gates = torch.empty((T, k), dtype=torch.float32, device=dev)
        self.keep = torch.empty((T, k), dtype=torch.uint8, device=dev)
        self.mask = torch.empty(T, dtype=torch.int64, device=dev)
        self.logits = torch.empty((T, E), dtype=torch.float32, device=dev)
        self.counts = torch.empty((n_seq, E), **i32)
        self.probs = torch.empty((n_seq, E), dtype=torch.float32, device=dev)
        self.tokens = torch.empty(n_seq + 2, **i32)
        self.loss = torch.empty(3, dtype=torch.float32, device=dev)
        # bf16, as the product of both on the matrix cores takes and gives them: 2^-9 of each value, twice, below what
        # the orthogonalised update rounds by itself
        self.d_logits = torch.empty((T, E), dtype=_BF16, device=dev)
        self.d_w = torch.empty((1, E, d), dtype=_BF16, device=dev)
        self.rows = torch.empty((T, d), dtype=_BF16, device=dev)
        self.token = torch.arange(T, **i32)
        self.counted, self.one_rule = (torch.empty(T, dtype=torch.bool, device=dev) for _ in range(2))
        self.zero = torch.zeros((), dtype=_BF16, device=dev)
        self.ws = _workspace(capi.cap_workspace_size(capi.CAP_OP_BALANCE_LOSS, self.topo, max_rows=n_seq), dev)
        self.opt = Muon(1, E, d, lr, mu, device=device)

    def _check_batch(self, x, seq_offsets, token_mask, d_gates=None, d_loss=None):
        dev = self.w.device
        _check("x", x, (self.T, self.d), (_BF16,), dev, optional=False)
        _check("seq_offsets", seq_offsets, (self.n_seq + 1,), (torch.int32,), dev)
        _check("token_mask", token_mask, (self.T,), (torch.uint8, torch.bool), dev)
        _check("d_gates", d_gates, (self.T, self.k), (torch.float32,), dev)
        if d_loss is not None:
            _check("d_loss", d_loss.reshape(-1) if isinstance(d_loss, torch.Tensor) else d_loss, (1,), (torch.float32,), dev)

    def _counted_rows(self, x: torch.Tensor, seq_offsets, token_mask) -> torch.Tensor:
        """x, with zeros in the rows of tokens that a mask or the offsets leave out."""
        if seq_offsets is None and token_mask is None:
            return x
        self.counted.fill_(True)
        if seq_offsets is not None:
            self.counted.logical_and_(torch.ge(self.token, seq_offsets[0], out=self.one_rule))
            self.counted.logical_and_(torch.lt(self.token, seq_offsets[-1], out=self.one_rule))
        if token_mask is not None:
            self.counted.logical_and_(torch.ne(token_mask, 0, out=self.one_rule))
        return torch.where(self.counted[:, None], x, self.zero, out=self.rows)

    def forward(self, x: torch.Tensor, seq_offsets=None, token_mask=None, stream=None):
        """Logits, routing, pruning and the losses of x (bf16 [T][d]); seq_offsets int32 [n_seq + 1] on the device
        (None: one sequence), token_mask uint8 or bool [T] (0: padding)."""
        self._check_batch(x, seq_offsets, token_mask)
        with _on(stream):
            self._forward(self._counted_rows(x, seq_offsets, token_mask), seq_offsets, token_mask)

    def _forward(self, x, seq_offsets, token_mask):
        capi.cap_router_route_prune(self.topo, capi.CAP_DTYPE_BF16, self.d, x, self.w_bf16, self.p, self.idx,
                                    self.gates, self.keep, self.mask, self.logits)
        capi.cap_balance_loss(self.T, self.k, self.E, self.logits, self.idx, self.keep, token_mask, seq_offsets,
                              self.n_seq, self.balance_coef, self.z_coef, self.counts, self.probs, self.tokens,
                              self.loss, self.ws)

    def backward(self, x: torch.Tensor, d_gates=None, seq_offsets=None, token_mask=None, d_loss=None, stream=None):
        """d_logits and the weights' gradient, for the gradient d_gates at the gates (None: of the losses alone) and
        d_loss at their total (a device scalar; None: 1)."""
        self._check_batch(x, seq_offsets, token_mask, d_gates, d_loss)
        with _on(stream):
            self._backward(self._counted_rows(x, seq_offsets, token_mask), d_gates, seq_offsets, token_mask, d_loss)

    def _backward(self, x, d_gates, seq_offsets, token_mask, d_loss):
        capi.cap_router_grad(self.T, self.k, self.E, self.logits, self.idx, self.keep, self.gates, d_gates, token_mask,
                             seq_offsets, self.n_seq, self.counts, self.tokens, self.balance_coef, self.z_coef, d_loss,
                             capi.CAP_DTYPE_BF16, self.d_logits)
        torch.mm(self.d_logits.t(), x, out=self.d_w[0])

    def step(self, x: torch.Tensor, d_gates=None, seq_offsets=None, token_mask=None):
        """One training step on the current stream."""
        self._check_batch(x, seq_offsets, token_mask, d_gates)
        x = self._counted_rows(x, seq_offsets, token_mask)
        self._forward(x, seq_offsets, token_mask)
        self._backward(x, d_gates, seq_offsets, token_mask, None)
        self.opt.step(self.w, self.d_w, self.w_bf16)

    def expert_loads(self) -> torch.Tensor:
        """Kept slots per expert of the last batch."""
        return self.counts.sum(0)


def _example(steps: int = 40):
    T, d, E, k, R, n_seq = 8192, 2048, 128, 8, 8, 8
    g = torch.Generator(device="cuda").manual_seed(0)
    e = torch.arange(E, dtype=torch.int32)
    w = torch.randn((E, d), generator=g, device="cuda") / math.sqrt(d)
    # tokens share a direction, which the untrained router answers with a few hot experts
    common = torch.randn((1, d), generator=g, device="cuda")
    offsets = torch.linspace(0, T, n_seq + 1, device="cuda").to(torch.int32)
    trainer = RouterTrainer(T, d, E, k, R, R, e // (E // R), e % (E // R), w, p=0.1, n_seq=n_seq, lr=2e-3)
    for i in range(steps):
        x = (torch.randn((T, d), generator=g, device="cuda") + 1.5 * common).to(_BF16)
        trainer.step(x, seq_offsets=offsets)
        if i % 10 == 0 or i + 1 == steps:
            loads = trainer.expert_loads().float()
            print(f"step {i:3d}: balance loss {trainer.loss[1].item():.3f}, z loss {trainer.loss[2].item():.3f}, "
                  f"most loaded expert {loads.max().item() / loads.mean().item():.2f} x the mean", flush=True)


if __name__ == "__main__":
    _example()
