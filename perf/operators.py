"""Performance cases of the MoE layer's training operators, measured through the public entry points.

Four operators train the router and the weights of an expert-parallel MoE layer:

  balance   the load-balance and z loss of a batch's routing, with per-sequence expert counts
  grad      its gradient and that of the gates, joined into the gradient of the router logits
  orth      the orthogonalised form of a batch of weight gradients (five Newton-Schulz steps)
  muon      momentum, then the same, as an optimizer step asks for it

With `own` false, run() computes them in elementary torch operations in 32 bits; with `own` true it calls the
package.  Shapes are the layers of workloads.generator.CONFIGS (Qwen3-30B-A3B, DeepSeek-V2-Lite, DeepSeek-V3).
"""
import math
import types

import torch

own = False

DEV = "cuda"
COEF = (3.4445, -4.7750, 2.0315)     # the quintic X <- a X + b (X X^T) X + c (X X^T)^2 X
STEPS = 5
EPS = 1e-7
LARGEST_FLOPS = 3.95e12              # the largest listed case; drawn ones stay below


def listed():
    return [
        # ---- balance loss, forward
        # a training batch of 8 sequences through a DeepSeek-V3 layer's router
        dict(name="balance_batch_dsv3", path="balance", T=32768, E=256, k=8, n_seq=8, masked=False, pruned=True),
        # a packed micro-batch of many short sequences with padding, DeepSeek-V2-Lite layer
        dict(name="balance_packed_dsv2lite", path="balance", T=8192, E=64, k=6, n_seq=211, masked=True, pruned=True),
        # one short sequence, small layer
        dict(name="balance_short", path="balance", T=61, E=16, k=2, n_seq=1, masked=False, pruned=False),
        # ---- gradient of the router logits
        # the training batch's, as the router's weight gradient in fp32 takes it
        dict(name="grad_batch_dsv3", path="grad", T=32768, E=256, k=8, n_seq=8, masked=False, pruned=True,
             out="f32"),
        # the packed micro-batch's, for bf16 products
        dict(name="grad_packed_dsv2lite", path="grad", T=8192, E=64, k=6, n_seq=211, masked=True, pruned=True,
             out="bf16"),
        # one short sequence, small layer
        dict(name="grad_short", path="grad", T=61, E=16, k=2, n_seq=1, masked=False, pruned=False, out="f32"),
        # ---- orthogonalised gradients
        # the gate weights of a DeepSeek-V3 layer's experts on one of 32 ranks
        dict(name="orth_experts_dsv3", path="orth", batch=8, rows=2048, cols=7168, dtype="bf16"),
        # the down weights of a Qwen3-30B-A3B layer's experts on one of 8 ranks (more rows than columns)
        dict(name="orth_down_qwen3", path="orth", batch=16, rows=2048, cols=768, dtype="f32"),
        # the router's weights of a DeepSeek-V3 layer: one matrix of few rows
        dict(name="orth_router_dsv3", path="orth", batch=1, rows=256, cols=7168, dtype="f32"),
        # ---- with momentum
        # the gate weights of a DeepSeek-V2-Lite layer's experts on one of 8 ranks
        dict(name="muon_experts_dsv2lite", path="muon", batch=8, rows=1408, cols=2048, dtype="bf16"),
        # the router's weights of a Qwen3-30B-A3B layer
        dict(name="muon_router_qwen3", path="muon", batch=1, rows=128, cols=2048, dtype="f32"),
        # a few small matrices of odd sizes
        dict(name="muon_odd", path="muon", batch=3, rows=333, cols=517, dtype="f32"),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _flops(batch, rows, cols):
    """Multiplications and additions of the steps, a symmetric product's mirrored half not counted."""
    n, m = min(rows, cols), max(rows, cols)
    return float(STEPS) * batch * (3.0 * n * n * m + float(n) ** 3)


def draw(rng):
    path = rng.choice(["balance", "grad", "orth", "muon"])
    if path in ("balance", "grad"):
        E = rng.choice([16, 64, 128, 256, rng.randint(2, 256)])
        T = _log(rng, 1, 32768)
        if T == 3072:
            T += 1
        c = dict(path=path, T=T, E=E, k=rng.randint(1, min(8, E)), n_seq=_log(rng, 1, max(1, min(512, T))),
                 masked=rng.random() < 0.5, pruned=rng.random() < 0.5)
        if path == "grad":
            c["out"] = rng.choice(["f32", "bf16"])
        return c
    while True:
        c = dict(path=path, batch=_log(rng, 1, 32), rows=_log(rng, 1, 7168), cols=_log(rng, 1, 7168),
                 dtype=rng.choice(["bf16", "f32"]))
        if rng.random() < 0.5:              # the sizes that layers have
            c["rows"], c["cols"] = 64 * -(-c["rows"] // 64), 64 * -(-c["cols"] // 64)
        if 3072 in (c["rows"], c["cols"]):
            continue
        if _flops(c["batch"], c["rows"], c["cols"]) <= LARGEST_FLOPS and c["batch"] * c["rows"] * c["cols"] <= 2 ** 27:
            return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _logits(g, T, E):
    """Latent-topic router logits with Zipf expert popularity; the model part (clusters, popularity) is fixed."""
    C = max(1, E // 8)
    fixed = torch.Generator().manual_seed(17)
    cluster = (torch.randperm(E, generator=fixed) * C // E).to(DEV)
    bias = (-1.1 * torch.log(torch.randperm(E, generator=fixed).double() + 1)).float().to(DEV)
    topic = torch.randint(0, C, (T, 1), generator=g, device=DEV)
    return 2.0 * (cluster[None, :] == topic) + bias + torch.randn((T, E), generator=g, device=DEV)


def _routing(g, case):
    """Logits, the chosen experts, which of them pruning kept, and the kept gates renormalised."""
    T, E, k = case["T"], case["E"], case["k"]
    logits = _logits(g, T, E)
    top, idx = torch.sort(logits, dim=1, descending=True, stable=True)
    q = torch.exp(top[:, :k] - top[:, :1])
    w = q / q.sum(1, keepdim=True)
    keep = torch.ones((T, k), dtype=torch.bool, device=DEV)
    if case["pruned"]:
        keep = torch.cumsum(w, 1) - w < 0.9
    w = torch.where(keep, w, 0.0)
    return (logits, idx[:, :k].to(torch.int32).contiguous(), keep.to(torch.uint8),
            (w / w.sum(1, keepdim=True)).contiguous())


def _sequences(case, g):
    """Offsets of ragged sequences over the batch (some may be empty), and the padding mask."""
    T, S = case["T"], case["n_seq"]
    fixed = torch.Generator().manual_seed(29 + T + S)
    cuts = torch.randint(0, T + 1, (S - 1,), generator=fixed).sort().values
    offs = torch.cat([torch.zeros(1, dtype=torch.long), cuts, torch.full((1,), T)]).to(torch.int32).to(DEV)
    mask = None
    if case["masked"]:
        mask = (torch.rand(T, generator=g, device=DEV) < 0.9).to(torch.uint8)
    return offs, mask


def _matrices(g, case):
    """Gradients: a few strong directions over noise, as gradients of weights have them."""
    b, r, c = case["batch"], case["rows"], case["cols"]
    rank = min(16, r, c)
    u = torch.randn((b, r, rank), generator=g, device=DEV)
    v = torch.randn((b, rank, c), generator=g, device=DEV) / torch.arange(1, rank + 1, device=DEV)[:, None]
    x = torch.bmm(u, v) + torch.randn((b, r, c), generator=g, device=DEV)
    return (1e-3 * x).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)


def prepare(case, seed):
    g = _gen(seed)
    s = types.SimpleNamespace(path=case["path"], case=case)
    if case["path"] in ("balance", "grad"):
        T, E, S = case["T"], case["E"], case["n_seq"]
        s.logits, s.idx, s.keep, s.w = _routing(g, case)
        s.offs, s.mask = _sequences(case, g)
        s.balance_coef, s.z_coef = 1e-2, 1e-3
        if case["path"] == "balance":
            s.counts = torch.empty((S, E), dtype=torch.int32, device=DEV)
            s.probs = torch.empty((S, E), device=DEV)
            s.tokens = torch.empty(S + 2, dtype=torch.int32, device=DEV)
            s.loss = torch.empty(3, device=DEV)
            s.ws = torch.empty(4 * (2 * E + 4) * (T // 4 + S + 64), dtype=torch.uint8, device=DEV)
        else:
            seg = _segments(s)
            valid = torch.ones(T, dtype=torch.bool, device=DEV) if s.mask is None else s.mask.bool()
            s.counts, s.tokens = _counts(s, seg, valid)
            s.d_w = torch.randn(s.w.shape, generator=g, device=DEV) * 1e-3
            s.d_loss = torch.ones((), device=DEV)
            s.d_logits = torch.empty((T, E), device=DEV,
                                     dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32)
        return s
    b, r, c = case["batch"], case["rows"], case["cols"]
    s.g = _matrices(g, case)
    s.out = torch.empty((b, r, c), dtype=torch.bfloat16, device=DEV)
    if case["path"] == "muon":
        s.mu = 0.95
        s.momentum = 10.0 * _matrices(g, dict(case, dtype="f32"))
    n, m = (256 * -(-v // 256) for v in (min(r, c), max(r, c)))
    s.ws = torch.empty(16 * b * n * (m + n) + 64 * 2 ** 20, dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------ the plain form
def _segments(s):
    """The sequence of every token."""
    t = torch.arange(s.case["T"], device=DEV)
    return torch.bucketize(t, s.offs[1:].long(), right=True)


def _members(seg, S):
    return (torch.arange(S, device=DEV)[:, None] == seg[None, :]).float()


def _counts(s, seg, valid):
    """Kept slots per sequence and expert; valid tokens per sequence, sequences that have one, tokens in all."""
    T, E, S = s.case["T"], s.case["E"], s.case["n_seq"]
    chosen = torch.zeros((T, E), device=DEV).scatter_add_(1, s.idx.long(), s.keep.float())
    member = _members(seg, S)
    counts = member @ torch.where(valid[:, None], chosen, 0.0)
    n = (member @ valid.float()[:, None])[:, 0].to(torch.int32)
    return counts.to(torch.int32), torch.cat([n, (n > 0).sum()[None].to(torch.int32), n.sum()[None].to(torch.int32)])


def _softmax(s):
    """Probabilities and log-sum-exp; rows of masked tokens, and of those without a finite logit, are 0."""
    top = s.logits.max(1, keepdim=True).values
    valid = top[:, 0] > -math.inf
    if s.mask is not None:
        valid = valid & (s.mask != 0)
    e = torch.exp(s.logits - top)
    total = e.sum(1, keepdim=True)
    p = torch.where(valid[:, None], e / total, 0.0)
    lse = torch.where(valid, (top + torch.log(total))[:, 0], 0.0)
    return p, lse, valid


def _plain_balance(s):
    E, k, S = s.case["E"], s.case["k"], s.case["n_seq"]
    p, lse, valid = _softmax(s)
    seg = _segments(s)
    counts, tokens = _counts(s, seg, valid)
    n = tokens[:S].float().clamp(min=1.0)[:, None]
    probs = (_members(seg, S) @ p) / n
    balance = (counts * probs / n).sum() * (E / k) / tokens[S].clamp(min=1)
    z = lse.square().sum() / tokens[S + 1].clamp(min=1)
    return dict(counts=counts, probs=probs, tokens=tokens,
                loss=torch.stack([s.balance_coef * balance + s.z_coef * z, balance, z]))


def _plain_grad(s):
    E, k, S = s.case["E"], s.case["k"], s.case["n_seq"]
    p, lse, valid = _softmax(s)
    n = s.tokens[:S].float().clamp(min=1.0)[:, None]
    per = s.counts * (s.d_loss * s.balance_coef * (E / k) / s.tokens[S].clamp(min=1)) / (n * n)
    c = per[_segments(s)]
    d = p * (c - (p * c).sum(1, keepdim=True))
    d = d + p * (lse * (s.d_loss * 2.0 * s.z_coef / s.tokens[S + 1].clamp(min=1)))[:, None]
    w = torch.where(s.keep != 0, s.w, 0.0)
    gate = w * (s.d_w - (w * s.d_w).sum(1, keepdim=True))
    d = d.scatter_add(1, s.idx.long(), gate)
    return torch.where(valid[:, None], d, 0.0).to(s.d_logits.dtype)


def _newton_schulz(x):
    """One step: a X + (b S + c S S) X with S = X X^T."""
    a, b, c = COEF
    t = torch.bmm(x, x.transpose(1, 2).contiguous())
    return a * x + torch.bmm(b * t + c * torch.bmm(t, t), x)


def _plain_orth(u):
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    x = _newton_schulz(_newton_schulz(_newton_schulz(_newton_schulz(_newton_schulz(x)))))
    return (x.transpose(1, 2).contiguous() if tall else x).to(torch.bfloat16)


def _plain(s):
    if s.path == "balance":
        return _plain_balance(s)
    if s.path == "grad":
        return _plain_grad(s)
    g = s.g.float()
    if s.path == "orth":
        return _plain_orth(g)
    s.momentum.mul_(s.mu).add_(g)
    return dict(update=_plain_orth(g + s.mu * s.momentum), momentum=s.momentum)


# ------------------------------------------------------------------ the package's calls
def _own(s):
    from paper_2607_05116_amd import capi
    c = s.case
    if s.path == "balance":
        capi.cap_balance_loss(c["T"], c["k"], c["E"], s.logits, s.idx, s.keep, s.mask, s.offs, c["n_seq"],
                              s.balance_coef, s.z_coef, s.counts, s.probs, s.tokens, s.loss, s.ws)
        return dict(counts=s.counts, probs=s.probs, tokens=s.tokens, loss=s.loss)
    if s.path == "grad":
        dt = capi.CAP_DTYPE_BF16 if c["out"] == "bf16" else capi.CAP_DTYPE_F32
        capi.cap_router_grad(c["T"], c["k"], c["E"], s.logits, s.idx, s.keep, s.w, s.d_w, s.mask, s.offs, c["n_seq"],
                             s.counts, s.tokens, s.balance_coef, s.z_coef, s.d_loss, dt, s.d_logits)
        return s.d_logits
    dt = capi.CAP_DTYPE_BF16 if c["dtype"] == "bf16" else capi.CAP_DTYPE_F32
    if s.path == "orth":
        capi.cap_orthogonalise(dt, c["batch"], c["rows"], c["cols"], s.g, STEPS, None, EPS, s.out, s.ws)
        return s.out
    capi.cap_muon_update(dt, c["batch"], c["rows"], c["cols"], s.g, s.momentum, s.mu, True, STEPS, None, EPS, s.out,
                         s.ws)
    return dict(update=s.out, momentum=s.momentum)


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["path"] in ("balance", "grad"):
        T, E, k, S = case["T"], case["E"], case["k"], case["n_seq"]
        rows = 4.0 * T * E + 5.0 * T * k + (T if case["masked"] else 0) + 4.0 * S * (E + 2)
        if case["path"] == "balance":
            return dict(bytes=rows + 4.0 * S * E, flops=5.0 * T * E)
        return dict(bytes=rows + (2.0 if case["out"] == "bf16" else 4.0) * T * E + 8.0 * T * k, flops=9.0 * T * E)
    values = float(case["batch"]) * case["rows"] * case["cols"]
    each = (2 if case["dtype"] == "bf16" else 4) + 2 + (8 if case["path"] == "muon" else 0)
    return dict(bytes=each * values, flops=_flops(case["batch"], case["rows"], case["cols"]))


# ------------------------------------------------------------------ the same in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)

    def losses(x):
        """Counts, mean probabilities, tokens, the two losses and the valid tokens; sequence by sequence."""
        E, k, S = case["E"], case["k"], case["n_seq"]
        cuts = s.offs.tolist()
        valid = torch.ones(case["T"], dtype=torch.bool, device=DEV) if s.mask is None else s.mask.bool()
        p = torch.softmax(x, 1)
        balance, n, counts, probs = 0.0, [], [], []
        for i in range(S):
            at = torch.arange(cuts[i], cuts[i + 1], device=DEV)
            at = at[valid[at]]
            n.append(len(at))
            chosen = s.idx[at].long()[s.keep[at] != 0]
            counts.append(torch.bincount(chosen.flatten(), minlength=E))
            probs.append(p[at].sum(0) / max(1, len(at)))
            balance = balance + E / (k * max(1, len(at))) * (counts[-1] * probs[-1]).sum()
        present = sum(1 for v in n if v)
        z = torch.logsumexp(x[valid], 1).square().sum() / max(1, sum(n))
        tokens = torch.tensor(n + [present, sum(n)], dtype=torch.int32, device=DEV)
        return (torch.stack(counts).to(torch.int32), torch.stack(probs), tokens, balance / max(1, present), z, valid)

    if case["path"] == "balance":
        counts, probs, tokens, balance, z, _ = losses(s.logits.double())
        return dict(counts=counts, probs=probs, tokens=tokens,
                    loss=torch.stack([s.balance_coef * balance + s.z_coef * z, balance, z]))
    if case["path"] == "grad":
        x = s.logits.double().requires_grad_(True)
        _, _, _, balance, z, valid = losses(x)
        kept = torch.gather(x, 1, s.idx.long()).masked_fill(s.keep == 0, -math.inf)
        gates = (torch.softmax(kept, 1) * s.d_w.double())[valid].sum()
        (s.d_loss.double() * (s.balance_coef * balance + s.z_coef * z) + gates).backward()
        return x.grad
    u = s.g.double()
    if case["path"] == "muon":
        momentum = s.mu * s.momentum.double() + u
        u = u + s.mu * momentum
    u = u / (torch.linalg.vector_norm(u, dim=(1, 2), keepdim=True) + EPS)
    a, b, c = COEF
    for _ in range(STEPS):
        if u.shape[1] <= u.shape[2]:
            t = u @ u.mT
            u = a * u + (b * t + c * (t @ t)) @ u
        else:                              # (X X^T) X = X (X^T X): the smaller product
            t = u.mT @ u
            u = a * u + u @ (b * t + c * (t @ t))
    return dict(update=u, momentum=momentum) if case["path"] == "muon" else u
