"""Performance cases of scored routing and of the experts' products in 8-bit floating point.

Five operators, measured through the public entry points:

  route     routing by sigmoid or softmax scores, with a bias for balance, groups of experts, top-k, gates and pruning
  grad      the gradient of the router logits through its gates
  quantise  rows or weights in e4m3 with a power-of-two scale for each block of 128
  product   rows times their expert's weights, both in e4m3 with a scale for each block of 128
  ffn       the experts' SwiGLU feed-forward in that form

With `own` false, run() computes them in elementary torch operations (32 bits; the routing's decisions in 64); with
`own` true it calls the package.  Shapes are the layers of workloads.generator.CONFIGS (Qwen3-30B-A3B,
DeepSeek-V2-Lite, DeepSeek-V3).
"""
import math
import types

import torch

own = False

DEV = "cuda"
B = 128                              # values that share a scale
TOP = 448.0                          # the largest e4m3 value
F8 = torch.float8_e4m3fn
LARGEST_FLOPS = 2.92e12              # the largest listed case; drawn ones stay below
SIGMOID = dict(kind="sigmoid", n_groups=8, topk_groups=4, group_top=2, bias=True, normalise=True, scale=2.5)
SOFTMAX = dict(kind="softmax", n_groups=1, topk_groups=1, group_top=1, bias=False, normalise=False, scale=1.0)


def listed():
    return [
        # ---- routing
        # a training or prefill batch through a DeepSeek-V3 layer's router, pruned to fewer devices
        dict(name="route_batch_dsv3", path="route", T=32768, E=256, k=8, R=32, node=8, p=0.1, masked=False, **SIGMOID),
        # a packed batch with padding, DeepSeek-V2-Lite layer (softmax over all experts, gates as they are)
        dict(name="route_packed_dsv2lite", path="route", T=8192, E=64, k=6, R=8, node=8, p=0.0, masked=True, **SOFTMAX),
        # a decode step, one token on each rank of a DeepSeek-V3 layer
        dict(name="route_decode_dsv3", path="route", T=32, E=256, k=8, R=32, node=8, p=0.1, masked=False, **SIGMOID),
        # ---- its gradient
        # the training batch's, joined with the balance loss's gradient, as products in bf16 take it
        dict(name="grad_batch_dsv3", path="grad", T=32768, E=256, k=8, R=32, node=8, p=0.1, masked=False, add=True,
             out="bf16", **SIGMOID),
        # the packed batch's, in fp32
        dict(name="grad_packed_dsv2lite", path="grad", T=8192, E=64, k=6, R=8, node=8, p=0.0, masked=True, add=False,
             out="f32", **SOFTMAX),
        # ---- quantisation
        # the activations of a batch of a DeepSeek-V3 layer, before its experts read them
        dict(name="quantise_rows_dsv3", path="quantise", batch=1, rows=32768, cols=7168, block_rows=1, dtype="bf16"),
        # the gate weights of a Qwen3-30B-A3B layer's experts on one of 8 ranks, after an optimizer step
        dict(name="quantise_weights_qwen3", path="quantise", batch=16, rows=768, cols=2048, block_rows=128,
             dtype="f32"),
        # ---- grouped product
        # the down projection of rank 0's rows in the DeepSeek-V3 layer
        dict(name="product_down_dsv3", path="product", E_loc=8, rows=33234, n=7168, kdim=2048, x_rows=0, out="bf16"),
        # a projection of a few decoded tokens with an odd number of outputs, rows taken from the tokens
        dict(name="product_few_odd", path="product", E_loc=8, rows=37, n=1003, kdim=2048, x_rows=19, out="f32"),
        # ---- feed-forward
        # rank 0's experts of the DeepSeek-V3 layer over a batch, rows read through their tokens
        dict(name="ffn_batch_dsv3", path="ffn", E_loc=8, rows=33234, d=7168, inter=2048, x_rows=32768),
        # a ragged batch of the DeepSeek-V2-Lite layer
        dict(name="ffn_ragged_dsv2lite", path="ffn", E_loc=8, rows=3001, d=2048, inter=1408, x_rows=0),
        # a decode step of the DeepSeek-V3 layer: one token's row at each of a rank's experts
        dict(name="ffn_decode_dsv3", path="ffn", E_loc=8, rows=8, d=7168, inter=2048, x_rows=8),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _flops(c):
    if c["path"] == "product":
        return 2.0 * c["rows"] * c["n"] * c["kdim"]
    return 6.0 * c["rows"] * c["d"] * c["inter"]


def draw(rng):
    path = rng.choice(["route", "grad", "quantise", "product", "ffn"])
    if path in ("route", "grad"):
        R = rng.choice([1, 2, 4, 8, 16, 32])
        E = R * rng.randint(1, 256 // R)
        k = rng.randint(1, min(8, E))
        G = rng.choice([g for g in range(1, min(E, 32) + 1) if E % g == 0])
        least = -(-k // (E // G))
        c = dict(path=path, T=R * _log(rng, 1, 32768 // R), E=E, k=k, R=R, node=rng.choice([R, max(1, R // 2)]),
                 p=rng.choice([0.0, 0.1, 0.3]), masked=rng.random() < 0.3, kind=rng.choice(["sigmoid", "softmax"]),
                 n_groups=G, topk_groups=rng.randint(least, G), group_top=rng.choice([1, 2]),
                 bias=rng.random() < 0.5, normalise=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]))
        if path == "grad":
            c.update(add=rng.random() < 0.5, out=rng.choice(["f32", "bf16"]))
            if k == 1:              # a single normalised gate is constant: no gradient to compare
                c["normalise"] = False
            if c["T"] < 64:                 # nor is there one where pruning leaves every token a single gate
                c["p"] = 0.0
        return c
    if path == "quantise":
        while True:
            c = dict(path=path, batch=_log(rng, 1, 16), rows=_log(rng, 1, 32768), cols=B * _log(rng, 1, 56),
                     block_rows=rng.choice([1, 128]), dtype=rng.choice(["bf16", "f32"]))
            if c["batch"] * c["rows"] * c["cols"] <= 2 ** 27:
                return c
    while True:
        rows = _log(rng, 1, 33234)
        c = dict(path=path, E_loc=_log(rng, 1, 32), rows=rows, x_rows=rng.choice([0, _log(rng, 1, 32768)]))
        if path == "product":
            c.update(n=_log(rng, 1, 7168), kdim=B * _log(rng, 1, 56), out=rng.choice(["f32", "bf16"]))
            weights = c["E_loc"] * c["n"] * c["kdim"]
        else:
            c.update(d=B * _log(rng, 1, 56), inter=B * _log(rng, 1, 16))
            weights = 3 * c["E_loc"] * c["d"] * c["inter"]
        if _flops(c) <= LARGEST_FLOPS and weights <= 2 ** 29:
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


def _prepare_routing(s, g, case):
    T, E, k, R = case["T"], case["E"], case["k"], case["R"]
    s.logits = _logits(g, T, E)
    s.bias = 0.2 * torch.rand(E, generator=g, device=DEV) if case["bias"] else None
    s.token_mask = (torch.rand(T, generator=g, device=DEV) < 0.9).to(torch.uint8) if case["masked"] else None
    e = torch.arange(E, dtype=torch.int32, device=DEV)
    s.expert_rank, s.expert_local = e // (E // R), e % (E // R)
    s.idx = torch.empty((T, k), dtype=torch.int32, device=DEV)
    s.w = torch.empty((T, k), device=DEV)
    s.keep = torch.empty((T, k), dtype=torch.uint8, device=DEV)
    s.mask = torch.empty(T, dtype=torch.int64, device=DEV)
    if case["path"] == "grad":
        r = _plain_route(s)
        s.idx, s.w, s.keep = r["idx"], r["w"], r["keep"]
        s.d_w = 1e-3 * torch.randn((T, k), generator=g, device=DEV)
        s.d_add = 1e-4 * torch.randn((T, E), generator=g, device=DEV) if case["add"] else None
        s.d_logits = torch.empty((T, E), device=DEV, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32)
    s.options = s.topo = None
    if own:
        from paper_2607_05116_amd import capi
        s.topo = capi.make_topology(E, R, case["node"], T, k, s.expert_rank, s.expert_local)
        kind = capi.CAP_SCORE_SIGMOID if case["kind"] == "sigmoid" else capi.CAP_SCORE_SOFTMAX
        s.options = capi.make_score_options(kind, case["n_groups"], case["topk_groups"], case["group_top"],
                                            case["normalise"], case["scale"], s.bias, s.token_mask)


def _rows_of_experts(case):
    """Rows of each expert, ragged, some experts with none where rows are few."""
    n, fixed = case["E_loc"], torch.Generator().manual_seed(31 + case["rows"])
    if case["rows"] == n:
        return [1] * n
    share = torch.rand(n, generator=fixed) + 0.5
    cuts = (torch.cumsum(share, 0) / share.sum() * case["rows"]).round().long().tolist()
    cuts[-1] = case["rows"]
    return [b - a for a, b in zip([0] + cuts[:-1], cuts)]


def _weights(g, E_loc, n, k):
    """Weights in e4m3 with a scale in fp32 for each 128 x 128 block, as checkpoints hold them."""
    q = torch.empty((E_loc, n, k), dtype=F8, device=DEV)
    scale = torch.empty((E_loc, -(-n // B), k // B), device=DEV)
    for e in range(E_loc):
        w = torch.randn((n, k), generator=g, device=DEV) / math.sqrt(k)
        pad = torch.nn.functional.pad(w, (0, 0, 0, -n % B)).reshape(-1, B, k // B, B)
        s = pad.abs().amax((1, 3)) / TOP
        q[e] = (pad / s[:, None, :, None]).reshape(-1, k)[:n].to(F8)
        scale[e] = s
    return q, scale


def _prepare_product(s, g, case):
    rows, E_loc = case["rows"], case["E_loc"]
    k = case["kdim"] if case["path"] == "product" else case["d"]
    x_rows = case["x_rows"] or rows
    s.counts = _rows_of_experts(case)
    s.offsets = torch.tensor([sum(s.counts[:i]) for i in range(E_loc + 1)], dtype=torch.int32, device=DEV)
    s.row_src = None
    if case["x_rows"]:
        s.row_src = torch.randint(0, x_rows, (rows,), generator=g, device=DEV, dtype=torch.int32)
    x = torch.randn((x_rows, k), generator=g, device=DEV).to(torch.bfloat16)
    s.x, s.x_scale = _plain_quantise(x[None], 1)
    s.x, s.x_scale, s.x_rows = s.x[0], s.x_scale[0], x_rows
    if case["path"] == "product":
        s.w, s.w_scale = _weights(g, E_loc, case["n"], k)
        s.y = torch.empty((rows, case["n"]), device=DEV, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32)
        s.ws = torch.empty(2 ** 26, dtype=torch.uint8, device=DEV)
        return
    inter = case["inter"]
    s.w1, s.s1 = _weights(g, E_loc, inter, k)
    s.w3, s.s3 = _weights(g, E_loc, inter, k)
    s.w2, s.s2 = _weights(g, E_loc, k, inter)
    s.y = torch.empty((rows, k), device=DEV, dtype=torch.bfloat16)
    s.ws = torch.empty(2 * rows * inter + 2 ** 26, dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    g = _gen(seed)
    s = types.SimpleNamespace(path=case["path"], case=case)
    if case["path"] in ("route", "grad"):
        _prepare_routing(s, g, case)
    elif case["path"] == "quantise":
        shape = (case["batch"], case["rows"], case["cols"])
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s.x = torch.randn(shape, generator=g, device=DEV).to(dtype)
        # channels of different size, as activations and weights have them
        s.x *= torch.exp(torch.randn(case["cols"], generator=g, device=DEV)).to(dtype)
        s.q = torch.empty(shape, dtype=F8, device=DEV)
        s.scale = torch.empty((shape[0], -(-shape[1] // case["block_rows"]), shape[2] // B), device=DEV)
    else:
        _prepare_product(s, g, case)
    return s


# ------------------------------------------------------------------ the plain form
def _scores(s):
    """Scores in 64 bits; experts that are switched off, and tokens that are masked, have none."""
    x = s.logits.double()
    on = s.logits > -math.inf
    if s.token_mask is not None:
        on = on & (s.token_mask != 0)[:, None]
    if s.case["kind"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-x))
    else:
        top = torch.where(on, x, -math.inf).amax(1, keepdim=True)
        e = torch.where(on, torch.exp(x - top), 0.0)
        score = e / e.sum(1, keepdim=True)
    return torch.where(on, score, 0.0), on


def _plain_route(s):
    c = s.case
    T, E, k, G = c["T"], c["E"], c["k"], c["n_groups"]
    score, on = _scores(s)
    biased = score if s.bias is None else score + s.bias.double()
    key = torch.where(on, s.logits.double() if s.bias is None else biased, -1e300)
    if c["topk_groups"] < G:
        first = torch.where(on, biased, -math.inf).view(T, G, E // G).sort(dim=2, descending=True).values
        first = first[:, :, :c["group_top"]]
        total = torch.where(first > -math.inf, first, 0.0).sum(2)
        total = torch.where(first[:, :, 0] > -math.inf, total, -math.inf)
        chosen = total.sort(dim=1, descending=True, stable=True).indices[:, :c["topk_groups"]]
        open_ = torch.zeros((T, G), dtype=torch.bool, device=DEV).scatter_(1, chosen, True)
        key = torch.where(open_.repeat_interleave(E // G, 1), key, -math.inf)
    idx = key.sort(dim=1, descending=True, stable=True).indices[:, :k]
    live = on.gather(1, idx)
    q = score.gather(1, idx)
    total = q.sum(1, keepdim=True)
    share = torch.where(total > 0, q / total, 0.0)
    dev = s.expert_rank.long()[idx]
    keep = live
    if c["p"] > 0:
        own_rank = torch.arange(T, device=DEV)[:, None] // (T // c["R"])
        cost = torch.where(dev // c["node"] != own_rank // c["node"], 5.0, 1.0)
        same = (dev[:, :, None] == dev[:, None, :]) & live[:, None, :] & live[:, :, None]
        a = (same * share[:, None, :]).sum(2)
        earlier = torch.ones((k, k), dtype=torch.bool, device=DEV).tril(-1)
        first = live & ~(same & earlier).any(2)
        ratio = torch.where(dev == own_rank, math.inf, a / cost)
        ratio = torch.where(first, ratio, -math.inf)
        by_dev = dev.sort(dim=1, stable=True).indices
        order = by_dev.gather(1, ratio.gather(1, by_dev).sort(dim=1, descending=True, stable=True).indices)
        ranked = torch.where(first, a, 0.0).gather(1, order)
        before = ranked.cumsum(1) - ranked
        p = torch.tensor(c["p"], dtype=torch.float32).double().item()
        kept_rank = first.gather(1, order) & (before < 1.0 - p)
        kept = torch.zeros_like(live).scatter(1, order, kept_rank)
        keep = live & (same & kept[:, None, :]).any(2)
    q = torch.where(keep, q, 0.0)
    total = q.sum(1, keepdim=True) if c["normalise"] else torch.ones((T, 1), dtype=torch.float64, device=DEV)
    w = torch.where(total > 0, c["scale"] * q / total, 0.0).float()
    mask = torch.zeros(T, dtype=torch.int64, device=DEV)
    for d in range(c["R"]):
        mask |= (keep & (dev == d)).any(1).long() << d
    return dict(idx=idx.to(torch.int32), w=w, keep=keep.to(torch.uint8), mask=mask)


def _plain_grad(s):
    c = s.case
    kept = s.keep != 0
    g = torch.where(kept, s.w * s.d_w, 0.0)
    total = g.sum(1, keepdim=True)
    idx = s.idx.long()
    x = s.logits.gather(1, idx)
    d = torch.zeros((c["T"], c["E"]), device=DEV)
    if c["normalise"]:
        slot = g - torch.where(kept, s.w, 0.0) * (total / c["scale"])
    else:
        slot = g
        if c["kind"] == "softmax":
            top = s.logits.amax(1, keepdim=True)
            e = torch.exp(s.logits - top)
            d = torch.where(kept.any(1, keepdim=True), -total * e / e.sum(1, keepdim=True), 0.0)
    if c["kind"] == "sigmoid":
        slot = slot / (1.0 + torch.exp(x))
    d = d.scatter_add(1, idx, torch.where(kept, slot, 0.0))
    if s.d_add is not None:
        d = d + s.d_add
    return d.to(s.d_logits.dtype)


def _plain_quantise(x, block_rows):
    """Codes and scales: the least power of two (from 2^-126 on) with which a block's largest value fits e4m3."""
    batch, rows, cols = x.shape
    pad = torch.nn.functional.pad(x.float(), (0, 0, 0, -rows % block_rows))
    pad = pad.view(batch, -1, block_rows, cols // B, B)
    bits = pad.abs().amax((2, 4)).view(torch.int32)
    exponent = ((bits + 0x1FFFFF) >> 23).sub(8).clamp(min=1)
    scale = (exponent << 23).view(torch.float32)
    q = (pad / scale[:, :, None, :, None]).to(F8)
    return q.view(batch, -1, cols)[:, :rows].contiguous(), scale


def _values(q, scale, block_rows):
    """What codes and scales stand for, in fp32."""
    full = scale.repeat_interleave(block_rows, -2)[..., :q.shape[-2], :].repeat_interleave(B, -1)
    return q.float() * full


def _plain_product(s, x, scale, w, w_scale):
    x = _values(x, scale, 1)
    return torch.cat([x[a:a + n] @ _values(w[e], w_scale[e], B).t()
                      for e, (a, n) in enumerate(zip(_starts(s.counts), s.counts))])


def _starts(counts):
    return [sum(counts[:i]) for i in range(len(counts))]


def _plain(s):
    if s.path == "route":
        return _plain_route(s)
    if s.path == "grad":
        return _plain_grad(s)
    if s.path == "quantise":
        q, scale = _plain_quantise(s.x, s.case["block_rows"])
        return dict(q=q, scale=scale)
    x, scale = s.x, s.x_scale
    if s.row_src is not None:
        x, scale = x.view(torch.uint8)[s.row_src.long()].view(F8), scale[s.row_src.long()]
    if s.path == "product":
        return _plain_product(s, x, scale, s.w, s.w_scale).to(s.y.dtype)
    gate = _plain_product(s, x, scale, s.w1, s.s1)
    h = gate / (1.0 + torch.exp(-gate)) * _plain_product(s, x, scale, s.w3, s.s3)
    h, scale = _plain_quantise(h[None], 1)
    return _plain_product(s, h[0], scale[0], s.w2, s.s2).to(s.y.dtype)


# ------------------------------------------------------------------ the package's calls
def _own(s):
    from paper_2607_05116_amd import capi
    c = s.case
    if s.path == "route":
        capi.cap_route_scores(s.topo, s.logits, s.options, c["p"], s.idx, s.w, s.keep, s.mask)
        return dict(idx=s.idx, w=s.w, keep=s.keep, mask=s.mask)
    if s.path == "grad":
        dt = capi.CAP_DTYPE_BF16 if c["out"] == "bf16" else capi.CAP_DTYPE_F32
        capi.cap_route_scores_grad(c["T"], c["k"], c["E"], s.logits, s.idx, s.keep, s.w, s.d_w, s.options, s.d_add, dt,
                                   s.d_logits)
        return s.d_logits
    if s.path == "quantise":
        dt = capi.CAP_DTYPE_BF16 if c["dtype"] == "bf16" else capi.CAP_DTYPE_F32
        capi.cap_quantise_fp8(dt, c["batch"], c["rows"], c["cols"], c["block_rows"], s.x, s.q, s.scale)
        return dict(q=s.q, scale=s.scale)
    if s.path == "product":
        dt = capi.CAP_DTYPE_BF16 if c["out"] == "bf16" else capi.CAP_DTYPE_F32
        capi.cap_product_fp8(dt, c["E_loc"], c["n"], c["kdim"], c["rows"], s.x, s.x_scale, s.x_rows, s.row_src,
                             s.offsets, s.w, s.w_scale, s.y, s.ws)
        return s.y
    capi.cap_expert_ffn_fp8(c["E_loc"], c["d"], c["inter"], c["rows"], s.x, s.x_scale, s.x_rows, s.row_src, s.offsets,
                            s.w1, s.s1, s.w3, s.s3, s.w2, s.s2, s.y, s.ws)
    return s.y


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["path"] in ("route", "grad"):
        T, E, k = case["T"], case["E"], case["k"]
        if case["path"] == "route":
            return dict(bytes=4.0 * T * E + T * (9.0 * k + 8) + 4.0 * E + (T if case["masked"] else 0),
                        flops=12.0 * T * E)
        full = case["kind"] == "softmax" and not case["normalise"]      # every logit is read, else the chosen ones
        some = 0 if case["kind"] == "softmax" else 4.0 * T * k
        return dict(bytes=(2.0 if case["out"] == "bf16" else 4.0) * T * E + (4.0 * T * E if case["add"] else 0)
                    + (4.0 * T * E if full else some) + 13.0 * T * k, flops=(8.0 if full else 1.0) * T * E)
    if case["path"] == "quantise":
        n = float(case["batch"]) * case["rows"] * case["cols"]
        scales = 4.0 * case["batch"] * -(-case["rows"] // case["block_rows"]) * (case["cols"] // B)
        return dict(bytes=n * (3 if case["dtype"] == "bf16" else 5) + scales, flops=3.0 * n)
    rows, x_rows = case["rows"], min(case["x_rows"] or case["rows"], case["rows"])
    used = sum(1 for n in _rows_of_experts(case) if n)
    if case["path"] == "product":
        n, k = case["n"], case["kdim"]
        out = 2.0 if case["out"] == "bf16" else 4.0
        return dict(bytes=x_rows * k * (1 + 4 / B) + used * (float(n) * k + 4 * -(-n // B) * (k // B)) + out * rows * n,
                    flops=_flops(case))
    d, inter = case["d"], case["inter"]
    return dict(bytes=x_rows * d * (1 + 4 / B) + used * 3.0 * d * inter + 2.0 * rows * d, flops=_flops(case))


# ------------------------------------------------------------------ the same in 64 bits, from the definitions
def _exact_route(s):
    """By counting: a group or an expert is taken if fewer than that many come before it."""
    c = s.case
    T, E, k, G, R = c["T"], c["E"], c["k"], c["n_groups"], c["R"]
    out = [[], [], [], []]
    for t0 in range(0, T, 1024):
        x = s.logits[t0:t0 + 1024].double()
        n = len(x)
        on = x > -math.inf
        if s.token_mask is not None:
            on = on & s.token_mask[t0:t0 + 1024].bool()[:, None]
        off = x.masked_fill(~on, -math.inf)
        score = torch.sigmoid(off) if c["kind"] == "sigmoid" else torch.softmax(off, 1).nan_to_num(0.0)
        biased = score if s.bias is None else score + s.bias.double()
        group = torch.arange(E, device=DEV) // (E // G)
        open_ = torch.ones((n, E), dtype=torch.bool, device=DEV)
        if c["topk_groups"] < G:
            total = torch.full((n, G), -math.inf, dtype=torch.float64, device=DEV)
            for i in range(G):
                v = biased[:, group == i].masked_fill(~on[:, group == i], -math.inf)
                best = v.topk(min(c["group_top"], v.shape[1]), 1).values
                total[:, i] = torch.where(best[:, 0] > -math.inf, best.masked_fill(best == -math.inf, 0.0).sum(1), -math.inf)
            i = torch.arange(G, device=DEV)
            ahead = (total[:, :, None] > total[:, None, :]) | \
                ((total[:, :, None] == total[:, None, :]) & (i[:, None] < i[None, :]))
            open_ = (ahead.sum(1) < c["topk_groups"])[:, group]
        key = x if s.bias is None else biased
        # classes: experts that are on, then those off, then those of closed groups
        rank = on.long() + open_.long() * 2
        rank = torch.where(open_, rank, 0)
        key = torch.where(on & open_, key, 0.0)
        e = torch.arange(E, device=DEV)
        idx = torch.zeros((n, k), dtype=torch.long, device=DEV)
        for a in range(0, n, 128):
            b = min(n, a + 128)
            before = (rank[a:b, :, None] > rank[a:b, None, :]) | ((rank[a:b, :, None] == rank[a:b, None, :]) & (
                (key[a:b, :, None] > key[a:b, None, :])
                | ((key[a:b, :, None] == key[a:b, None, :]) & (e[:, None] < e[None, :]))))
            place = before.sum(1)
            token, expert = (place < k).nonzero(as_tuple=True)
            idx[a + token, place[token, expert]] = expert
        # pruning over all devices at once
        live, q = on.gather(1, idx), score.gather(1, idx)
        share = q / q.sum(1, keepdim=True)
        share = torch.where(live, share.nan_to_num(0.0), 0.0)
        dev = s.expert_rank.long()[idx]
        a = torch.zeros((n, R), dtype=torch.float64, device=DEV).scatter_add_(1, dev, share)
        there = torch.zeros((n, R), device=DEV).scatter_add_(1, dev, live.float()) > 0
        kept = there
        if c["p"] > 0:
            own_rank = torch.arange(t0, t0 + n, device=DEV) // (T // R)
            d = torch.arange(R, device=DEV)
            cost = 1.0 + 4.0 * (d[None, :] // c["node"] != own_rank[:, None] // c["node"]).double()
            worth = a / cost
            worth[d[None, :] == own_rank[:, None]] = math.inf
            worth[~there] = -math.inf
            ahead = (worth[:, :, None] > worth[:, None, :]) | \
                ((worth[:, :, None] == worth[:, None, :]) & (d[:, None] < d[None, :]))
            before = (ahead * a[:, :, None]).sum(1)
            kept = there & (before < 1.0 - torch.tensor(c["p"], dtype=torch.float32).double().item())
        keep = live & kept.gather(1, dev)
        q = torch.where(keep, q, 0.0)
        total = q.sum(1, keepdim=True) if c["normalise"] else torch.ones_like(q[:, :1])
        out[0].append(idx.to(torch.int32))
        out[1].append((c["scale"] * q / total).nan_to_num(0.0))
        out[2].append(keep.to(torch.uint8))
        out[3].append((kept.long() << torch.arange(R, device=DEV)).sum(1))
    return dict(zip(("idx", "w", "keep", "mask"), (torch.cat(v) for v in out)))


def _exact_grad(s):
    c = s.case
    x = s.logits.double().requires_grad_(True)
    score = torch.sigmoid(x) if c["kind"] == "sigmoid" else torch.softmax(x, 1)
    kept = s.keep != 0
    q = torch.where(kept, score.gather(1, s.idx.long()), 0.0)
    gates = c["scale"] * q
    if c["normalise"]:
        total = q.sum(1, keepdim=True)
        gates = gates / torch.where(total > 0, total, 1.0)
    (torch.where(kept, gates, 0.0) * s.d_w.double()).sum().backward()
    return x.grad if s.d_add is None else x.grad + s.d_add.double()


def _round_e4m3(v):
    """The nearest e4m3 value, ties to even: steps of 2^-3 of the binade, of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))).clamp(max=8.0) - 3.0)
    return (torch.round(v / step) * step).clamp(-TOP, TOP)


def _exact_quantise(x, block_rows):
    rows = x.shape[-2]
    top = x.abs().unflatten(-1, (-1, B)).amax(-1)
    if block_rows > 1:
        top = torch.nn.functional.pad(top, (0, 0, 0, -rows % block_rows)).unflatten(-2, (-1, block_rows)).amax(-2)
    scale = torch.exp2(torch.ceil(torch.log2(top / TOP)).clamp(min=-126.0))
    scale = torch.where(top > TOP * scale, 2.0 * scale, scale)            # the logarithm's own rounding
    scale = torch.where((top <= TOP * scale / 2) & (scale > 2.0 ** -126), scale / 2, scale)
    full = scale.repeat_interleave(B, -1)
    if block_rows > 1:
        full = full.repeat_interleave(block_rows, -2)[..., :rows, :]
    return _round_e4m3(x / full), scale, full


def exact(case, seed):
    s = prepare(case, seed)
    if s.path == "route":
        return _exact_route(s)
    if s.path == "grad":
        return _exact_grad(s)
    if s.path == "quantise":
        q, scale, _ = _exact_quantise(s.x.double(), case["block_rows"])
        return dict(q=q, scale=scale)

    def weights(w, scale, e):
        full = scale[e].double().repeat_interleave(B, 0).repeat_interleave(B, 1)
        return w[e].double() * full[:w.shape[1]]

    x = s.x.double() * s.x_scale.double().repeat_interleave(B, 1)
    out, a = [], 0
    for e, n in enumerate(s.counts):
        rows = x[a:a + n] if s.row_src is None else x[s.row_src[a:a + n].long()]
        a += n
        if s.path == "product":
            out.append(rows @ weights(s.w, s.w_scale, e).t())
            continue
        h = torch.nn.functional.silu(rows @ weights(s.w1, s.s1, e).t()) * (rows @ weights(s.w3, s.s3, e).t())
        q, _, full = _exact_quantise(h, 1)
        out.append((q * full) @ weights(s.w2, s.s2, e).t())
    return torch.cat(out)
